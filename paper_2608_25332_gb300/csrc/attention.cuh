// Attention behind the pruning: what its kernels share.
//
// Rows. The rows of one key/value head g are (token, query head of g's group) pairs,
// token-major: row r of a sequence is token r / R, head g * R + r % R with R = H_q / H_kv.
// All R heads of a group read the same keys, so a tile of packed rows reads them once.
//
// Keys. A sequence's keys are a prefix that every sequence of the call shares, then its
// own; token i of q_len sees every prefix key and, of its own k_len keys, all of them or
// (causal) the first k_len - q_len + i + 1 (the last token sees the last key). Keys come as
// rows of a tensor or as slots of a paged cache (page_size rows a page, the pages of a
// sequence listed in its block table).
//
// Sums. Scores are kept in the base-2 domain: s = q . k * log2(e) * scale; a row's partial
// result over a part of its keys is o = sum 2^(s - m) v / l and its base-2 log-sum-exp
// m + log2 l, so parts join as sum_p w_p o_p / sum_p w_p with w_p = 2^(lse_p - max).
#pragma once

#include "common.cuh"
#include "kernels.h"

namespace provip {

constexpr float kLn2 = 0.693147180559945309f;

// where a sequence's queries, keys and values lie (validated)
struct AttnSeq {
  int q0, q_len;         // first query token, tokens
  int k_len;             // own keys
  long long k0;          // first own key row (contiguous keys)
  const int* pages;      // own block table (paged keys)
  bool ok;
};

__device__ __forceinline__ AttnSeq attn_seq(const AttnArgs& a, int b) {
  AttnSeq s;
  s.pages = nullptr;
  s.k0 = 0;
  if (a.paged) {  // one token per request
    s.q0 = b;
    s.q_len = 1;
    s.k_len = a.k_len[b];
    s.pages = a.block_table + (size_t)b * a.max_pages;
    s.ok = s.k_len >= 0 && s.k_len <= a.k_len_max && s.k_len <= (long long)a.max_pages * a.page_size;
    if (!s.ok) s.k_len = 0;  // reported; the shared prefix is still attended to
  } else {
    s.q0 = a.q_start[b];
    s.q_len = a.q_len[b];
    s.k_len = a.k_len[b];
    s.k0 = a.k_start[b];
    s.ok = s.q0 >= 0 && s.q_len >= 0 && s.q_len <= a.q_len_max && s.q_len <= a.T_q - s.q0 && s.k0 >= 0 &&
           s.k_len >= 0 && s.k_len <= a.k_len_max && s.k_len <= a.T_k - s.k0;
    if (!s.ok) s.q_len = 0;  // reported; the sequence's rows are left untouched
  }
  return s;
}

// own keys that token i sees
__device__ __forceinline__ int attn_visible(const AttnArgs& a, int q_len, int k_len, int i) {
  return a.causal ? min(max(k_len - q_len + i + 1, 0), k_len) : k_len;
}

// row of the pool (paged) that holds key j of a page list; a page outside the pool is
// reported and read as page 0
__device__ __forceinline__ long long attn_slot(const AttnArgs& a, const int* pages, int j) {
  int p = __ldg(pages + (j >> a.page_shift));
  if ((unsigned)p >= (unsigned)a.n_pages) {
    set_error(a.err, kErrBadDeviceArg);
    p = 0;
  }
  return ((long long)p << a.page_shift) + (j & (a.page_size - 1));
}

// row pointers of prefix key j and of own key j, key/value head g
template <typename T>
__device__ __forceinline__ const T* attn_prefix_row(const AttnArgs& a, bool v, int j, int g) {
  const T* base = static_cast<const T*>(v ? a.Vp : a.Kp) + (size_t)g * kHeadDim;
  return base + (a.paged ? attn_slot(a, a.prefix_table, j) : (long long)j) * (v ? a.vp_stride : a.kp_stride);
}
template <typename T>
__device__ __forceinline__ const T* attn_own_row(const AttnArgs& a, const AttnSeq& s, bool v, int j, int g) {
  const T* base = static_cast<const T*>(v ? a.V : a.K) + (size_t)g * kHeadDim;
  return base + (a.paged ? attn_slot(a, s.pages, j) : s.k0 + j) * (v ? a.v_stride : a.k_stride);
}

template <typename T>
__device__ __forceinline__ void load4(const T* p, float* o);
template <>
__device__ __forceinline__ void load4<float>(const float* p, float* o) {
  const float4 v = __ldg(reinterpret_cast<const float4*>(p));
  o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
}
template <>
__device__ __forceinline__ void load4<__nv_bfloat16>(const __nv_bfloat16* p, float* o) {
  const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
  const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.x));
  const float2 y = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u.y));
  o[0] = x.x; o[1] = x.y; o[2] = y.x; o[3] = y.y;
}
__device__ __forceinline__ void store4(float* p, const float* v) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float* v) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(v[0], v[1]), y = __floats2bfloat162_rn(v[2], v[3]);
  uint2 u;
  u.x = *reinterpret_cast<const uint32_t*>(&x);
  u.y = *reinterpret_cast<const uint32_t*>(&y);
  *reinterpret_cast<uint2*>(p) = u;
}

// One row over keys [lo, hi) of its list (prefix keys, then own ones), key by key, by one
// warp: the plain definition, which no key outside the range touches. The tile kernels
// weigh every value row of a tile, the hidden ones by zero, and divide at the end; zero times an
// infinite or NaN value is NaN, and a sum of values may pass the largest float where their mean does
// not, so a row that did not come out finite is computed again here, with its sums in 64 bits. A lane
// gets E elements from col on (four: 4 lane); returns the base-2 log-sum-exp (-inf: no weight at
// all). beat, if any, is given the time every 64 keys.
template <typename T, int E = 4>
__device__ __noinline__ float attn_row_plain(const AttnArgs& a, const AttnSeq& s, int n_prefix, int token, int h,
                                             int lo, int hi, int col, float* o, unsigned long long* beat) {
  const int lane = threadIdx.x & 31, g = h / (a.H_q / a.H_kv);
  float q[4], m = -INFINITY;
  double l = 0., acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.;
  load4(static_cast<const T*>(a.Q) + (size_t)(s.q0 + token) * a.q_stride + (size_t)h * kHeadDim + lane * 4, q);
  for (int j = lo; j < hi; ++j) {
    float k[4], v[E];
    if (beat && lane == 0 && ((j - lo) & 63) == 0) *static_cast<volatile unsigned long long*>(beat) = global_timer_ns();
    const bool pre = j < n_prefix;
    load4((pre ? attn_prefix_row<T>(a, false, j, g) : attn_own_row<T>(a, s, false, j - n_prefix, g)) + lane * 4, k);
    const T* pv = (pre ? attn_prefix_row<T>(a, true, j, g) : attn_own_row<T>(a, s, true, j - n_prefix, g)) + col;
    if (E == 4)
      load4(pv, v);
    else
      v[0] = (float)*pv;
    // (rounded as the maximum is: no fma with the subtraction below)
    const float x = __fmul_rn(warp_sum(fmaf(q[0], k[0], fmaf(q[1], k[1], fmaf(q[2], k[2], q[3] * k[3])))), a.scale_log2);
    if (x == -INFINITY) continue;
    if (x > m) {
      const float r = exp2f(m - x);
      m = x;
      l *= r;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= r;
    }
    const double w = exp2f(x - m);
    l += w;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fma(w, (double)v[e], acc[e]);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = l == 0. ? 0.f : (float)(acc[e] / l);
  return l == 0. ? -INFINITY : m + log2f((float)l);
}

// Element col (a lane's own) of a request's row over its own keys [lo, hi), where it came out infinite
// or NaN (odd) though the row's weights are finite. With values that are all finite it was their sum
// that passed the largest float: the element with its sums in 64 bits. Else what is not finite among
// them shows: NaN, or infinities of both signs, as NaN, of one sign as that. By a warp, the head's
// (paged keys); returns the element.
template <typename T>
__device__ __noinline__ float attn_element_again(const AttnArgs& a, int b, int h, int lo, int hi, int col, bool odd,
                                                 unsigned long long* beat) {
  const AttnSeq s = attn_seq(a, b);
  float v = 0.f;
  bool up = false, down = false;  // (both for NaN)
#pragma unroll 8
  for (int j = lo; j < hi; ++j) {
    if (beat && (threadIdx.x & 31) == 0 && ((j - lo) & 1023) == 0)
      *static_cast<volatile unsigned long long*>(beat) = global_timer_ns();
    const float x = (float)attn_own_row<T>(a, s, true, j, h / (a.H_q / a.H_kv))[col];
    up = up || !(x < INFINITY);
    down = down || !(x > -INFINITY);
  }
  if (__any_sync(0xffffffffu, odd && !up && !down)) attn_row_plain<T, 1>(a, s, 0, 0, h, lo, hi, col, &v, beat);
  return up && down ? NAN : up ? INFINITY : down ? -INFINITY : v;
}

// Weighs n more parts of a row and adds them to s (by one warp): lse(p) in base 2 and 128 floats at part(p).
// A round's loads are all under way before the first is used. The weights carry a factor of 2^-10:
// a row has fewer than 2^10 parts (128 shared out, or 64 and the pieces of 304 spans; over 4-bit pages a
// prefix's 256 and 512), so they add up to less than one and no sum of parts passes the largest float where their mean does not.
constexpr float kJoinUnit = 1.f / 1024.f;
struct Joined {
  float o[4], w, m;  // weighted sum of lane's elements, sum of the weights 2^(lse - m) kJoinUnit
  __device__ __forceinline__ float lse() const { return m + log2f(w * (1.f / kJoinUnit)); }  // (base 2)
};
template <int kRound = 12, typename Lse, typename Part>
__device__ __forceinline__ void join_parts(Joined& s, int n, Lse lse, Part part) {
  const int lane = threadIdx.x & 31;
  for (int p0 = 0; p0 < n; p0 += kRound) {
    float x[kRound];
    float4 v[kRound];
#pragma unroll
    for (int p = 0; p < kRound; ++p) {
      x[p] = -INFINITY;
      v[p] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (p0 + p < n) {
        x[p] = lse(p0 + p);
        v[p] = *reinterpret_cast<const float4*>(part(p0 + p) + lane * 4);
      }
    }
    float mn = s.m;
#pragma unroll
    for (int p = 0; p < kRound; ++p) mn = fmaxf(mn, x[p]);
    const float base = mn == -INFINITY ? 0.f : mn, c = exp2f(s.m - base);
    s.m = mn;
    s.w *= c;
#pragma unroll
    for (int e = 0; e < 4; ++e) s.o[e] *= c;
#pragma unroll
    for (int p = 0; p < kRound; ++p) {
      const float w = exp2f(x[p] - base) * kJoinUnit;
      s.w += w;
      if (w != 0.f) {  // (a part without weight may hold anything)
        s.o[0] = fmaf(w, v[p].x, s.o[0]);
        s.o[1] = fmaf(w, v[p].y, s.o[1]);
        s.o[2] = fmaf(w, v[p].z, s.o[2]);
        s.o[3] = fmaf(w, v[p].w, s.o[3]);
      }
    }
  }
}

}  // namespace provip
