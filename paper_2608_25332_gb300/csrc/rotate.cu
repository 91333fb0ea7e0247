// Norm and position rotation of packed rows' queries and keys, on the way into the paged cache or
// not, and rows in and out of pages of 4 bits.
//
// Rotation. Pair i of a head is (x_i, x_{i+64}); at position p (of the pair's axis) it turns by the
// angle p f_i. The frequencies come as turns a position in units of 2^-64, so p times that, modulo
// 2^64, is the angle modulo a full turn, exact to 2^-33 of one after dropping the lower half, for any
// 32-bit position; 32-bit floats of p f_i would be off by 0.06 rad at position 10^6. Sine and cosine
// are taken of the signed fraction (sincospif).
//
// 4 bits. Each 32 values of a head share a bf16 scale d = -e / 8, e the one of largest magnitude (the
// positive of two), so that e itself is code 0 exactly where it fits 8 bits; codes n = round(x (1/d))
// + 8, at most 15, stand for d (n - 8). Reciprocal, product and rounding are each one fp32 operation
// rounded to nearest, so codes are the same wherever they are computed. From 2^100 on (and for
// infinities and NaN) d is NaN, below 2^-123 it is 0. Layout of a page of one head: its rows' codes,
// 64 bytes each, then their scales, 8 bytes each; the 16 bits at place 4 g + q of a row's codes are
// values 32 q + 4 g .. + 3, the first in the lowest bits. (So eight bytes hold four values of each
// group, and a lane of the decoding kernel gets whole groups' operands from what it loads.)
//
// A warp handles up to kIter times four heads of a row: eight lanes a head, lane l with values 8 l
// .. + 7 and 64 + 8 l .. + 7, which are pairs. A row's 64 sines are worked out two a lane and passed
// round. Bound by HBM (each value is read and written once) from about a thousand rows on, below
// that by the launch.
#include "common.cuh"
#include "kernels.h"

namespace provip {
namespace {

constexpr int kThr = 256;

// 8 + 8 values of a head's lane
template <typename T>
struct Raw;
template <>
struct Raw<__nv_bfloat16> {
  uint4 u[2];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    u[0] = *reinterpret_cast<const uint4*>(p);
    u[1] = *reinterpret_cast<const uint4*>(p + 64);
  }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const {
    *reinterpret_cast<uint4*>(p) = u[0];
    *reinterpret_cast<uint4*>(p + 64) = u[1];
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t w[4] = {u[h].x, u[h].y, u[h].z, u[h].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[8 * h + 2 * i] = __uint_as_float(w[i] << 16);
        x[8 * h + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ void set(const float* x) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x[8 * h + 2 * i], x[8 * h + 2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
      }
      u[h] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
};
template <>
struct Raw<float> {
  float4 u[4];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = *reinterpret_cast<const float4*>(p + 64 * (i >> 1) + 4 * (i & 1));
  }
  __device__ __forceinline__ void store(float* p) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(p + 64 * (i >> 1) + 4 * (i & 1)) = u[i];
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[4 * i] = u[i].x;
      x[4 * i + 1] = u[i].y;
      x[4 * i + 2] = u[i].z;
      x[4 * i + 3] = u[i].w;
    }
  }
  __device__ __forceinline__ void set(const float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  }
};

// The scale of a group whose eight values a lane are x, over the four lanes that hold it.
__device__ __forceinline__ float group_scale(const float* x, uint16_t& bits) {
  // magnitude above the sign: the positive of two equal ones is the larger
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(x[i]);
    m = max(m, ((b << 1) | (b >> 31)) ^ 1u);
  }
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  const float mag = __uint_as_float(m >> 1);
  float d = mag * 0.125f;
  if (m & 1u) d = -d;
  __nv_bfloat16 h = __float2bfloat16_rn(d);
  bits = *reinterpret_cast<const uint16_t*>(&h);
  if (!(mag < 0x1p100f)) bits = 0x7fff;
  if (mag < 0x1p-123f) bits = 0;
  return __uint_as_float((uint32_t)bits << 16);
}
// codes of eight values: four of them in each half of the result
__device__ __forceinline__ uint32_t group_codes(const float* x, float d) {
  const float r = d == 0.f ? 0.f : __frcp_rn(d);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = fminf(fmaxf(__fmul_rn(x[i], r), -8.f), 7.f);
    w |= (__float_as_uint(__fadd_rn(y, 12582920.f)) & 15u) << (4 * i);  // 3 * 2^22 + 8: the sum's unit is 1
  }
  return w;
}

// A head's row (eight lanes with 16 values each) into its place in 4-bit pages.
__device__ __forceinline__ void store4bit(const float* x, uint8_t* codes, uint8_t* scales, int l, bool on) {
  uint16_t b0, b1;
  const float d0 = group_scale(x, b0), d1 = group_scale(x + 8, b1);
  const uint32_t c0 = group_codes(x, d0), c1 = group_codes(x + 8, d1);
  // lanes 0-3 hold groups 0 and 2, lanes 4-7 groups 1 and 3 of the same places: one keeps its lower
  // four values of each, the other its upper ones
  const bool up = l & 4;
  const uint32_t give = up ? __byte_perm(c0, c1, 0x5410) : __byte_perm(c0, c1, 0x7632);
  const uint32_t got = __shfl_xor_sync(0xffffffffu, give, 4);
  const uint32_t d_got = __shfl_xor_sync(0xffffffffu, (uint32_t)b0 | (uint32_t)b1 << 16, 4);
  uint2 w;
  if (!up) {
    w.x = __byte_perm(c0, got, 0x5410);
    w.y = __byte_perm(c1, got, 0x7610);
  } else {
    w.x = __byte_perm(got, c0, 0x7610);
    w.y = __byte_perm(got, c1, 0x7632);
  }
  if (!on) return;
  *reinterpret_cast<uint2*>(codes + (2 * (l & 3) + (up ? 1 : 0)) * 8) = w;
  if (l == 0) *reinterpret_cast<uint2*>(scales) = make_uint2((uint32_t)b0 | d_got << 16, (uint32_t)b1 | (d_got & 0xffff0000u));
}

// a head's place in 4-bit pages: its codes; its scales lie *scales bytes behind them
__device__ __forceinline__ size_t place4(long long slot, int h, int H_kv, int page_shift, size_t* scales) {
  const long long page = slot >> page_shift, row = slot - (page << page_shift);
  *scales = ((size_t)kCodes4 << page_shift) - row * (kCodes4 - 8);
  return ((size_t)(page * H_kv + h) << page_shift) * kRow4 + (size_t)row * kCodes4;
}

template <typename T, int ITER>
__global__ void __launch_bounds__(kThr) rotate_kernel(const __grid_constant__ RotateArgs a, int per_row, int q_items, int k_items) {
  const int lane = threadIdx.x & 31, l = lane & 7;
  const long long item = (long long)blockIdx.x * (kThr / 32) + (threadIdx.x >> 5);
  const long long t = item / per_row;
  if (t >= a.T) return;
  if (a.n_rows) {
    const int n = *a.n_rows;
    if (item == 0 && lane == 0 && (n < 0 || n > a.T)) set_error(a.err, kErrBadDeviceArg);
    if (t >= n) return;
  }
  int part = (int)(item - t * per_row);
  // 0: queries, 1: keys, 2: values
  const int kind = part < q_items ? 0 : part < q_items + k_items ? 1 : 2;
  if (kind == 1) part -= q_items;
  if (kind == 2) part -= q_items + k_items;
  const int H = kind == 0 ? a.H_q : a.H_kv, h0 = part * (4 * ITER) + (lane >> 3);
  const T* src = kind == 0 ? static_cast<const T*>(a.Q) + t * a.q_stride
                 : kind == 1 ? static_cast<const T*>(a.K) + t * a.k_stride
                             : static_cast<const T*>(a.V) + t * a.v_stride;
  Raw<T> raw[ITER];
#pragma unroll
  for (int i = 0; i < ITER; ++i)
    if (h0 + 4 * i < H) raw[i].load(src + (size_t)(h0 + 4 * i) * kHeadDim + l * 8);
  // where the row goes
  T* out = kind == 0 ? static_cast<T*>(a.q_out) + t * a.qo_stride
           : kind == 1 && a.k_out ? static_cast<T*>(a.k_out) + t * a.ko_stride : nullptr;
  long long slot = -1;
  if (kind != 0 && a.slot_map) {
    slot = a.slot_map[t];
    if (slot >= a.n_slots) {
      if (lane == 0) set_error(a.err, kErrBadDeviceArg);
      slot = -1;
    }
  }
  if (out == nullptr && slot < 0) return;
  uint8_t* pages = static_cast<uint8_t*>(kind == 1 ? a.k_pages : a.v_pages);
  const bool turn = a.turn && kind != 2;
  float c[8], s[8];
  if (turn) {
    float s2[2], c2[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int p = 2 * lane + i;
      const long long at = a.pos[a.axis[p] * a.pos_stride + t];
      const int part_turn = (int)(((unsigned long long)at * a.turns[p]) >> 32);  // 2^-32 of a turn, signed
      sincospif((float)part_turn * 0x1p-31f, &s2[i], &c2[i]);
      s2[i] *= a.factor;
      c2[i] *= a.factor;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s[i] = __shfl_sync(0xffffffffu, s2[i & 1], 4 * l + (i >> 1));
      c[i] = __shfl_sync(0xffffffffu, c2[i & 1], 4 * l + (i >> 1));
    }
  }
  const T* w = turn ? static_cast<const T*>(kind == 0 ? a.wq : a.wk) : nullptr;
  float g[16];
  if (w) {
    Raw<T> r;
    r.load(w + l * 8);
    r.get(g);
  }
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    const int h = h0 + 4 * i;
    const bool on = h < H;
    if (h - (lane >> 3) >= H) break;  // (the whole warp)
    if (turn || a.four) {
      float x[16];
      if (on) {
        raw[i].get(x);
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.f;
      }
      if (turn) {
        if (w) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
          for (int o = 1; o < 8; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
          const float r = rsqrtf(ss * (1.f / kHeadDim) + a.eps);
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] = x[e] * r * g[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = x[e], v = x[e + 8];
          x[e] = u * c[e] - v * s[e];
          x[e + 8] = v * c[e] + u * s[e];
        }
        raw[i].set(x);
        raw[i].get(x);  // the cache takes in what k_out holds
      }
      if (a.four && slot >= 0 && kind != 0) {
        size_t scales;
        uint8_t* at = pages + place4(slot, on ? h : 0, a.H_kv, a.page_shift, &scales);
        store4bit(x, at, at + scales, l, on);
      }
    }
    if (on && out) raw[i].store(out + (size_t)h * kHeadDim + l * 8);
    if (on && !a.four && slot >= 0)
      raw[i].store(reinterpret_cast<T*>(pages) + ((size_t)slot * a.H_kv + h) * kHeadDim + l * 8);
  }
}

template <typename T, int ITER>
cudaError_t rotate_go(const RotateArgs& a, cudaStream_t s) {
  const int per = 4 * ITER;
  const int q = a.Q ? (a.H_q + per - 1) / per : 0, k = a.K ? (a.H_kv + per - 1) / per : 0, v = a.V ? (a.H_kv + per - 1) / per : 0;
  const long long items = (long long)(q + k + v) * a.T;
  rotate_kernel<T, ITER><<<(unsigned)((items + kThr / 32 - 1) / (kThr / 32)), kThr, 0, s>>>(a, q + k + v, q, k);
  return cudaGetLastError();
}

// ---------------------------------------------------------------------------
// rows out of 4-bit pages: the same eight lanes a head. Lane l's values lie in 16 bytes of codes,
// which lanes l and l + 4 share.
// ---------------------------------------------------------------------------
template <typename T, int ITER>
__global__ void __launch_bounds__(kThr) read4_kernel(const __grid_constant__ Read4Args a, int per_row) {
  const int lane = threadIdx.x & 31, l = lane & 7;
  const long long item = (long long)blockIdx.x * (kThr / 32) + (threadIdx.x >> 5);
  const long long t = item / per_row;
  if (t >= a.T) return;
  const int h0 = (int)(item - t * per_row) * (4 * ITER) + (lane >> 3);
  const long long slot = a.slot_map[t];
  if (slot < 0) return;
  if (slot >= a.n_slots) {
    if (lane == 0) set_error(a.err, kErrBadDeviceArg);
    return;
  }
  const uint8_t* pages = blockIdx.y ? a.v_pages : a.k_pages;
  T* out = static_cast<T*>(blockIdx.y ? a.v_out : a.k_out) + t * (blockIdx.y ? a.v_stride : a.k_stride);
  uint4 codes[ITER];
  uint2 scales[ITER];
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    if (h0 + 4 * i >= a.H_kv) continue;
    size_t behind;
    const uint8_t* at = pages + place4(slot, h0 + 4 * i, a.H_kv, a.page_shift, &behind);
    codes[i] = *reinterpret_cast<const uint4*>(at + (l & 3) * 16);
    scales[i] = *reinterpret_cast<const uint2*>(at + behind);
  }
  const uint32_t half = l & 4 ? 0x7632 : 0x5410;
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    if (h0 + 4 * i >= a.H_kv) continue;
    const uint32_t c[2] = {__byte_perm(codes[i].x, codes[i].z, half), __byte_perm(codes[i].y, codes[i].w, half)};
    const uint32_t b[2] = {scales[i].x, scales[i].y};
    float x[16];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float d = __uint_as_float(l & 4 ? b[k] & 0xffff0000u : b[k] << 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[8 * k + e] = d * (float)((int)((c[k] >> (4 * e)) & 15u) - 8);
    }
    Raw<T> r;
    r.set(x);
    r.store(out + (size_t)(h0 + 4 * i) * kHeadDim + l * 8);
  }
}

template <typename T, int ITER>
cudaError_t read4_go(const Read4Args& a, cudaStream_t s) {
  const int per_row = (a.H_kv + 4 * ITER - 1) / (4 * ITER);
  const long long items = (long long)per_row * a.T;
  read4_kernel<T, ITER><<<dim3((unsigned)((items + kThr / 32 - 1) / (kThr / 32)), 2), kThr, 0, s>>>(a, per_row);
  return cudaGetLastError();
}

}  // namespace

cudaError_t rotate_launch(const RotateArgs& a, int dtype, cudaStream_t s) {
  return dtype == 0 ? rotate_go<float, 1>(a, s) : rotate_go<__nv_bfloat16, 1>(a, s);
}

cudaError_t read4_launch(const Read4Args& a, int dtype, cudaStream_t s) {
  return dtype == 0 ? read4_go<float, 1>(a, s) : read4_go<__nv_bfloat16, 1>(a, s);
}

}  // namespace provip
