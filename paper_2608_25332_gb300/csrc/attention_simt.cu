// Attention behind the pruning on the CUDA cores: fp32 tensors (FFMA, no reduced
// precision), and bf16 on request.
#include "attention.cuh"

namespace provip {
namespace {

// ---------------------------------------------------------------------------
// tiles of 64 rows by 64 keys
//
// A CTA holds 64 packed rows of a key/value head (Q in shared memory as fp32, 8 rows of
// scores and of the output in each thread's registers) and passes over its keys once in
// tiles of 64 with a running maximum and sum. Bound by the FFMA pipe: pairs of products in one
// instruction, a thread's 8 x 4 scores take 12 16-byte loads from shared memory per 64 of
// them, its 8 x 8 outputs 16 per 128. P takes the place of the keys it came from, so that two
// CTAs fit an SM and one multiplies while the other waits for its next tile (cp.async).
// ---------------------------------------------------------------------------
constexpr int kBM = 64, kBN = 64, kThr = 128;
constexpr int kPitch = kHeadDim + 4;  // floats a row of Q and K: rows 4 banks apart, 16 bytes aligned
constexpr int kVPitch = kHeadDim;     // V is read along its rows
constexpr int kPPitch = kBN + 4;
constexpr size_t kTileSmem = sizeof(float) * ((size_t)(kBM + kBN) * kPitch + (size_t)kBN * kVPitch);
static_assert(kBM * kPPitch <= kBN * kPitch, "P fits in the place of K");

// four elements of a row; zeros for a null source
__device__ __forceinline__ void fill4(float* dst, const float* src, bool have) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(have ? 16 : 0) : "memory");
}
__device__ __forceinline__ void fill4(float* dst, const __nv_bfloat16* src, bool have) {
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (have) load4(src, v);
  *reinterpret_cast<float4*>(dst) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void fill_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void fill_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ void unpair(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}

// blockIdx: x row tile, y = key/value head * parts + part, z sequence. PREFIX: the rows of
// every request's token against the prefix alone (paged), parts part0 .. part0 + n - 1.
template <typename T, bool PREFIX>
__global__ void __launch_bounds__(kThr, 2) attn_tile_simt(const __grid_constant__ AttnArgs a, int part0, int n_parts) {
  extern __shared__ __align__(16) float sm[];
  float* qs = sm;
  float* ks = qs + kBM * kPitch;
  float* ps = ks;
  float* vs = ks + kBN * kPitch;
  const int R = a.H_q / a.H_kv, g = blockIdx.y / n_parts, part = blockIdx.y % n_parts, b = blockIdx.z;
  AttnSeq s;
  if (PREFIX) {
    s.q0 = 0;
    s.q_len = a.B;
    s.k_len = 0;
    s.k0 = 0;
    s.pages = nullptr;
    s.ok = true;
  } else {
    s = attn_seq(a, b);
    if (!s.ok && threadIdx.x == 0) set_error(a.err, kErrBadDeviceArg);
  }
  const int n_rows = s.q_len * R, r0 = blockIdx.x * kBM;
  if (r0 >= n_rows) return;
  const int rows = min(kBM, n_rows - r0);
  const int P = a.prefix_len;
  // keys of the list that some row of the tile sees, and this part's share of their tiles
  const int n_keys = P + (PREFIX ? 0 : attn_visible(a, s.q_len, s.k_len, (r0 + rows - 1) / R));
  const int n_tiles = (n_keys + kBN - 1) / kBN, per = (n_tiles + n_parts - 1) / n_parts;
  const int k_lo = min(part * per * kBN, n_keys), k_hi = min((part + 1) * per * kBN, n_keys);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;  // rows ty*8.., columns tx + 16 j / 4 tx..

  // Keys k0 .. k0 + 63 of the list (past k_hi: zeros) to dst, from this lane's column of the
  // prefix's and the own rows (a key of the list is added to either base; worked out per row, the
  // addresses had cost as much as a third of the products).
  const size_t col = (size_t)g * kHeadDim + lane * 4;
  const T *k_pre = static_cast<const T*>(a.Kp) + col, *v_pre = static_cast<const T*>(a.Vp) + col;
  const T* k_own = static_cast<const T*>(a.K) + col + (s.k0 - P) * a.k_stride;
  const T* v_own = static_cast<const T*>(a.V) + col + (s.k0 - P) * a.v_stride;
  auto fill = [&](float* dst, int pitch, int k0, bool v) {
    const T *pre = v ? v_pre : k_pre, *own = v ? v_own : k_own;
    const long long sp = v ? a.vp_stride : a.kp_stride, so = v ? a.v_stride : a.k_stride;
#pragma unroll 4
    for (int j = warp; j < kBN; j += kThr / 32) {
      const int key = k0 + j;
      const bool have = key < k_hi;
      const T* src = pre;
      if (PREFIX) {
        if (have) src = pre + attn_slot(a, a.prefix_table, key) * sp;
      } else if (have) {
        src = key < P ? pre + key * sp : own + key * so;
      }
      fill4(dst + j * pitch + lane * 4, have ? src : static_cast<const T*>(a.Q), have);
    }
    fill_commit();
  };
  for (int r = warp; r < kBM; r += kThr / 32) {
    const bool have = r < rows;
    const int t = have ? (r0 + r) / R : 0, h = g * R + (have ? (r0 + r) % R : 0);
    fill4(qs + r * kPitch + lane * 4, static_cast<const T*>(a.Q) + (size_t)(s.q0 + t) * a.q_stride + (size_t)h * kHeadDim + lane * 4,
          have);
  }
  if (k_lo < k_hi) {
    fill(ks, kPitch, k_lo, false);  // (with Q)
    fill(vs, kVPitch, k_lo, true);
  }
  int lim[8];  // keys of the list that each row sees
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + ty * 8 + i;
    lim[i] = r < n_rows ? P + (PREFIX ? 0 : attn_visible(a, s.q_len, s.k_len, r / R)) : 0;
  }
  uint64_t o2[8][4];
  float m[8], l[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) o2[i][j] = 0;
  }
  for (int k0 = k_lo; k0 < k_hi; k0 += kBN) {
    fill_wait<1>();
    __syncthreads();  // K is there
    uint64_t x2[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) x2[i][j] = 0;
#pragma unroll 2
    for (int d = 0; d < kHeadDim; d += 4) {
      ulonglong2 kv[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const ulonglong2*>(ks + (tx + 16 * j) * kPitch + d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const ulonglong2 qv = *reinterpret_cast<const ulonglong2*>(qs + (ty * 8 + i) * kPitch + d);
#pragma unroll
        for (int j = 0; j < 4; ++j) x2[i][j] = fma_pair(qv.y, kv[j].y, fma_pair(qv.x, kv[j].x, x2[i][j]));
      }
    }
    float x[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float e, f;
        unpair(x2[i][j], e, f);
        x[i][j] = e + f;
      }
    __syncthreads();  // K is read: P takes its place
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i][j] = k0 + tx + 16 * j < min(lim[i], k_hi) ? __fmul_rn(x[i][j], a.scale_log2) : -INFINITY;  // as in the maximum
        mx = fmaxf(mx, x[i][j]);
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float mn = fmaxf(m[i], mx), base = mn == -INFINITY ? 0.f : mn;
      const float r = exp2f(m[i] - base);
      m[i] = mn;
      float t = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = exp2f(x[i][j] - base);
        t += p;
        ps[(ty * 8 + i) * kPPitch + tx + 16 * j] = p;
      }
      l[i] = l[i] * r + t;
      const uint64_t r2 = pair(r, r);
#pragma unroll
      for (int j = 0; j < 4; ++j) o2[i][j] = fma_pair(o2[i][j], r2, 0);
    }
    fill_wait<0>();
    __syncthreads();  // V is there (and a row's probabilities, written and read by the same 16 lanes)
#pragma unroll 1
    for (int k = 0; k < kBN; k += 4) {
      float4 p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = *reinterpret_cast<const float4*>(ps + (ty * 8 + i) * kPPitch + k);
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const ulonglong2 v0 = *reinterpret_cast<const ulonglong2*>(vs + (k + kk) * kVPitch + tx * 4);
        const ulonglong2 v1 = *reinterpret_cast<const ulonglong2*>(vs + (k + kk) * kVPitch + 64 + tx * 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float w = kk == 0 ? p[i].x : kk == 1 ? p[i].y : kk == 2 ? p[i].z : p[i].w;
          const uint64_t w2 = pair(w, w);
          o2[i][0] = fma_pair(w2, v0.x, o2[i][0]);
          o2[i][1] = fma_pair(w2, v0.y, o2[i][1]);
          o2[i][2] = fma_pair(w2, v1.x, o2[i][2]);
          o2[i][3] = fma_pair(w2, v1.y, o2[i][3]);
        }
      }
    }
    __syncthreads();  // P and V are read
    if (k0 + kBN < k_hi) {
      fill(ks, kPitch, k0 + kBN, false);
      fill(vs, kVPitch, k0 + kBN, true);
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");  // a part without keys leaves Q's copies under way
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int w = 8; w > 0; w >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
    const int r = r0 + ty * 8 + i;
    const bool live = r < n_rows;
    const int t = r / R, h = g * R + r % R;
    const size_t row = (size_t)(s.q0 + t) * a.H_q + h;
    bool fine = true;
    const float den = l[i] == 0.f ? 1.f : l[i];
    float o[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) unpair(o2[i][j], o[2 * j], o[2 * j + 1]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      o[j] /= den;
      fine = fine && isfinite(o[j]);
    }
    float lse = l[i] == 0.f ? -INFINITY : m[i] + log2f(l[i]);
    fine = fine || isnan(l[i]);  // a NaN score, which masked ones are not: every element is NaN
    if (live && fine) {
      if (a.n_part > 1) {
        float* po = a.part_o + ((size_t)(part0 + part) * a.T_q * a.H_q + row) * kHeadDim;
        store4(po + tx * 4, o);
        store4(po + 64 + tx * 4, o + 4);
        if (tx == 0) a.part_lse[(size_t)(part0 + part) * a.T_q * a.H_q + row] = lse;
      } else {
        if (l[i] == 0.f && lim[i] > 0) {
          lse = NAN;  // every score is -inf: 0 / 0, as the formula has it
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] = NAN;
        }
        T* op = static_cast<T*>(a.out) + (size_t)(s.q0 + t) * a.o_stride + (size_t)h * kHeadDim;
        store4(op + tx * 4, o);
        store4(op + 64 + tx * 4, o + 4);
        if (tx == 0 && a.lse) a.lse[row] = lse * kLn2;
      }
    }
    // rows that are not finite, one at a time by the whole warp
    __syncwarp();  // their stores above come first
    unsigned bad = __ballot_sync(0xffffffffu, live && !fine);
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
      if (!((bad >> (16 * half)) & 0xffffu)) continue;
      const int rb = __shfl_sync(0xffffffffu, r, 16 * half), tb = rb / R, hb = g * R + rb % R;
      const int hi = min(__shfl_sync(0xffffffffu, lim[i], 16 * half), k_hi);
      float ob[4];
      float lb = attn_row_plain<T>(a, s, P, tb, hb, k_lo, hi, lane * 4, ob, nullptr);
      const size_t rowb = (size_t)(s.q0 + tb) * a.H_q + hb;
      if (a.n_part > 1) {
        store4(a.part_o + ((size_t)(part0 + part) * a.T_q * a.H_q + rowb) * kHeadDim + lane * 4, ob);
        if (lane == 0) a.part_lse[(size_t)(part0 + part) * a.T_q * a.H_q + rowb] = lb;
      } else {
        if (lb == -INFINITY) lb = ob[0] = ob[1] = ob[2] = ob[3] = NAN;
        store4(static_cast<T*>(a.out) + (size_t)(s.q0 + tb) * a.o_stride + (size_t)hb * kHeadDim + lane * 4, ob);
        if (lane == 0 && a.lse) a.lse[rowb] = lb * kLn2;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// one token against its request's own pages
//
// A CTA takes one part of a request's keys for up to RT heads of a group. Each warp
// passes over its keys, four elements of a row per lane and four keys' rows in flight, with
// its own running maximum and sum; the warps are joined in shared memory at the end. Bound
// by HBM: every key and
// value row is read once for the RT heads.
// ---------------------------------------------------------------------------
constexpr int kDecThr = 256;

// blockIdx: x = key/value head * heads' tiles + tile, y part, z request
template <typename T, int RT>
__global__ void __launch_bounds__(kDecThr) attn_token_simt(const __grid_constant__ AttnArgs a, int n_own) {
  constexpr int kUnroll = 4, kWarps = kDecThr / 32;
  const int R = a.H_q / a.H_kv, n_rt = (R + RT - 1) / RT;
  const int g = blockIdx.x / n_rt, h0 = g * R + (blockIdx.x % n_rt) * RT, part = blockIdx.y, b = blockIdx.z;
  const int nh = min(RT, g * R + R - h0);
  const AttnSeq s = attn_seq(a, b);
  if (!s.ok && threadIdx.x == 0) set_error(a.err, kErrBadDeviceArg);
  const int per = (s.k_len + n_own - 1) / n_own;
  const int k_lo = min(part * per, s.k_len), k_hi = min(k_lo + per, s.k_len);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  float q[RT][4], o[RT][4], m[RT], l[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) q[r][e] = o[r][e] = 0.f;
    if (r < nh) {
      load4(static_cast<const T*>(a.Q) + (size_t)b * a.q_stride + (size_t)(h0 + r) * kHeadDim + lane * 4, q[r]);
#pragma unroll
      for (int e = 0; e < 4; ++e) q[r][e] *= a.scale_log2;
    }
  }
  for (int j0 = k_lo + warp * kUnroll; j0 < k_hi; j0 += kWarps * kUnroll) {
    float k[kUnroll][4], v[kUnroll][4];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int j = min(j0 + u, k_hi - 1);
      load4(attn_own_row<T>(a, s, false, j, g) + lane * 4, k[u]);
      load4(attn_own_row<T>(a, s, true, j, g) + lane * 4, v[u]);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float x[kUnroll], mx = m[r];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        x[u] = warp_sum(fmaf(q[r][0], k[u][0], fmaf(q[r][1], k[u][1], fmaf(q[r][2], k[u][2], q[r][3] * k[u][3]))));
        if (j0 + u >= k_hi) x[u] = -INFINITY;
        mx = fmaxf(mx, x[u]);
      }
      const float base = mx == -INFINITY ? 0.f : mx, c = exp2f(m[r] - base);
      m[r] = mx;
      l[r] *= c;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[r][e] *= c;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (j0 + u < k_hi) {
          const float p = exp2f(x[u] - base);
          l[r] += p;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[r][e] = fmaf(p, v[u][e], o[r][e]);
        }
      }
    }
  }
  __shared__ float so[kWarps][kHeadDim];
  __shared__ float sml[kWarps][2];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    if (r >= nh) break;
    __syncthreads();
    store4(&so[warp][lane * 4], o[r]);
    if (lane == 0) {
      sml[warp][0] = m[r];
      sml[warp][1] = l[r];
    }
    __syncthreads();
    if (threadIdx.x < kHeadDim) {
      float mx = -INFINITY, acc = 0.f, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, sml[w][0]);
      const float base = mx == -INFINITY ? 0.f : mx;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float c = exp2f(sml[w][0] - base);
        sum = fmaf(sml[w][1], c, sum);
        if (sml[w][1] != 0.f) acc = fmaf(so[w][threadIdx.x], c, acc);
      }
      const size_t row = (size_t)b * a.H_q + h0 + r;
      float val = sum == 0.f ? 0.f : acc / sum, lse = sum == 0.f ? -INFINITY : mx + log2f(sum);
      const bool odd = sum != 0.f && isfinite(sum) && !isfinite(val);
      if (__any_sync(0xffffffffu, odd)) {
        const float v = attn_element_again<T>(a, b, h0 + r, k_lo, k_hi, threadIdx.x, odd, nullptr);
        val = odd ? v : val;
      }
      if (a.n_part > 1) {
        a.part_o[((size_t)part * a.T_q * a.H_q + row) * kHeadDim + threadIdx.x] = val;
        if (threadIdx.x == 0) a.part_lse[(size_t)part * a.T_q * a.H_q + row] = lse;
      } else {
        if (sum == 0.f && s.k_len > 0) val = lse = NAN;  // every score is -inf
        T* op = static_cast<T*>(a.out) + (size_t)b * a.o_stride + (size_t)(h0 + r) * kHeadDim;
        op[threadIdx.x] = static_cast<T>(val);
        if (threadIdx.x == 0 && a.lse) a.lse[row] = lse * kLn2;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// parts of a row -> the row: a warp per (token, head)
// ---------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256) attn_join(const __grid_constant__ AttnArgs a) {
  pdl_wait_prior();
  const int lane = threadIdx.x & 31;
  const long long n_rows = (long long)a.T_q * a.H_q, row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= n_rows) return;
  const int t = (int)(row / a.H_q), h = (int)(row % a.H_q);
  int n_vis = a.prefix_len;
  if (a.paged) {
    n_vis += attn_seq(a, t).k_len;
  } else {
    // the sequence that holds token t; rows outside every sequence are left untouched
    bool found = false;
    for (int b0 = 0; b0 < a.B && !found; b0 += 32) {
      AttnSeq s;
      bool mine = false;
      if (b0 + lane < a.B) {
        s = attn_seq(a, b0 + lane);
        mine = s.ok && t >= s.q0 && t - s.q0 < s.q_len;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, mine);
      if (hit) {
        found = true;
        n_vis += __shfl_sync(0xffffffffu, mine ? attn_visible(a, s.q_len, s.k_len, t - s.q0) : 0, __ffs(hit) - 1);
      }
    }
    if (!found) return;
  }
  Joined s = {{0.f, 0.f, 0.f, 0.f}, 0.f, -INFINITY};
  join_parts(
      s, a.n_part, [&](int p) { return a.part_lse[(size_t)p * n_rows + row]; },
      [&](int p) { return a.part_o + ((size_t)p * n_rows + row) * kHeadDim; });
  const float den = s.w == 0.f ? (n_vis > 0 ? NAN : 1.f) : s.w;  // every score -inf: 0 / 0, as the formula has it
#pragma unroll
  for (int e = 0; e < 4; ++e) s.o[e] /= den;
  store4(static_cast<T*>(a.out) + (size_t)t * a.o_stride + (size_t)h * kHeadDim + lane * 4, s.o);
  if (lane == 0 && a.lse)
    a.lse[row] = s.w == 0.f ? (n_vis > 0 ? NAN : -INFINITY) : s.lse() * kLn2;
}

template <typename T, bool PREFIX>
cudaError_t tile_launch(const AttnArgs& a, dim3 grid, int part0, int n_parts, cudaStream_t s) {
  static std::atomic<bool> configured[64];  // per device, zero-initialised
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 0 && dev < 64 && !configured[dev]) {
    cudaError_t e = cudaFuncSetAttribute(attn_tile_simt<T, PREFIX>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)kTileSmem);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  attn_tile_simt<T, PREFIX><<<grid, kThr, kTileSmem, s>>>(a, part0, n_parts);
  return cudaGetLastError();
}

template <typename T>
cudaError_t token_launch(const AttnArgs& a, int n_own, cudaStream_t s) {
  const int R = a.H_q / a.H_kv;
  // heads that share a key row's load: as many as the group has, four at most
  const dim3 grid((unsigned)(a.H_kv * (R == 1 ? 1 : R == 2 ? 1 : (R + 3) / 4)), (unsigned)n_own, (unsigned)a.B);
  if (R == 1)
    attn_token_simt<T, 1><<<grid, kDecThr, 0, s>>>(a, n_own);
  else if (R == 2)
    attn_token_simt<T, 2><<<grid, kDecThr, 0, s>>>(a, n_own);
  else
    attn_token_simt<T, 4><<<grid, kDecThr, 0, s>>>(a, n_own);
  return cudaGetLastError();
}

template <typename T>
cudaError_t prompt_simt(const AttnArgs& a, cudaStream_t s) {
  const long long rows = (long long)a.q_len_max * (a.H_q / a.H_kv);
  return tile_launch<T, false>(a, dim3((unsigned)((rows + kBM - 1) / kBM), (unsigned)(a.H_kv * a.n_part), (unsigned)a.B),
                               0, a.n_part, s);
}
template <typename T>
cudaError_t decode_simt(const AttnArgs& a, int n_own, cudaStream_t s) {
  cudaError_t e = n_own > 0 ? token_launch<T>(a, n_own, s) : cudaSuccess;
  if (e != cudaSuccess || a.n_part == n_own) return e;
  const long long rows = (long long)a.B * (a.H_q / a.H_kv);
  const int n = a.n_part - n_own;
  return tile_launch<T, true>(a, dim3((unsigned)((rows + kBM - 1) / kBM), (unsigned)(a.H_kv * n), 1), n_own, n, s);
}

}  // namespace

cudaError_t attn_prompt_simt_launch(const AttnArgs& a, int dtype, cudaStream_t s) {
  return dtype == 0 ? prompt_simt<float>(a, s) : prompt_simt<__nv_bfloat16>(a, s);
}

cudaError_t attn_decode_simt_launch(const AttnArgs& a, int n_own, int dtype, cudaStream_t s) {
  return dtype == 0 ? decode_simt<float>(a, n_own, s) : decode_simt<__nv_bfloat16>(a, n_own, s);
}

cudaError_t attn_join_launch(const AttnArgs& a, int dtype, cudaStream_t s) {
  const dim3 grid((unsigned)(((long long)a.T_q * a.H_q + 7) / 8));
  return dtype == 0 ? launch_pdl(attn_join<float>, grid, dim3(256), 0, s, a)
                    : launch_pdl(attn_join<__nv_bfloat16>, grid, dim3(256), 0, s, a);
}

}  // namespace provip
