// One token per request against pages of 4 bits.
//
// A row of 128 values is d_q (n - 8) with codes n and a scale d_q for each 32 values q (rotate.cu),
// so with integers c = n - 8, exact in bf16,
//   score_t = sum_q dk_{t,q} (Q_q . c_{t,q})        o_q = sum_t (p_t dv_{t,q}) c_{t,q}:
// scales stay outside the first product and go into the weights of the second, and no value is
// ever rounded to 16 bits. Both products run on mma.sync (m16n8k16, bf16 in, fp32 sums) with the codes
// as the 16-row operand A straight from registers: eight query rows ("columns") are enough to fill
// it, where a tcgen05 product would want the expanded codes written to shared memory first, four times
// the bytes that come from HBM, on every one of them.
//   S[16 keys x 8] = 4 groups x 2 MMAs over the dims, then 4 FMAs a score with dk
//   O^T[16 dims x 8] += 8 MMAs over 16 keys, with P dv from S's registers by movmatrix (a transpose)
// The order of the dims in the codes (rotate.cu) is such that a lane's 16 bytes of a key hold whole
// MMA operands of one group each: shifts and masks, no exchange. A nibble becomes c as bf16 in a mask-or
// to 128 + n and a subtraction, two at a time.
//
// Work: a CTA of four warps takes a part of one (request, key/value head)'s keys, or of the prefix's for
// a block of rows of all requests; a warp 32 keys at a time, from a ring of its own that bulk copies
// fill (a page of one head is contiguous), with its own softmax state; the four join in shared memory.
// Rows of several parts are joined by a second kernel. No maximum is looked for while no score passes
// the one before by 2^10. Statistics and sums are fp32; P dv is rounded to bf16 (2^-8 of each weight at most;
// values then add up as integers times weights). For fp32 queries the queries and P dv are split into
// three bf16 pieces each (24 bits), a product each.
#include "attention.cuh"

namespace provip {
namespace {

constexpr int kWarps = 4, kThr = kWarps * 32;
constexpr int kStep = 32;      // keys of a warp's stage
constexpr int kStages = 3;
constexpr int kCodeBytes = kStep * kCodes4, kScaleBytes = kStep * 8;
constexpr int kStageBytes = 2 * (kCodeBytes + kScaleBytes);  // K codes, V codes, K scales, V scales
constexpr int kRing = kStages * kStageBytes;
constexpr size_t kSmem = (size_t)kWarps * kRing;

__device__ __forceinline__ void mma_bf16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
// nibble t of each half of x, less 8, as bf16
__device__ __forceinline__ uint32_t code_pair(uint32_t x, int t) {
  const uint32_t v = ((x >> (4 * t)) & 0x000f000fu) | 0x43004300u;  // 128 + n
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), __bfloat162bfloat162(__float2bfloat16_rn(136.f)));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// x, y as kP bf16 pairs that add up to them
template <int kP>
__device__ __forceinline__ void split2(float x, float y, uint32_t* r) {
#pragma unroll
  for (int p = 0; p < kP; ++p) {
    r[p] = pack2(x, y);
    if (p + 1 < kP) {
      x -= lo_f(r[p]);
      y -= hi_f(r[p]);
    }
  }
}

// which query row a column is (-1: none), as b * H_q + h
template <bool kPrefix>
__device__ __forceinline__ int column_row(const AttnArgs& a, int R, int block, int g, int c) {
  if (!kPrefix) return c < R ? block * a.H_q + g * R + c : -1;  // (block: the request; g, R: virtual)
  const long long r = (long long)block + c;
  if (r >= (long long)a.B * R) return -1;
  const int b = (int)(r / R);
  return b * a.H_q + g * R + (int)(r - (long long)b * R);
}

template <typename T, int NT, bool kPrefix>
__global__ void __launch_bounds__(kThr) attn4_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ Attn4Plan plan) {
  constexpr int kP = sizeof(T) == 4 ? 3 : 1;  // bf16 pieces of a query and of a weight
  constexpr int C = 8 * NT;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t full[kWarps][kStages];
  __shared__ float s_m[kWarps][C], s_l[kWarps][C];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
  if (kPrefix) pdl_allow_next();

  // this CTA's piece: heads run fastest (their parts of a page lie next to each other)
  const int R = kPrefix ? a.group : a.group / plan.n_cut, H = kPrefix ? a.H_kv : a.H_kv * plan.n_cut;
  const long long id = blockIdx.x;
  const int head = (int)(id % H);
  const int n_part = kPrefix ? plan.n_pre : plan.n_own, part = (int)(id / H % n_part);
  const int unit = (int)(id / H / n_part);
  const int block = kPrefix ? unit * C : unit;
  const int kv_head = kPrefix ? head : head / plan.n_cut;
  int len = a.prefix_len;
  const int* table = a.prefix_table;
  if (!kPrefix) {
    len = a.k_len[unit];
    if (len < 0 || len > a.k_len_max || len > (long long)a.max_pages * a.page_size) {
      if (part == 0 && threadIdx.x == 0) set_error(a.err, kErrBadDeviceArg);
      len = 0;
    }
    table = a.block_table + (size_t)unit * a.max_pages;
  }
  const int part_keys = kPrefix ? plan.pre_keys : plan.own_keys;
  const int k_lo = part * part_keys;
  const bool alone = !kPrefix && a.prefix_len == 0 && len <= part_keys;  // the row's only part
  if (len <= k_lo && !(alone && part == 0)) {
    if (!kPrefix && blockIdx.x == 0 && threadIdx.x == 0) pdl_wait_prior();
    return;
  }
  const int k_hi = k_lo + min(len - k_lo, part_keys);
  const int n_steps = max(0, (k_hi - k_lo + kStep - 1) / kStep);

  if (lane == 0) {
    for (int s = 0; s < kStages; ++s) mbar_init(&full[warp][s], 1);
    fence_mbar_init();
  }
  __syncwarp();

  // loads: a lane per copy of a stage (up to four boxes of rows, K and V codes and scales of each)
  const int box = min(a.page_size, kStep), kind = lane & 3, my_box = lane >> 2;
  const uint32_t ring = smem_u32(smem) + warp * kRing;
  const uint32_t dst = (kind < 2 ? kind * kCodeBytes + my_box * box * kCodes4
                                 : 2 * kCodeBytes + (kind - 2) * kScaleBytes + my_box * box * 8);
  const uint32_t bytes = box * (kind < 2 ? kCodes4 : 8);
  const uint8_t* pool = static_cast<const uint8_t*>(kind & 1 ? a.V : a.K);
  auto page_of = [&](int step) {
    const int k = k_lo + step * kStep + my_box * box;
    return my_box * box < kStep && step < n_steps && k < k_hi ? __ldg(table + (k >> a.page_shift)) : 0;
  };
  int page = page_of(warp);
  auto load = [&](int step, int stage) {  // (steps: this warp's, in order)
    const int k = k_lo + step * kStep, n = min(kStep, k_hi - k), boxes = (n + box - 1) / box;
    int p = page;
    page = page_of(step + kWarps);
    if (lane == 0) mbar_arrive_expect_tx(&full[warp][stage], (uint32_t)(boxes * box * kRow4 * 2));
    __syncwarp();
    if (my_box < boxes) {
      if ((unsigned)p >= (unsigned)a.n_pages) {
        set_error(a.err, kErrBadDeviceArg);
        p = 0;
      }
      const int row = (k + my_box * box) & (a.page_size - 1);
      const size_t base = ((size_t)((long long)p * a.H_kv + kv_head) << a.page_shift) * kRow4;
      const size_t at = kind < 2 ? (size_t)row * kCodes4 : ((size_t)kCodes4 << a.page_shift) + (size_t)row * 8;
      bulk_load(ring + stage * kStageBytes + dst, pool + base + at, bytes, smem_u32(&full[warp][stage]));
    }
    __syncwarp();
  };
  int issued = 0, used = 0;
#pragma unroll
  for (int s = 0; s < kStages; ++s) {
    const int step = warp + s * kWarps;
    if (step < n_steps) {
      load(step, s);
      ++issued;
    }
  }

  // queries: column g's dims 32 q + 8 j .. + 7, as B operands
  uint32_t qf[NT][kP][4][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = column_row<kPrefix>(a, R, block, head, nt * 8 + g);
    const T* qp = nullptr;
    if (row >= 0) {
      const int b = row / a.H_q;
      qp = static_cast<const T*>(a.Q) + (size_t)b * a.q_stride + (size_t)(row - b * a.H_q) * kHeadDim + 8 * j;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.f;
      if (qp) load8(qp + 32 * q, x);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        uint32_t r[kP];
        split2<kP>(x[t], x[t + 4], r);
#pragma unroll
        for (int p = 0; p < kP; ++p) qf[nt][p][q][t] = r[p];
      }
    }
  }

  float o[4][2][NT][4], m[NT][2], l[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      m[nt][c] = -INFINITY;
      l[nt][c] = 0.f;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[q][h][nt][e] = 0.f;
  }

  bool failed = false;
  int stage = 0;
  uint32_t phase = 0;
  for (int step = warp; step < n_steps; step += kWarps) {
    if (__any_sync(0xffffffffu, !mbar_wait(&full[warp][stage], phase, a.err))) {
      failed = true;
      break;
    }
    ++used;
    const uint8_t* st = smem + warp * kRing + stage * kStageBytes;
    const uint8_t *kc = st, *vc = st + kCodeBytes, *ks = st + 2 * kCodeBytes, *vs = ks + kScaleBytes;
    const int left = k_hi - k_lo - step * kStep;  // keys from this step's first on
    float s[2][NT][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const int r0 = mt * 16 + g, r1 = r0 + 8;
      const uint4 wa = *reinterpret_cast<const uint4*>(kc + r0 * kCodes4 + 16 * j);
      const uint4 wb = *reinterpret_cast<const uint4*>(kc + r1 * kCodes4 + 16 * j);
      const uint2 da = *reinterpret_cast<const uint2*>(ks + r0 * 8), db = *reinterpret_cast<const uint2*>(ks + r1 * 8);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t sel = q & 1 ? 0x7632 : 0x5410;
        const uint32_t xa = q < 2 ? __byte_perm(wa.x, wa.z, sel) : __byte_perm(wa.y, wa.w, sel);
        const uint32_t xb = q < 2 ? __byte_perm(wb.x, wb.z, sel) : __byte_perm(wb.y, wb.w, sel);
        uint32_t ca[4], cb[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          ca[t] = code_pair(xa, t);
          cb[t] = code_pair(xb, t);
        }
        const uint32_t ua = q < 2 ? da.x : da.y, ub = q < 2 ? db.x : db.y;
        const float fa = q & 1 ? hi_f(ua) : lo_f(ua), fb = q & 1 ? hi_f(ub) : lo_f(ub);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int p = kP - 1; p >= 0; --p) {
            mma_bf16(x, ca[0], cb[0], ca[1], cb[1], qf[nt][p][q][0], qf[nt][p][q][1]);
            mma_bf16(x, ca[2], cb[2], ca[3], cb[3], qf[nt][p][q][2], qf[nt][p][q][3]);
          }
          if (q == 0) {
            s[mt][nt][0] = x[0] * fa;
            s[mt][nt][1] = x[1] * fa;
            s[mt][nt][2] = x[2] * fb;
            s[mt][nt][3] = x[3] * fb;
          } else {
            s[mt][nt][0] = fmaf(x[0], fa, s[mt][nt][0]);
            s[mt][nt][1] = fmaf(x[1], fa, s[mt][nt][1]);
            s[mt][nt][2] = fmaf(x[2], fb, s[mt][nt][2]);
            s[mt][nt][3] = fmaf(x[3], fb, s[mt][nt][3]);
          }
        }
      }
    }
    // base 2, hidden keys out (rounded before a maximum is subtracted: no fma with that)
    bool raise = false;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool seen = mt * 16 + (e >> 1) * 8 + g < left;
          s[mt][nt][e] = seen ? __fmul_rn(s[mt][nt][e], a.scale_log2) : -INFINITY;
          raise = raise || s[mt][nt][e] > m[nt][e & 1] + 10.f;
        }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float x = fmaxf(fmaxf(s[0][nt][c], s[0][nt][c + 2]), fmaxf(s[1][nt][c], s[1][nt][c + 2]));
#pragma unroll
          for (int b = 4; b < 32; b <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, b));
          x = fmaxf(x, m[nt][c]);
          const float f = x == m[nt][c] ? 1.f : ex2_approx(m[nt][c] - x);
          m[nt][c] = x;
          l[nt][c] *= f;
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              o[q][h][nt][c] *= f;
              o[q][h][nt][c + 2] *= f;
            }
        }
    }
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float mm = m[nt][e & 1];
          const float p = ex2_approx(s[mt][nt][e] - (mm == -INFINITY ? 0.f : mm));
          s[mt][nt][e] = p;
          l[nt][e & 1] += p;
        }
    // (fp32: a step's sums start from zero and are added in fp32, as the MMAs' own sums truncate)
    float add[kP > 1 ? 4 : 1][2][NT][4];
    if (kP > 1) {
#pragma unroll
      for (int i = 0; i < 4 * 2 * NT * 4; ++i) (&add[0][0][0][0])[i] = 0.f;
    }
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const int r0 = mt * 16 + g, k0 = mt * 16 + 2 * j;
      // a row past the end has no scale, whatever lies there
      uint2 da = *reinterpret_cast<const uint2*>(vs + r0 * 8), db = *reinterpret_cast<const uint2*>(vs + (r0 + 8) * 8);
      if (r0 >= left) da = make_uint2(0u, 0u);
      if (r0 + 8 >= left) db = make_uint2(0u, 0u);
      uint2 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint2*>(vc + (k0 + (i >> 1) * 8 + (i & 1)) * kCodes4 + 8 * g);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t sel = q & 1 ? 0x7632 : 0x5410;
        const uint32_t ya = q < 2 ? __byte_perm(v[0].x, v[1].x, sel) : __byte_perm(v[0].y, v[1].y, sel);
        const uint32_t yb = q < 2 ? __byte_perm(v[2].x, v[3].x, sel) : __byte_perm(v[2].y, v[3].y, sel);
        uint32_t ca[4], cb[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          ca[t] = code_pair(ya, t);
          cb[t] = code_pair(yb, t);
        }
        const uint32_t ua = q < 2 ? da.x : da.y, ub = q < 2 ? db.x : db.y;
        const float fa = q & 1 ? hi_f(ua) : lo_f(ua), fb = q & 1 ? hi_f(ub) : lo_f(ub);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          uint32_t wa[kP], wb[kP];
          split2<kP>(s[mt][nt][0] * fa, s[mt][nt][1] * fa, wa);
          split2<kP>(s[mt][nt][2] * fb, s[mt][nt][3] * fb, wb);
#pragma unroll
          for (int p = kP - 1; p >= 0; --p) {
            const uint32_t b0 = transpose8x8(wa[p]), b1 = transpose8x8(wb[p]);
            mma_bf16(kP > 1 ? add[q][0][nt] : o[q][0][nt], ca[0], ca[1], cb[0], cb[1], b0, b1);
            mma_bf16(kP > 1 ? add[q][1][nt] : o[q][1][nt], ca[2], ca[3], cb[2], cb[3], b0, b1);
          }
        }
      }
    }
    if (kP > 1) {
#pragma unroll
      for (int i = 0; i < 4 * 2 * NT * 4; ++i) (&o[0][0][0][0])[i] += (&add[0][0][0][0])[i];
    }
    __syncwarp();  // every lane has read the stage
    const int next = step + kStages * kWarps;
    if (next < n_steps) {
      load(next, stage);
      ++issued;
    }
    if (++stage == kStages) {
      stage = 0;
      phase ^= 1;
    }
  }
  if (failed) {
    // copies still in flight into the block's shared memory: waited for once more, with a limit
    for (int i = used; i < issued; ++i) mbar_wait(&full[warp][i % kStages], (uint32_t)(i / kStages) & 1u, a.err);
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int b = 4; b < 32; b <<= 1) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], b);

  // the four warps' results: [warp][column][128] over the rings
  __syncthreads();
  float* so = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int col = nt * 8 + 2 * j + c;
      if (g == 0) {
        s_m[warp][col] = m[nt][c];
        s_l[warp][col] = l[nt][c];
      }
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(so + ((size_t)warp * C + col) * kHeadDim + 32 * q + 4 * g) =
            make_float4(o[q][0][nt][c], o[q][0][nt][c + 2], o[q][1][nt][c], o[q][1][nt][c + 2]);
    }
  __syncthreads();
  // a warp takes every fourth column, a lane four dims
  const size_t slot = (size_t)((kPrefix ? 0 : plan.n_pre) + part) * a.B * a.H_q;
  for (int col = warp; col < C; col += kWarps) {
    const int row = column_row<kPrefix>(a, R, block, head, col);
    if (row < 0) continue;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_m[w][col]);
    float L = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = s_m[w][col] == -INFINITY ? 0.f : ex2_approx(s_m[w][col] - M);
      const float4 v = *reinterpret_cast<const float4*>(so + ((size_t)w * C + col) * kHeadDim + 4 * lane);
      // (a warp without keys, or one whose scores are all -inf, has weight 0; a NaN one shows)
      if (s_m[w][col] == -INFINITY && !(s_l[w][col] != 0.f)) continue;
      L += s_l[w][col] * f;
      x[0] = fmaf(v.x, f, x[0]);
      x[1] = fmaf(v.y, f, x[1]);
      x[2] = fmaf(v.z, f, x[2]);
      x[3] = fmaf(v.w, f, x[3]);
    }
    const bool nil = L == 0.f;
    // no keys: 0 and -inf; keys whose scores are all -inf: 0 / 0, as the formula has it
    const float inv = nil ? (alone && len > 0 ? NAN : 0.f) : 1.f / L;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= inv;
    const float lse = nil ? (alone && len > 0 ? NAN : -INFINITY) : M + log2f(L);
    if (alone) {
      const int b = row / a.H_q;
      store4(static_cast<T*>(a.out) + (size_t)b * a.o_stride + (size_t)(row - b * a.H_q) * kHeadDim + 4 * lane, x);
      if (lane == 0 && a.lse) a.lse[row] = lse * kLn2;
    } else {
      store4(a.part_o + (slot + row) * kHeadDim + 4 * lane, x);
      if (lane == 0) a.part_lse[slot + row] = lse;
    }
  }
  // beside the prefix's kernel: the joining one waits for this one alone
  if (!kPrefix && blockIdx.x == 0 && threadIdx.x == 0) pdl_wait_prior();
}

// parts -> rows, a warp each
template <typename T>
__global__ void __launch_bounds__(256) attn4_join(const __grid_constant__ AttnArgs a, const __grid_constant__ Attn4Plan plan) {
  pdl_wait_prior();
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), n_rows = (long long)a.B * a.H_q;
  if (row >= n_rows) return;
  const int b = (int)(row / a.H_q);
  int len = a.k_len[b];
  if (len < 0 || len > a.k_len_max || len > (long long)a.max_pages * a.page_size) len = 0;
  if (a.prefix_len == 0 && len <= plan.own_keys) return;  // written by its only part
  const int n_own = plan.n_own > 0 ? (len + plan.own_keys - 1) / plan.own_keys : 0;
  Joined s = {{0.f, 0.f, 0.f, 0.f}, 0.f, -INFINITY};
  join_parts(
      s, plan.n_pre + n_own, [&](int p) { return a.part_lse[p * n_rows + row]; },
      [&](int p) { return a.part_o + (p * n_rows + row) * kHeadDim; });
  const float den = s.w == 0.f ? NAN : s.w;  // (there are keys: every score -inf is 0 / 0)
  float o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = s.o[e] / den;
  store4(static_cast<T*>(a.out) + (size_t)b * a.o_stride + (size_t)(row - (long long)b * a.H_q) * kHeadDim + lane * 4, o);
  if (lane == 0 && a.lse) a.lse[row] = s.w == 0.f ? NAN : s.lse() * kLn2;
}

template <typename T, int NT, bool kPrefix>
cudaError_t go(const AttnArgs& a, const Attn4Plan& plan, cudaStream_t s) {
  static std::atomic<bool> configured[64];  // per device, zero-initialised
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 0 && dev < 64 && !configured[dev]) {
    cudaError_t e = cudaFuncSetAttribute(attn4_kernel<T, NT, kPrefix>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  const long long rows = (long long)a.B * a.group;
  const long long ctas = kPrefix ? (rows + 8 * NT - 1) / (8 * NT) * a.H_kv * plan.n_pre
                                 : (long long)a.B * a.H_kv * plan.n_cut * plan.n_own;
  if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
  if (!kPrefix && plan.n_pre > 0)  // beside the prefix's kernel, whose results it does not read
    return launch_pdl(attn4_kernel<T, NT, kPrefix>, dim3((unsigned)ctas), dim3(kThr), kSmem, s, a, plan);
  attn4_kernel<T, NT, kPrefix><<<(unsigned)ctas, kThr, kSmem, s>>>(a, plan);
  return cudaGetLastError();
}

template <typename T>
cudaError_t run(const AttnArgs& a, const Attn4Plan& plan, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  constexpr int kWide = sizeof(T) == 4 ? 1 : 2;  // (fp32 at 16 columns spills registers)
  if (plan.n_pre > 0) e = plan.pre_cols == 16 ? go<T, kWide, true>(a, plan, s) : go<T, 1, true>(a, plan, s);
  if (e == cudaSuccess) e = plan.own_cols == 16 ? go<T, kWide, false>(a, plan, s) : go<T, 1, false>(a, plan, s);
  if (e != cudaSuccess || plan.n_pre + plan.n_own <= 1) return e;
  return launch_pdl(attn4_join<T>, dim3((unsigned)(((long long)a.B * a.H_q + 7) / 8)), dim3(256), 0, s, a, plan);
}

}  // namespace

cudaError_t attn4_launch(const AttnArgs& a, const Attn4Plan& plan, int dtype, cudaStream_t s) {
  return dtype == 0 ? run<float>(a, plan, s) : run<__nv_bfloat16>(a, plan, s);
}

}  // namespace provip
