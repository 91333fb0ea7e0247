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
#include <cuda_fp16.h>

#include "attention.cuh"

namespace provip {
namespace {

constexpr int kWarps = 4, kThr = kWarps * 32;
constexpr int kStep = 64;      // keys of a warp's stage
constexpr int kTiles = kStep / 16;
constexpr int kStages = 2;
constexpr int kCodeBytes = kStep * kCodes4, kScaleBytes = kStep * 8;
constexpr int kStageBytes = 2 * (kCodeBytes + kScaleBytes);  // K codes, V codes, K scales, V scales
constexpr int kRing = kStages * kStageBytes;
constexpr size_t kSmem = (size_t)kWarps * kRing;

// D = C + A B, fp32 sums; both operands fp16 (F16) or both bf16; C is D, or zero (FIRST)
template <bool F16, bool FIRST>
__device__ __forceinline__ void mma16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  const float c0 = FIRST ? 0.f : d[0], c1 = FIRST ? 0.f : d[1], c2 = FIRST ? 0.f : d[2], c3 = FIRST ? 0.f : d[3];
  if (F16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
// (x & mask) | magic in one instruction: the mask an immediate, the magic a register
template <uint32_t kMask>
__device__ __forceinline__ uint32_t mask_or(uint32_t x, uint32_t magic) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(x), "n"(kMask), "r"(magic));
  return r;
}
// What the expansion of codes keeps in registers (as an instruction takes one constant, and of known ones the
// compiler makes more instructions)
struct CodeRegs {
  uint32_t f16, bf16, sixteenth;  // 1024 as fp16, 128 as bf16, 1/16 as fp16, twice each
};
// The four nibbles of each half of x, less 8, as pairs of fp16: 1024 + n, or with the nibble at bit
// 4 1024 + 16 n, by a mask-or, then a multiply-add. One shift for the four.
__device__ __forceinline__ void codes_f16(uint32_t x, const CodeRegs& k, uint32_t* c) {
#pragma unroll
  for (int t = 0; t < 4; t += 2) {
    const uint32_t w = t ? x >> 8 : x;
    const uint32_t v0 = mask_or<0x000f000fu>(w, k.f16), v1 = mask_or<0x00f000f0u>(w, k.f16);
    const __half2 h0 = __hadd2(*reinterpret_cast<const __half2*>(&v0), __float2half2_rn(-1032.f));
    const __half2 h1 = __hfma2(*reinterpret_cast<const __half2*>(&v1), *reinterpret_cast<const __half2*>(&k.sixteenth), __float2half2_rn(-72.f));
    c[t] = *reinterpret_cast<const uint32_t*>(&h0);
    c[t + 1] = *reinterpret_cast<const uint32_t*>(&h1);
  }
}
// The same as pairs of bf16, whose seven bits want each nibble at bit 0 (128 + n): three shifts. (Shifts by the
// upper halves of products, to spare the integer pipe, took 94.9 us where these take 88.7.)
__device__ __forceinline__ void codes_bf16(uint32_t x, const CodeRegs& k, uint32_t* c) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const uint32_t v = mask_or<0x000f000fu>(x >> (4 * t), k.bf16);
    const __nv_bfloat162 h = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), __bfloat162bfloat162(__float2bfloat16_rn(136.f)));
    c[t] = *reinterpret_cast<const uint32_t*>(&h);
  }
}
__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// x, y as kP fp16 pairs that add up to them
template <int kP>
__device__ __forceinline__ void split2_f16(float x, float y, uint32_t* r) {
#pragma unroll
  for (int p = 0; p < kP; ++p) {
    const __half2 h = __floats2half2_rn(x, y);
    r[p] = *reinterpret_cast<const uint32_t*>(&h);
    if (p + 1 < kP) {
      x -= __low2float(h);
      y -= __high2float(h);
    }
  }
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

// A column's query row: its request and head (h < 0: none). Own keys: head `block * R + c` of request
// `unit`; the prefix: row `block` + c of the packed (request, head of the group) rows of head `unit`.
struct Column {
  int b, h;
};
template <bool kPrefix>
__device__ __forceinline__ Column column(const AttnArgs& a, int R, int unit, int block, int c) {
  if (!kPrefix) return {unit, c < R ? block * R + c : -1};
  const unsigned r = (unsigned)block + c, b = r / (unsigned)R;  // (B R fits 31 bits)
  return {(int)b, b < (unsigned)a.B ? unit * R + (int)(r - b * R) : -1};
}

// kHeads: query rows to a tile of eight columns. Eight: a column each, with the scores of the four groups of
// dims from sums of their own. Two: four columns each, one a group (its queries are zero outside the group),
// so that one sum over all dims leaves the groups' scores side by side, and the second product's columns carry a
// weight for each group: a fifth of the instructions about scores and weights less where a head is alone
// (or two are), and most of the columns are empty otherwise.
template <typename T, int NT, int kHeads, bool kPrefix>
__global__ void __launch_bounds__(kThr, sizeof(T) == 4 || NT > 1 ? 2 : 3)
    attn4_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ Attn4Plan plan) {
  constexpr bool kSplit = kHeads == 2;
  constexpr int kE = kSplit ? 2 : 4;          // scores a lane and tile: its rows, by its columns' heads
  constexpr int kH = kSplit ? 1 : 2;          // heads of a lane's columns
  constexpr int kQ = sizeof(T) == 4 ? 2 : 1;  // fp16 pieces of a query
  constexpr int kP = sizeof(T) == 4 ? 3 : 1;  // bf16 pieces of a weight
  constexpr int C = kHeads * NT;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t full[kWarps][kStages];
  __shared__ float s_m[kWarps][C], s_l[kWarps][C];
  __shared__ __align__(16) uint32_t s_q[NT][kQ][4][32][4];
  __shared__ float s_most[4][C];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
  const bool first = threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0;
  pdl_allow_next();  // the joining kernel, and behind the prefix the own keys', may be scheduled

  // this CTA's piece. Own keys: x a virtual key/value head (their parts of a page lie next to each
  // other), y a part, z the request; the prefix: x a block of rows, y a part, z the head
  const int R = kPrefix ? a.group : a.group / plan.n_cut;
  const int part = blockIdx.y, unit = blockIdx.z, block = kPrefix ? (int)blockIdx.x * C : (int)blockIdx.x;
  const int kv_head = kPrefix ? unit : plan.n_cut == 1 ? block : block / plan.n_cut;
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
    if (!kPrefix && first) pdl_wait_prior();
    return;
  }
  const int k_hi = k_lo + min(len - k_lo, part_keys);
  const int n_steps = max(0, (k_hi - k_lo + kStep - 1) / kStep);

  // loads: a lane per copy of a stage (up to eight boxes of rows, K and V codes and scales of each)
  const int box = min(a.page_size, kStep), kind = lane & 3, box_row = (lane >> 2) * box;
  auto page_of = [&](int step) {
    const int k = k_lo + step * kStep + box_row;
    return box_row < kStep && step < n_steps && k < k_hi ? __ldg(table + (k >> a.page_shift)) : 0;
  };
  int page = page_of(warp);
  if (lane == 0) {
    for (int s = 0; s < kStages; ++s) mbar_init(&full[warp][s], 1);
    fence_mbar_init();
  }
  __syncwarp();
  const uint32_t ring = smem_u32(smem) + warp * kRing, bar = smem_u32(&full[warp][0]);
  const uint32_t unit_bytes = kind < 2 ? kCodes4 : 8;  // of a row
  const uint32_t dst = ring + box_row * unit_bytes + (kind < 2 ? kind * kCodeBytes : 2 * kCodeBytes + (kind - 2) * kScaleBytes);
  const uint8_t* src = static_cast<const uint8_t*>(kind & 1 ? a.V : a.K) + (((size_t)kv_head * kRow4 + (kind < 2 ? 0 : kCodes4)) << a.page_shift);
  const uint32_t page_bytes = (uint32_t)(a.H_kv * kRow4) << a.page_shift;
  auto load = [&](int step, int stage) {  // (steps: this warp's, in order)
    const int k = k_lo + step * kStep, rows = min(kStep, k_hi - k);
    int p = page;
    page = page_of(step + kWarps);
    if (lane == 0) mbar_arrive_expect_tx(&full[warp][stage], (uint32_t)(((rows + box - 1) & ~(box - 1)) * kRow4 * 2));
    __syncwarp();
    if (box_row < rows) {
      if ((unsigned)p >= (unsigned)a.n_pages) {
        set_error(a.err, kErrBadDeviceArg);
        p = 0;
      }
      bulk_load(dst + stage * kStageBytes, src + (size_t)p * page_bytes + ((k + box_row) & (a.page_size - 1)) * unit_bytes,
                box * unit_bytes, bar + stage * 8);
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

  // Queries: column g's dims 32 q + 8 j .. + 7, as B operands in fp16: times a power of two that brings
  // the column's largest into [2^14, 2^15), so that nothing is lost but what is below 2^-39 of that. The
  // scale of a column's scores makes up for it. Warp q works out group q for all.
  uint32_t qf[NT][kQ][4][4];
  float cs[NT][kH];
  {
    float x[NT][8];
    const bool mine = !kSplit || (g & 3) == warp;  // column g has this group
    const int g_head = kSplit ? g >> 2 : g;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[nt][e] = 0.f;
      const Column c = column<kPrefix>(a, R, unit, block, nt * kHeads + g_head);
      if (c.h >= 0 && mine)
        load8(static_cast<const T*>(a.Q) + (size_t)c.b * a.q_stride + (size_t)c.h * kHeadDim + 32 * warp + 8 * j, x[nt]);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float most = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[nt][e]));
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
      if (j == 0 && mine) s_most[warp][nt * kHeads + g_head] = most;
    }
    __syncthreads();
    // 2^(14 - exponent), and its reciprocal (exponents from -100 on: smaller queries need no more)
    auto up = [&](int c) {
      const float most = fmaxf(fmaxf(s_most[0][c], s_most[1][c]), fmaxf(s_most[2][c], s_most[3][c]));
      return 14 + 127 - max((int)(__float_as_uint(most) >> 23), 27);
    };
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float mul = __uint_as_float((uint32_t)(127 + up(nt * kHeads + g_head)) << 23);
      uint32_t r[4][kQ];
#pragma unroll
      for (int t = 0; t < 4; ++t) split2_f16<kQ>(x[nt][t] * mul, x[nt][t + 4] * mul, r[t]);
#pragma unroll
      for (int p = 0; p < kQ; ++p)
        *reinterpret_cast<uint4*>(s_q[nt][p][warp][lane]) = make_uint4(r[0][p], r[1][p], r[2][p], r[3][p]);
#pragma unroll
      for (int c = 0; c < kH; ++c)
        cs[nt][c] = __uint_as_float((uint32_t)(127 - up(nt * kHeads + (kSplit ? j >> 1 : 2 * j + c))) << 23) * a.scale_log2;
    }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int p = 0; p < kQ; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint4 v = *reinterpret_cast<const uint4*>(s_q[nt][p][q][lane]);
          qf[nt][p][q][0] = v.x;
          qf[nt][p][q][1] = v.y;
          qf[nt][p][q][2] = v.z;
          qf[nt][p][q][3] = v.w;
        }
  }

  const CodeRegs regs = {plan.regs[0], plan.regs[1], plan.regs[2]};
  float o[4][2][NT][4], m[NT][kH], base[NT][kH], l[NT][kH];  // base: the maximum, 0 for none
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int c = 0; c < kH; ++c) {
      m[nt][c] = -INFINITY;
      base[nt][c] = l[nt][c] = 0.f;
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
    float s[kTiles][NT][kE];
#pragma unroll
    for (int mt = 0; mt < kTiles; ++mt) {
      const int r0 = mt * 16 + g, r1 = r0 + 8;
      const uint4 wa = *reinterpret_cast<const uint4*>(kc + r0 * kCodes4 + 16 * j);
      const uint4 wb = *reinterpret_cast<const uint4*>(kc + r1 * kCodes4 + 16 * j);
      // scales of the rows: all four groups', or those of this lane's columns
      uint2 da, db;
      if (kSplit) {
        da.x = *reinterpret_cast<const uint32_t*>(ks + r0 * 8 + 4 * (j & 1));
        db.x = *reinterpret_cast<const uint32_t*>(ks + r1 * 8 + 4 * (j & 1));
      } else {
        da = *reinterpret_cast<const uint2*>(ks + r0 * 8);
        db = *reinterpret_cast<const uint2*>(ks + r1 * 8);
      }
      float x[NT][4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t sel = q & 1 ? 0x7632 : 0x5410;
        const uint32_t xa = q < 2 ? __byte_perm(wa.x, wa.z, sel) : __byte_perm(wa.y, wa.w, sel);
        const uint32_t xb = q < 2 ? __byte_perm(wb.x, wb.z, sel) : __byte_perm(wb.y, wb.w, sel);
        uint32_t ca[4], cb[4];
        codes_f16(xa, regs, ca);
        codes_f16(xb, regs, cb);
        const uint32_t ua = q < 2 ? da.x : da.y, ub = q < 2 ? db.x : db.y;
        const float fa = q & 1 ? hi_f(ua) : lo_f(ua), fb = q & 1 ? hi_f(ub) : lo_f(ub);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          if (!kSplit || q == 0)
            mma16<true, true>(x[nt], ca[0], cb[0], ca[1], cb[1], qf[nt][kQ - 1][q][0], qf[nt][kQ - 1][q][1]);
          else
            mma16<true, false>(x[nt], ca[0], cb[0], ca[1], cb[1], qf[nt][kQ - 1][q][0], qf[nt][kQ - 1][q][1]);
          mma16<true, false>(x[nt], ca[2], cb[2], ca[3], cb[3], qf[nt][kQ - 1][q][2], qf[nt][kQ - 1][q][3]);
          if (kQ > 1) {
            mma16<true, false>(x[nt], ca[0], cb[0], ca[1], cb[1], qf[nt][0][q][0], qf[nt][0][q][1]);
            mma16<true, false>(x[nt], ca[2], cb[2], ca[3], cb[3], qf[nt][0][q][2], qf[nt][0][q][3]);
          }
          if constexpr (!kSplit) {
            if (q == 0) {
              s[mt][nt][0] = x[nt][0] * fa;
              s[mt][nt][1] = x[nt][1] * fa;
              s[mt][nt][2] = x[nt][2] * fb;
              s[mt][nt][3] = x[nt][3] * fb;
            } else {
              s[mt][nt][0] = fmaf(x[nt][0], fa, s[mt][nt][0]);
              s[mt][nt][1] = fmaf(x[nt][1], fa, s[mt][nt][1]);
              s[mt][nt][2] = fmaf(x[nt][2], fb, s[mt][nt][2]);
              s[mt][nt][3] = fmaf(x[nt][3], fb, s[mt][nt][3]);
            }
          }
        }
      }
      if constexpr (kSplit) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float ra = fmaf(x[nt][0], lo_f(da.x), x[nt][1] * hi_f(da.x)), rb = fmaf(x[nt][2], lo_f(db.x), x[nt][3] * hi_f(db.x));
          s[mt][nt][0] = ra + __shfl_xor_sync(0xffffffffu, ra, 1);  // (the same bits in both lanes)
          s[mt][nt][1] = rb + __shfl_xor_sync(0xffffffffu, rb, 1);
        }
      }
    }
    // base 2, hidden keys out (rounded before a maximum is subtracted: no fma with that). Score e: of head
    // e % kH of the lane's, row g (+ 8 from kH on)
#pragma unroll
    for (int mt = 0; mt < kTiles; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < kE; ++e) s[mt][nt][e] = __fmul_rn(s[mt][nt][e], cs[nt][e % kH]);
    if (left < kStep) {
#pragma unroll
      for (int mt = 0; mt < kTiles; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < kE; ++e)
            if (mt * 16 + (e / kH) * 8 + g >= left) s[mt][nt][e] = -INFINITY;
    }
    bool raise = false;
    float top[NT][kH];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < kH; ++c) {
        top[nt][c] = fmaxf(s[0][nt][c], s[0][nt][c + kH]);
#pragma unroll
        for (int mt = 1; mt < kTiles; ++mt) top[nt][c] = fmaxf(top[nt][c], fmaxf(s[mt][nt][c], s[mt][nt][c + kH]));
        raise = raise || top[nt][c] > m[nt][c] + 10.f;
      }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < kH; ++c) {
          float x = top[nt][c];
#pragma unroll
          for (int b = 4; b < 32; b <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, b));
          x = fmaxf(x, m[nt][c]);
          const float f = x == m[nt][c] ? 1.f : ex2_approx(m[nt][c] - x);
          m[nt][c] = x;
          base[nt][c] = x == -INFINITY ? 0.f : x;
          l[nt][c] *= f;
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (e % kH == c) o[q][h][nt][e] *= f;
        }
    }
#pragma unroll
    for (int mt = 0; mt < kTiles; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const float p = ex2_approx(s[mt][nt][e] - base[nt][e % kH]);
          s[mt][nt][e] = p;
          l[nt][e % kH] += p;
        }
    // (fp32: a step's sums start from zero and are added in fp32, as the MMAs' own sums truncate)
    float add[kP > 1 ? 4 : 1][2][NT][4];
    if (kP > 1) {
#pragma unroll
      for (int i = 0; i < 4 * 2 * NT * 4; ++i) (&add[0][0][0][0])[i] = 0.f;
    }
#pragma unroll
    for (int mt = 0; mt < kTiles; ++mt) {
      const int r0 = mt * 16 + g, k0 = mt * 16 + 2 * j;
      // a row past the end has no scale, whatever lies there
      uint2 da, db;
      if (kSplit) {
        da.x = *reinterpret_cast<const uint32_t*>(vs + r0 * 8 + 4 * (j & 1));
        db.x = *reinterpret_cast<const uint32_t*>(vs + (r0 + 8) * 8 + 4 * (j & 1));
      } else {
        da = *reinterpret_cast<const uint2*>(vs + r0 * 8);
        db = *reinterpret_cast<const uint2*>(vs + (r0 + 8) * 8);
      }
      if (left < kStep) {
        if (r0 >= left) da = make_uint2(0u, 0u);
        if (r0 + 8 >= left) db = make_uint2(0u, 0u);
      }
      uint32_t b0[NT][kP], b1[NT][kP];
      if constexpr (kSplit) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          split2<kP>(s[mt][nt][0] * lo_f(da.x), s[mt][nt][0] * hi_f(da.x), b0[nt]);
          split2<kP>(s[mt][nt][1] * lo_f(db.x), s[mt][nt][1] * hi_f(db.x), b1[nt]);
#pragma unroll
          for (int p = 0; p < kP; ++p) {
            b0[nt][p] = transpose8x8(b0[nt][p]);
            b1[nt][p] = transpose8x8(b1[nt][p]);
          }
        }
      }
      uint2 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint2*>(vc + (k0 + (i >> 1) * 8 + (i & 1)) * kCodes4 + 8 * g);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t sel = q & 1 ? 0x7632 : 0x5410;
        const uint32_t ya = q < 2 ? __byte_perm(v[0].x, v[1].x, sel) : __byte_perm(v[0].y, v[1].y, sel);
        const uint32_t yb = q < 2 ? __byte_perm(v[2].x, v[3].x, sel) : __byte_perm(v[2].y, v[3].y, sel);
        uint32_t ca[4], cb[4];
        codes_bf16(ya, regs, ca);
        codes_bf16(yb, regs, cb);
        const uint32_t ua = q < 2 ? da.x : da.y, ub = q < 2 ? db.x : db.y;
        const float fa = q & 1 ? hi_f(ua) : lo_f(ua), fb = q & 1 ? hi_f(ub) : lo_f(ub);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          if constexpr (!kSplit) {
            split2<kP>(s[mt][nt][0] * fa, s[mt][nt][1] * fa, b0[nt]);
            split2<kP>(s[mt][nt][2] * fb, s[mt][nt][3] * fb, b1[nt]);
#pragma unroll
            for (int p = 0; p < kP; ++p) {
              b0[nt][p] = transpose8x8(b0[nt][p]);
              b1[nt][p] = transpose8x8(b1[nt][p]);
            }
          }
#pragma unroll
          for (int p = kP - 1; p >= 0; --p) {
            mma16<false, false>(kP > 1 ? add[q][0][nt] : o[q][0][nt], ca[0], ca[1], cb[0], cb[1], b0[nt][p], b1[nt][p]);
            mma16<false, false>(kP > 1 ? add[q][1][nt] : o[q][1][nt], ca[2], ca[3], cb[2], cb[3], b0[nt][p], b1[nt][p]);
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
    for (int c = 0; c < kH; ++c)
#pragma unroll
      for (int b = 4; b < 32; b <<= 1) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], b);

  // the four warps' results: [warp][column][128] over the rings
  const int n_cols = kPrefix ? C : R;
  __syncthreads();
  float* so = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int col = nt * kHeads + (kSplit ? j >> 1 : 2 * j + c);
      if (col >= n_cols) continue;
      if (g == 0 && (!kSplit || c == (j & 1))) {
        s_m[warp][col] = m[nt][kSplit ? 0 : c];
        s_l[warp][col] = l[nt][kSplit ? 0 : c];
      }
      float* to = so + (warp * C + col) * kHeadDim + 4 * g;
      if constexpr (kSplit) {  // column 2 j + c has the sums of group 2 (j & 1) + c alone
        const bool up = j & 1;
        *reinterpret_cast<float4*>(to + 32 * c + (up ? 64 : 0)) =
            make_float4(up ? o[2 + c][0][nt][c] : o[c][0][nt][c], up ? o[2 + c][0][nt][c + 2] : o[c][0][nt][c + 2],
                        up ? o[2 + c][1][nt][c] : o[c][1][nt][c], up ? o[2 + c][1][nt][c + 2] : o[c][1][nt][c + 2]);
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(to + 32 * q) =
              make_float4(o[q][0][nt][c], o[q][0][nt][c + 2], o[q][1][nt][c], o[q][1][nt][c + 2]);
      }
    }
  __syncthreads();
  // a warp takes every fourth column, a lane four dims
  for (int col = warp; col < n_cols; col += kWarps) {
    const Column at = column<kPrefix>(a, R, unit, block, col);
    if (at.h < 0) continue;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_m[w][col]);
    float L = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = s_m[w][col] == -INFINITY ? 0.f : ex2_approx(s_m[w][col] - M);
      const float4 v = *reinterpret_cast<const float4*>(so + (w * C + col) * kHeadDim + 4 * lane);
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
    const size_t row = (size_t)at.b * a.H_q + at.h;
    if (alone) {
      store4(static_cast<T*>(a.out) + (size_t)at.b * a.o_stride + (size_t)at.h * kHeadDim + 4 * lane, x);
      if (lane == 0 && a.lse) a.lse[row] = lse * kLn2;
    } else {
      const size_t slot = (size_t)((kPrefix ? 0 : plan.n_pre) + part) * a.B * a.H_q + row;
      store4(a.part_o + slot * kHeadDim + 4 * lane, x);
      if (lane == 0) a.part_lse[slot] = lse;
    }
  }
  // beside the prefix's kernel: the joining one waits for this one alone
  if (!kPrefix && first) pdl_wait_prior();
}

// ---------------------------------------------------------------------------
// The prefix, for many rows (bf16 queries). The same products as above, but a key's codes are expanded once
// for all columns of the CTA: c d is exact in fp16 (three bits of c, or a power of two, times eight of
// d) next to a power of two, so values go into shared memory as fp16 MMA operands, each lane's registers at
// its place, and neither product knows of groups:
//   score_t = 2^{e_t} (Q . k_t)        o_q = 2^{u_q} sum_t p_t v_{t,q}
// with k_t relative to the largest scale of its row, and the values of group q to u_q, the largest scale in the
// group among the first 64 keys. Five bits of exponent hold that while a row's scales lie within 2^10 of each
// other, and a group's, over 16 keys, within 2^9 and at 2^u_q to a factor of 2^4. Sixteen keys that do not fit are
// done as above, codes and scales apart. 64 keys at a time, four warps expand 16 of them each into one of two
// buffers, while eight others take the 64 before from the other against their 8 NT columns.
// Bound by the MMAs (half of one an SM and clock) and by their operands' way out of shared memory (128 bytes
// a clock), which take equally long.
// ---------------------------------------------------------------------------
constexpr int kWideWarps = 8, kExpand = 4, kWideThr = (kWideWarps + kExpand) * 32;
constexpr int kFragBytes = kTiles * 8 * 32 * 16;  // operands of 64 keys, K's or V's
constexpr int kWideStages = 3;
constexpr size_t kWideSmem = 4 * (size_t)kFragBytes + (size_t)kWideStages * kStageBytes;
constexpr int kAtOnce = 2;  // tiles of 16 keys a warp has scores of
constexpr int kLift = 4;  // weights are 2^4 higher than they are, so that small ones keep their bits
constexpr int kRowSpread = 10, kTileSpread = 9, kUnitSpread = 4, kUnitMost = 40;

// named barriers: 1 among the expanding warps; 2, 3 a buffer is whole, 4, 5 it may be overwritten
__device__ __forceinline__ void expand_sync() { asm volatile("barrier.cta.sync 1, %0;" ::"n"(kExpand * 32) : "memory"); }
__device__ __forceinline__ void wide_sync(int id) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "n"(kWideThr) : "memory"); }
__device__ __forceinline__ void wide_arrive(int id) { asm volatile("barrier.cta.arrive %0, %1;" ::"r"(id), "n"(kWideThr) : "memory"); }
__device__ __forceinline__ float pow2(int biased) { return __uint_as_float((uint32_t)biased << 23); }
// biased exponent of scale q of a row (0 for a scale of zero; infinite and NaN ones, which show in any case, too)
__device__ __forceinline__ int exponent_of(uint2 d, int q) {
  const uint32_t w = (q < 2 ? d.x : d.y) >> (q & 1 ? 16 : 0);
  const int x = (int)((w >> 7) & 255u);
  return x == 255 ? 0 : (w & 0x7fffu) ? max(min(x, 253), 1) : 0;
}
__device__ __forceinline__ float scale_f(uint2 d, int q) {
  const uint32_t w = q < 2 ? d.x : d.y;
  return q & 1 ? hi_f(w) : lo_f(w);
}
__device__ __forceinline__ uint32_t times(uint32_t x, __half2 d) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&x), d);
  return *reinterpret_cast<const uint32_t*>(&r);
}

template <int N>
struct Tiles {
  static constexpr int n = N;
};

template <int NT>
__global__ void __launch_bounds__(kWideThr, 1)
    attn4_prefix(const __grid_constant__ AttnArgs a, const __grid_constant__ Attn4Plan plan) {
  constexpr int C = kWideWarps * 8 * NT;  // columns a CTA
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t full[kWideStages];
  __shared__ int s_ek[2][kStep];       // exponents of the keys' rows
  __shared__ __align__(16) int s_top[2][4][4];  // largest exponents of 16 keys' groups of values
  __shared__ __align__(16) int s_unit[2][4];    // exponents that the groups' values are relative to
  __shared__ int s_apart[2][2][kTiles];  // 16 keys whose codes and scales stay apart: K's, V's
  __shared__ uint2 s_d[2][2][kStep];   // scales
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
  pdl_allow_next();
  const int R = a.group, block = (int)blockIdx.x * C, part = blockIdx.y, kv_head = blockIdx.z;
  const int k_lo = part * plan.pre_keys;
  const int k_hi = k_lo + min(a.prefix_len - k_lo, plan.pre_keys);
  const int n_steps = (k_hi - k_lo + kStep - 1) / kStep;
  uint8_t* ring = smem + 4 * kFragBytes;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kWideStages; ++s) mbar_init(&full[s], 1);
    fence_mbar_init();
  }
  __syncthreads();
  const CodeRegs regs = {plan.regs[0], plan.regs[1], plan.regs[2]};

  if (warp >= kWideWarps) {
    // ---- expanding warps: 16 keys each as operands. Rows past the end are zeros, whatever lies there ----
    const int w = warp - kWideWarps;
    const bool first = w == 0;
    // loads, by the first of them: a lane per copy of a stage
    const int box = min(a.page_size, kStep), kind = lane & 3, box_row = (lane >> 2) * box;
    auto page_of = [&](int step) {
      const int k = k_lo + step * kStep + box_row;
      return box_row < kStep && step < n_steps && k < k_hi ? __ldg(a.prefix_table + (k >> a.page_shift)) : 0;
    };
    int page = first ? page_of(0) : 0;
    const uint32_t unit_bytes = kind < 2 ? kCodes4 : 8;
    const uint32_t dst = smem_u32(ring) + box_row * unit_bytes + (kind < 2 ? kind * kCodeBytes : 2 * kCodeBytes + (kind - 2) * kScaleBytes);
    const uint8_t* src = static_cast<const uint8_t*>(kind & 1 ? a.V : a.K) + (((size_t)kv_head * kRow4 + (kind < 2 ? 0 : kCodes4)) << a.page_shift);
    const uint32_t page_bytes = (uint32_t)(a.H_kv * kRow4) << a.page_shift;
    int issued = 0;  // (steps in order: stage issued % kWideStages)
    auto load = [&]() {
      const int k = k_lo + issued * kStep, rows = min(kStep, k_hi - k), stage = issued % kWideStages;
      int p = page;
      page = page_of(issued + 1);
      if (lane == 0) mbar_arrive_expect_tx(&full[stage], (uint32_t)(((rows + box - 1) & ~(box - 1)) * kRow4 * 2));
      __syncwarp();
      if (box_row < rows) {
        if ((unsigned)p >= (unsigned)a.n_pages) {
          set_error(a.err, kErrBadDeviceArg);
          p = 0;
        }
        bulk_load(dst + stage * kStageBytes, src + (size_t)p * page_bytes + ((k + box_row) & (a.page_size - 1)) * unit_bytes,
                  box * unit_bytes, smem_u32(&full[stage]));
      }
      __syncwarp();
      ++issued;
    };
    if (first)
      while (issued < kWideStages && issued < n_steps) load();
    int made[4] = {0, 0, 0, 0};  // exponents that the values are relative to
    bool failed = false;
    for (int step = 0; step < n_steps; ++step) {
      const int stage = step % kWideStages, buf = step & 1, left = k_hi - k_lo - step * kStep;
      // (a wait that gives up: no more waits, but every barrier is met)
      if (!failed && __any_sync(0xffffffffu, !mbar_wait(&full[stage], (uint32_t)(step / kWideStages) & 1u, a.err))) failed = true;
      if (step >= 2) wide_sync(4 + buf);
      const uint8_t* st = ring + stage * kStageBytes;
      uint4* to = reinterpret_cast<uint4*>(smem + buf * 2 * kFragBytes) + w * 8 * 32 + lane;
      {
        const uint8_t *kc = st, *ks = st + 2 * kCodeBytes;
        const int r0 = w * 16 + g, r1 = r0 + 8;
        uint2 da = *reinterpret_cast<const uint2*>(ks + r0 * 8), db = *reinterpret_cast<const uint2*>(ks + r1 * 8);
        if (r0 >= left) da = make_uint2(0u, 0u);
        if (r1 >= left) db = make_uint2(0u, 0u);
        int ea = 1, eb = 1, la = 255, lb = 255;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int x = exponent_of(da, q), y = exponent_of(db, q);
          ea = max(ea, x);
          eb = max(eb, y);
          la = min(la, x == 0 ? 255 : x);
          lb = min(lb, y == 0 ? 255 : y);
        }
        const bool apart = __any_sync(0xffffffffu, ea - la > kRowSpread || eb - lb > kRowSpread);
        if (lane == 0) s_apart[buf][0][w] = apart;
        if (j == 0) {
          s_ek[buf][r0] = ea;
          s_ek[buf][r1] = eb;
          s_d[buf][0][r0] = da;
          s_d[buf][0][r1] = db;
        }
        const float fa = pow2(254 - ea), fb = pow2(254 - eb);  // 2^-(e - 127)
        const uint4 wa = *reinterpret_cast<const uint4*>(kc + r0 * kCodes4 + 16 * j);
        const uint4 wb = *reinterpret_cast<const uint4*>(kc + r1 * kCodes4 + 16 * j);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t sel = q & 1 ? 0x7632 : 0x5410;
          uint32_t ca[4], cb[4];
          codes_f16(q < 2 ? __byte_perm(wa.x, wa.z, sel) : __byte_perm(wa.y, wa.w, sel), regs, ca);
          codes_f16(q < 2 ? __byte_perm(wb.x, wb.z, sel) : __byte_perm(wb.y, wb.w, sel), regs, cb);
          const __half2 ha = __float2half2_rn(apart ? 1.f : scale_f(da, q) * fa), hb = __float2half2_rn(apart ? 1.f : scale_f(db, q) * fb);
#pragma unroll
          for (int i = 0; i < 2; ++i)
            to[(2 * q + i) * 32] = make_uint4(times(ca[2 * i], ha), times(cb[2 * i], hb), times(ca[2 * i + 1], ha), times(cb[2 * i + 1], hb));
        }
      }
      {
        // keys 2 j, 2 j + 1, 2 j + 8, 2 j + 9 of the sixteen, dims 4 g .. + 3 of each group
        const uint8_t *vc = st + kCodeBytes, *vs = st + 2 * kCodeBytes + kScaleBytes;
        to += kFragBytes / 16;
        uint2 v[4], d[4];
        int hi[4] = {0, 0, 0, 0}, lo[4] = {255, 255, 255, 255};  // a group's largest and smallest exponent
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = w * 16 + 2 * j + (i >> 1) * 8 + (i & 1);
          v[i] = *reinterpret_cast<const uint2*>(vc + r * kCodes4 + 8 * g);
          d[i] = *reinterpret_cast<const uint2*>(vs + r * 8);
          if (r >= left) d[i] = make_uint2(0u, 0u);
          if (g == 0) s_d[buf][1][r] = d[i];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int e = exponent_of(d[i], q);
            hi[q] = max(hi[q], e);
            lo[q] = min(lo[q], e == 0 ? 255 : e);
          }
        }
        // (the eight lanes with another j have other keys, those with another g the same)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int b = 1; b < 4; b <<= 1) {
            hi[q] = max(hi[q], __shfl_xor_sync(0xffffffffu, hi[q], b));
            lo[q] = min(lo[q], __shfl_xor_sync(0xffffffffu, lo[q], b));
          }
        if (lane == 0) *reinterpret_cast<int4*>(s_top[buf][w]) = make_int4(hi[0], hi[1], hi[2], hi[3]);
        expand_sync();
        // (the stage before is read by all of them)
        if (first && issued < n_steps && step > 0) load();
        bool apart = false;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int top = max(max(max(s_top[buf][0][q], s_top[buf][1][q]), max(s_top[buf][2][q], s_top[buf][3][q])), 1);
          if (step == 0 || top > made[q] + kUnitMost) made[q] = top;  // (or far larger than what was before)
          apart = apart || hi[q] - lo[q] > kTileSpread || (hi[q] > 0 && abs(hi[q] - made[q]) > kUnitSpread);
        }
        if (lane == 0) {
          s_apart[buf][1][w] = apart;
          if (w == 0) *reinterpret_cast<int4*>(s_unit[buf]) = make_int4(made[0], made[1], made[2], made[3]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t sel = q & 1 ? 0x7632 : 0x5410;
          const uint32_t ya = q < 2 ? __byte_perm(v[0].x, v[1].x, sel) : __byte_perm(v[0].y, v[1].y, sel);
          const uint32_t yb = q < 2 ? __byte_perm(v[2].x, v[3].x, sel) : __byte_perm(v[2].y, v[3].y, sel);
          uint32_t ca[4], cb[4];
          if (apart) {
            codes_bf16(ya, regs, ca);
            codes_bf16(yb, regs, cb);
          } else {
            codes_f16(ya, regs, ca);
            codes_f16(yb, regs, cb);
            const float f = pow2(254 - made[q]);
            const __half2 ha = __floats2half2_rn(scale_f(d[0], q) * f, scale_f(d[1], q) * f);
            const __half2 hb = __floats2half2_rn(scale_f(d[2], q) * f, scale_f(d[3], q) * f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              ca[i] = times(ca[i], ha);
              cb[i] = times(cb[i], hb);
            }
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) to[(2 * q + i) * 32] = make_uint4(ca[2 * i], ca[2 * i + 1], cb[2 * i], cb[2 * i + 1]);
        }
      }
      wide_arrive(2 + buf);
    }
    if (failed && first) {
      // copies that may still be in flight into the block's shared memory: waited for once more, with a limit
      for (int i = max(issued - kWideStages, 0); i < issued; ++i) mbar_wait(&full[i % kWideStages], (uint32_t)(i / kWideStages) & 1u, a.err);
    }
    return;
  }

  // queries, as in the kernel above: a warp its own columns
  uint32_t qf[NT][4][4];
  float cs[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const Column c = column<true>(a, R, kv_head, block, (warp * NT + nt) * 8 + g);
    float x[4][8], most = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[q][e] = 0.f;
      if (c.h >= 0)
        load8(static_cast<const __nv_bfloat16*>(a.Q) + (size_t)c.b * a.q_stride + (size_t)c.h * kHeadDim + 32 * q + 8 * j, x[q]);
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[q][e]));
    }
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
    const int up = 14 + 127 - max((int)(__float_as_uint(most) >> 23), 27);
    const float mul = pow2(127 + up), back = pow2(127 - up) * a.scale_log2;
#pragma unroll
    for (int c2 = 0; c2 < 2; ++c2) cs[nt][c2] = __shfl_sync(0xffffffffu, back, 4 * (2 * j + c2));
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        uint32_t r[1];
        split2_f16<1>(x[q][t] * mul, x[q][t + 4] * mul, r);
        qf[nt][q][t] = r[0];
      }
  }

  float o[8][NT][4], m[NT][2], base[NT][2], l[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      m[nt][c] = -INFINITY;
      base[nt][c] = l[nt][c] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][nt][e] = 0.f;
  }
  int unit[4] = {0, 0, 0, 0};  // of o's sums; warps 4-7: of the values expanded last
  // a new maximum, where a score passes the one before by 2^10
  auto raise_to = [&](const float (*top)[2]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x = top[nt][c];
#pragma unroll
        for (int b = 4; b < 32; b <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, b));
        x = fmaxf(x, m[nt][c]);
        const float f = x == m[nt][c] ? 1.f : ex2_approx(m[nt][c] - x);
        m[nt][c] = x;
        base[nt][c] = x == -INFINITY ? 0.f : x;
        l[nt][c] *= f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          o[i][nt][c] *= f;
          o[i][nt][c + 2] *= f;
        }
      }
  };

  // ---- kN tiles of 16 keys from tile mt0 on against this warp's columns ----
  auto attend = [&](auto tiles, int buf, int mt0, int left, bool k_apart, bool v_apart) {
    constexpr int kN = decltype(tiles)::n;
    const uint4* kf = reinterpret_cast<const uint4*>(smem + buf * 2 * kFragBytes) + mt0 * 8 * 32 + lane;
    const uint4* vf = kf + kFragBytes / 16;
    float s[kN][NT][4];
    if (!k_apart) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int mt = 0; mt < kN; ++mt) {
          const uint4 c = kf[(mt * 8 + i) * 32];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if (i == 0)
              mma16<true, true>(s[mt][nt], c.x, c.y, c.z, c.w, qf[nt][0][0], qf[nt][0][1]);
            else
              mma16<true, false>(s[mt][nt], c.x, c.y, c.z, c.w, qf[nt][i >> 1][2 * (i & 1)], qf[nt][i >> 1][2 * (i & 1) + 1]);
          }
        }
#pragma unroll
      for (int mt = 0; mt < kN; ++mt) {
        const float ka = pow2(s_ek[buf][(mt0 + mt) * 16 + g]), kb = pow2(s_ek[buf][(mt0 + mt) * 16 + g + 8]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[mt][nt][e] *= e < 2 ? ka : kb;
      }
    } else {
#pragma unroll
      for (int mt = 0; mt < kN; ++mt) {
        const uint2 da = s_d[buf][0][(mt0 + mt) * 16 + g], db = s_d[buf][0][(mt0 + mt) * 16 + g + 8];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint4 c0 = kf[(mt * 8 + 2 * q) * 32], c1 = kf[(mt * 8 + 2 * q + 1) * 32];
          const float fa = scale_f(da, q), fb = scale_f(db, q);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float x[4];
            mma16<true, true>(x, c0.x, c0.y, c0.z, c0.w, qf[nt][q][0], qf[nt][q][1]);
            mma16<true, false>(x, c1.x, c1.y, c1.z, c1.w, qf[nt][q][2], qf[nt][q][3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[mt][nt][e] = q == 0 ? x[e] * (e < 2 ? fa : fb) : fmaf(x[e], e < 2 ? fa : fb, s[mt][nt][e]);
          }
        }
      }
    }
    bool raise = false;
    float top[NT][2];
#pragma unroll
    for (int mt = 0; mt < kN; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[mt][nt][e] = __fmul_rn(s[mt][nt][e], cs[nt][e & 1]);
    if (left < kStep) {
#pragma unroll
      for (int mt = 0; mt < kN; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if ((mt0 + mt) * 16 + g + (e >> 1) * 8 >= left) s[mt][nt][e] = -INFINITY;
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        top[nt][c] = fmaxf(s[0][nt][c], s[0][nt][c + 2]);
#pragma unroll
        for (int mt = 1; mt < kN; ++mt) top[nt][c] = fmaxf(top[nt][c], fmaxf(s[mt][nt][c], s[mt][nt][c + 2]));
        raise = raise || top[nt][c] > m[nt][c] + 10.f;
      }
    if (__any_sync(0xffffffffu, raise)) raise_to(top);
#pragma unroll
    for (int mt = 0; mt < kN; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = ex2_approx(s[mt][nt][e] - base[nt][e & 1]);
          l[nt][e & 1] += p;
          s[mt][nt][e] = p * (float)(1 << kLift);
        }
    if (!v_apart) {
#pragma unroll
      for (int mt = 0; mt < kN; ++mt) {
        uint32_t b0[NT], b1[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const __half2 x = __floats2half2_rn(s[mt][nt][0], s[mt][nt][1]), y = __floats2half2_rn(s[mt][nt][2], s[mt][nt][3]);
          b0[nt] = transpose8x8(*reinterpret_cast<const uint32_t*>(&x));
          b1[nt] = transpose8x8(*reinterpret_cast<const uint32_t*>(&y));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint4 c = vf[(mt * 8 + i) * 32];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma16<true, false>(o[i][nt], c.x, c.y, c.z, c.w, b0[nt], b1[nt]);
        }
      }
    } else {
#pragma unroll
      for (int mt = 0; mt < kN; ++mt) {
        const uint2 da = s_d[buf][1][(mt0 + mt) * 16 + g], db = s_d[buf][1][(mt0 + mt) * 16 + g + 8];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint4 c0 = vf[(mt * 8 + 2 * q) * 32], c1 = vf[(mt * 8 + 2 * q + 1) * 32];
          const float f = pow2(254 - unit[q]), fa = scale_f(da, q) * f, fb = scale_f(db, q) * f;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const uint32_t b0 = transpose8x8(pack2(s[mt][nt][0] * fa, s[mt][nt][1] * fa)), b1 = transpose8x8(pack2(s[mt][nt][2] * fb, s[mt][nt][3] * fb));
            mma16<false, false>(o[2 * q][nt], c0.x, c0.y, c0.z, c0.w, b0, b1);
            mma16<false, false>(o[2 * q + 1][nt], c1.x, c1.y, c1.z, c1.w, b0, b1);
          }
        }
      }
    }
  };

  for (int step = 0; step < n_steps; ++step) {
    const int buf = step & 1, left = k_hi - k_lo - step * kStep;
    wide_sync(2 + buf);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int u = s_unit[buf][q];
      if (u != unit[q]) {  // larger values: what there is, relative to them
        const float f = pow2(max(127 + unit[q] - u, 0));
#pragma unroll
        for (int i = 2 * q; i < 2 * q + 2; ++i)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][nt][e] *= f;
        unit[q] = u;
      }
    }
    int any = 0;
#pragma unroll
    for (int mt = 0; mt < kTiles; ++mt) any |= s_apart[buf][0][mt] | s_apart[buf][1][mt];
    if (!any) {
#pragma unroll 1
      for (int mt = 0; mt < kTiles && mt * 16 < left; mt += kAtOnce) attend(Tiles<kAtOnce>(), buf, mt, left, false, false);
    } else {
#pragma unroll 1
      for (int mt = 0; mt < kTiles && mt * 16 < left; ++mt)
        attend(Tiles<1>(), buf, mt, left, s_apart[buf][0][mt] != 0, s_apart[buf][1][mt] != 0);
    }
    if (step + 2 < n_steps) wide_arrive(4 + buf);  // these operands may be overwritten
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int b = 4; b < 32; b <<= 1) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], b);
      const Column at = column<true>(a, R, kv_head, block, (warp * NT + nt) * 8 + 2 * j + c);
      if (at.h < 0) continue;
      // (every score -inf: no weight)
      const bool nil = l[nt][c] == 0.f;
      const float inv = nil ? 0.f : (1.f / (1 << kLift)) / l[nt][c];
      const size_t slot = (size_t)part * a.B * a.H_q + (size_t)at.b * a.H_q + at.h;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float f = pow2(max(unit[q], 1));
        *reinterpret_cast<float4*>(a.part_o + slot * kHeadDim + 32 * q + 4 * g) =
            make_float4(o[2 * q][nt][c] * inv * f, o[2 * q][nt][c + 2] * inv * f, o[2 * q + 1][nt][c] * inv * f, o[2 * q + 1][nt][c + 2] * inv * f);
      }
      if (g == 0) a.part_lse[slot] = nil ? -INFINITY : m[nt][c] == -INFINITY ? NAN : m[nt][c] + log2f(l[nt][c]);
    }
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

template <typename T, int NT, int kHeads, bool kPrefix>
cudaError_t go(const AttnArgs& a, const Attn4Plan& plan, cudaStream_t s) {
  constexpr auto kernel = attn4_kernel<T, NT, kHeads, kPrefix>;
  static std::atomic<bool> configured[64];  // per device, zero-initialised
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 0 && dev < 64 && !configured[dev]) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  constexpr int C = kHeads * NT;
  const long long rows = (long long)a.B * a.group;
  const dim3 grid = kPrefix ? dim3((unsigned)((rows + C - 1) / C), plan.n_pre, a.H_kv) : dim3(a.H_kv * plan.n_cut, plan.n_own, a.B);
  if (!kPrefix && plan.n_pre > 0)  // beside the prefix's kernel, whose results it does not read
    return launch_pdl(kernel, grid, dim3(kThr), kSmem, s, a, plan);
  kernel<<<grid, kThr, kSmem, s>>>(a, plan);
  return cudaGetLastError();
}

template <typename T, bool kPrefix>
cudaError_t go_by_columns(int rows, const AttnArgs& a, const Attn4Plan& plan, cudaStream_t s) {
  if (rows == 2) return go<T, 1, 2, kPrefix>(a, plan, s);
  if (rows == 8) return go<T, 1, 8, kPrefix>(a, plan, s);
  if constexpr (sizeof(T) == 2) return go<T, 2, 8, kPrefix>(a, plan, s);  // (fp32 at 16 columns spills registers)
  return cudaErrorInvalidValue;
}

template <int NT>
cudaError_t go_wide(const AttnArgs& a, const Attn4Plan& plan, cudaStream_t s) {
  static std::atomic<bool> configured[64];  // per device, zero-initialised
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 0 && dev < 64 && !configured[dev]) {
    cudaError_t e = cudaFuncSetAttribute(attn4_prefix<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kWideSmem);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  const long long rows = (long long)a.B * a.group;
  constexpr int C = kWideWarps * 8 * NT;
  attn4_prefix<NT><<<dim3((unsigned)((rows + C - 1) / C), plan.n_pre, a.H_kv), kWideThr, kWideSmem, s>>>(a, plan);
  return cudaGetLastError();
}

template <typename T>
cudaError_t run(const AttnArgs& a, const Attn4Plan& plan, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (plan.n_pre > 0)
    e = plan.pre_rows == 256 ? attn4_prefix_tc_launch(a, plan, s)
        : plan.pre_rows == 128 ? go_wide<2>(a, plan, s)
        : plan.pre_rows == 64 ? go_wide<1>(a, plan, s) : go_by_columns<T, true>(plan.pre_rows, a, plan, s);
  if (e == cudaSuccess) e = go_by_columns<T, false>(plan.own_rows, a, plan, s);
  if (e != cudaSuccess || plan.n_pre + plan.n_own <= 1) return e;
  return launch_pdl(attn4_join<T>, dim3((unsigned)(((long long)a.B * a.H_q + 7) / 8)), dim3(256), 0, s, a, plan);
}

}  // namespace

cudaError_t attn4_launch(const AttnArgs& a, const Attn4Plan& plan, int dtype, cudaStream_t s) {
  return dtype == 0 ? run<float>(a, plan, s) : run<__nv_bfloat16>(a, plan, s);
}

}  // namespace provip
