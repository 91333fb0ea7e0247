// One token per request against pages of 4 bits.
//
// A row of 128 values is d_q (n - 8) with codes n and a scale d_q for each 32 values q (rotate.cu),
// so with integers c = n - 8, exact in fp16 and in bf16,
//   score_t = sum_q dk_{t,q} (Q_q . c_{t,q})        o_q = sum_t (p_t dv_{t,q}) c_{t,q}:
// scales stay outside the first product and go into the weights of the second, and no value is
// ever rounded to 16 bits. Both products run on mma.sync (m16n8k16, fp32 sums) with the codes
// as the 16-row operand A straight from registers: eight query rows ("columns") are enough to fill
// it, where a tcgen05 product would want the expanded codes written to shared memory first, four times
// the bytes that come from HBM, for every key. (It pays for a prefix that more than 16 bf16 rows share:
// attention_decode4_tc.cu. All else is here: own keys, few rows, fp32.)
//   S[16 keys x 8] = 4 groups x 2 MMAs over the dims, then 4 FMAs a score with dk
//   O^T[16 dims x 8] += 8 MMAs over 16 keys, with P dv from S's registers by movmatrix (a transpose)
// The order of the dims in the codes (rotate.cu) is such that a lane's 16 bytes of a key hold whole
// MMA operands of one group each: shifts and masks, no exchange.
//
// Work: a CTA of four warps takes a part of one (request, key/value head)'s keys, or of the prefix's for
// a block of rows of all requests; a warp 64 keys at a time, from a ring of its own that bulk copies
// fill (a page of one head is contiguous), with its own softmax state; the four join in shared memory.
// Rows of several parts are joined by a second kernel. No maximum is looked for while no score passes
// the one before by 2^10. Statistics and sums are fp32.
//
// Roundings. A query is fp16 after a power of two a row (bf16's eight bits fit), fp32 ones two fp16 pieces
// (2^-22 of a value at most); P dv is rounded to bf16 (2^-8 of each weight at most, as P is where keys are
// bf16), for fp32 split into three bf16 pieces (24 bits), a product each.
//
// What bounds it: no unit by itself. A lone head's kernel issues 2.3 of 4 instructions a clock (most of them take the codes
// apart), the integer units are busy for 56%, the tensor cores for 26 (fp32 48), HBM for 66: with twelve warps an SM it
// waits for its own chains of expansion, products and weights, and a CTA takes a whole list, so that the last ones
// leave SMs idle. 128 requests of 163 to 2339 keys (32 heads, bf16): 145 us, 5.1 TB/s of codes and scales; 32 of 163 to
// 1091 (32 heads, fp32): 39 us; one of 211: 9 us, of which the launch and the first loads' way are most; 64 of 3000 with 28
// heads over 4: 32 us, 3.5 TB/s. Stages of 32 keys, three stages,
// eight warps a CTA or more CTAs an SM took as long or longer; so did requests taken longest first, the first pages
// asked for beside the length, and scores summed in two chains.
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
// upper halves of products, to spare the integer pipe, took 94.9 us where these took 88.7, in an earlier build: 64 requests
// of 1250 keys, 32 heads, 71 now.)
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
// (or two are), and most of the columns are empty otherwise. A word of codes, which holds two groups' values side by side,
// is an operand as it is then, in both products: a pair meets a column's query or weight and a zero (128 requests:
// 154 -> 145 us with that). fp32 at three CTAs an SM: 64 requests of 1250 keys 108 -> 100 us.
template <typename T, int NT, int kHeads, bool kPrefix>
__global__ void __launch_bounds__(kThr, NT > 1 || (sizeof(T) == 4 && kHeads == 8) ? 2 : 3)
    attn4_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ Attn4Plan plan) {
  constexpr bool kSplit = kHeads == 2;
  constexpr int kE = kSplit ? 2 : 4;          // scores a lane and tile: its rows, by its columns' heads
  constexpr int kH = kSplit ? 1 : 2;          // heads of a lane's columns
  constexpr int kG = kSplit ? 2 : 4;          // sums a column: by word of the codes, or by group
  constexpr int kQ = sizeof(T) == 4 ? 2 : 1;  // fp16 pieces of a query
  constexpr int kP = sizeof(T) == 4 ? 3 : 1;  // bf16 pieces of a weight
  constexpr int C = kHeads * NT;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t full[kWarps][kStages];
  __shared__ float s_m[kWarps][C], s_l[kWarps][C];
  __shared__ __align__(16) uint32_t s_q[kSplit ? 1 : NT][kQ][kSplit ? 1 : 4][32][4];
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

  // Queries: dims 8 j .. + 7 of a column's groups, as B operands in fp16: times a power of two that brings
  // the column's largest into [2^14, 2^15), so that nothing is lost but what is below 2^-39 of that. The
  // scale of a column's scores makes up for it.
  // Of a lane's 16 bytes of codes a word holds four values of two groups, side by side. Columns of one group each take
  // the words as they are: a pair of values meets a query and a zero. For columns of all groups the words' halves are put
  // together by group, and warp q works out group q's queries for all.
  uint32_t qf[NT][kQ][4][4];
  float cs[NT][kH];
  // 2^(14 - exponent), and its reciprocal (exponents from -100 on: smaller queries need no more)
  auto up = [](float most) { return 14 + 127 - max((int)(__float_as_uint(most) >> 23), 27); };
  auto pow2 = [](int e) { return __uint_as_float((uint32_t)(127 + e) << 23); };
  if constexpr (kSplit) {
    const int q = g & 3;  // column g's group
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[8], most = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.f;
      const Column c = column<kPrefix>(a, R, unit, block, nt * kHeads + (g >> 2));
      if (c.h >= 0) load8(static_cast<const T*>(a.Q) + (size_t)c.b * a.q_stride + (size_t)c.h * kHeadDim + 32 * q + 8 * j, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));
#pragma unroll
      for (int b = 1; b < 16; b <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, b));
      const float mul = pow2(up(most));
      uint32_t r[4][kQ];
#pragma unroll
      for (int t = 0; t < 4; ++t) split2_f16<kQ>(x[t] * mul, x[t + 4] * mul, r[t]);
#pragma unroll
      for (int p = 0; p < kQ; ++p)
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const uint32_t v = w < 2 ? r[t][p] & 0xffffu : r[t][p] >> 16;
            qf[nt][p][w][t] = (w & 1) != (q >> 1) ? 0u : q & 1 ? v << 16 : v;
          }
      cs[nt][0] = pow2(-up(__shfl_sync(0xffffffffu, most, (j >> 1) * 16))) * a.scale_log2;
    }
  } else {
    float x[NT][8];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[nt][e] = 0.f;
      const Column c = column<kPrefix>(a, R, unit, block, nt * kHeads + g);
      if (c.h >= 0)
        load8(static_cast<const T*>(a.Q) + (size_t)c.b * a.q_stride + (size_t)c.h * kHeadDim + 32 * warp + 8 * j, x[nt]);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float most = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[nt][e]));
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
      if (j == 0) s_most[warp][nt * kHeads + g] = most;
    }
    __syncthreads();
    auto most_of = [&](int c) { return fmaxf(fmaxf(s_most[0][c], s_most[1][c]), fmaxf(s_most[2][c], s_most[3][c])); };
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float mul = pow2(up(most_of(nt * kHeads + g)));
      uint32_t r[4][kQ];
#pragma unroll
      for (int t = 0; t < 4; ++t) split2_f16<kQ>(x[nt][t] * mul, x[nt][t + 4] * mul, r[t]);
#pragma unroll
      for (int p = 0; p < kQ; ++p)
        *reinterpret_cast<uint4*>(s_q[nt][p][warp][lane]) = make_uint4(r[0][p], r[1][p], r[2][p], r[3][p]);
#pragma unroll
      for (int c = 0; c < kH; ++c) cs[nt][c] = pow2(-up(most_of(nt * kHeads + 2 * j + c))) * a.scale_log2;
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
  float o[kG][2][NT][4], m[NT][kH], base[NT][kH], l[NT][kH];  // base: the maximum, 0 for none
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int c = 0; c < kH; ++c) {
      m[nt][c] = -INFINITY;
      base[nt][c] = l[nt][c] = 0.f;
    }
#pragma unroll
    for (int q = 0; q < kG; ++q)
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
      float x[NT][4], y[NT][4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t xa, xb;  // a word (columns of a group each), or a group's halves of two
        if (kSplit) {
          xa = q == 0 ? wa.x : q == 1 ? wa.y : q == 2 ? wa.z : wa.w;
          xb = q == 0 ? wb.x : q == 1 ? wb.y : q == 2 ? wb.z : wb.w;
        } else {
          const uint32_t sel = q & 1 ? 0x7632 : 0x5410;
          xa = q < 2 ? __byte_perm(wa.x, wa.z, sel) : __byte_perm(wa.y, wa.w, sel);
          xb = q < 2 ? __byte_perm(wb.x, wb.z, sel) : __byte_perm(wb.y, wb.w, sel);
        }
        uint32_t ca[4], cb[4];
        codes_f16(xa, regs, ca);
        codes_f16(xb, regs, cb);
        const uint32_t ua = q < 2 ? da.x : da.y, ub = q < 2 ? db.x : db.y;
        const float fa = q & 1 ? hi_f(ua) : lo_f(ua), fb = q & 1 ? hi_f(ub) : lo_f(ub);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          // (a lone head's smaller pieces have a sum of their own: MMAs' sums truncate, at the size of what they hold)
          float* const lo = kSplit && kQ > 1 ? y[nt] : x[nt];
          if (!kSplit || q == 0)
            mma16<true, true>(lo, ca[0], cb[0], ca[1], cb[1], qf[nt][kQ - 1][q][0], qf[nt][kQ - 1][q][1]);
          else
            mma16<true, false>(lo, ca[0], cb[0], ca[1], cb[1], qf[nt][kQ - 1][q][0], qf[nt][kQ - 1][q][1]);
          mma16<true, false>(lo, ca[2], cb[2], ca[3], cb[3], qf[nt][kQ - 1][q][2], qf[nt][kQ - 1][q][3]);
          if (kQ > 1) {
            if (kSplit && q == 0)
              mma16<true, true>(x[nt], ca[0], cb[0], ca[1], cb[1], qf[nt][0][q][0], qf[nt][0][q][1]);
            else
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
          if (kQ > 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[nt][e] += y[nt][e];
          }
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
          for (int q = 0; q < kG; ++q)
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
    // (fp32: sums of 64 keys, or of 32 with twice the MMAs, start from zero and are added in fp32, as MMAs' sums truncate)
    float add[kP > 1 ? kG : 1][2][NT][4];
    if (kP > 1) {
#pragma unroll
      for (int i = 0; i < kG * 2 * NT * 4; ++i) (&add[0][0][0][0])[i] = 0.f;
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
      uint2 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint2*>(vc + (k0 + (i >> 1) * 8 + (i & 1)) * kCodes4 + 8 * g);
      if constexpr (kSplit) {
        // a word holds two groups' values of a key: operands of eight keys twice, whose columns of the one
        // group have zeros against the other's (sums of the other word's columns mean nothing)
        uint32_t b[NT][2][2][kP];  // of eight keys; keys 2 j, 2 j + 1
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          uint32_t w[2][kP];
          split2<kP>(s[mt][nt][0] * lo_f(da.x), s[mt][nt][0] * hi_f(da.x), w[0]);
          split2<kP>(s[mt][nt][1] * lo_f(db.x), s[mt][nt][1] * hi_f(db.x), w[1]);
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int p = 0; p < kP; ++p) {
              const uint32_t t = transpose8x8(w[i][p]);
              b[nt][i][0][p] = __byte_perm(t, 0u, g & 1 ? 0x1044 : 0x4410);
              b[nt][i][1][p] = __byte_perm(t, 0u, g & 1 ? 0x3244 : 0x4432);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t ca[4], cb[4];
            codes_bf16(q ? v[2 * i].y : v[2 * i].x, regs, ca);
            codes_bf16(q ? v[2 * i + 1].y : v[2 * i + 1].x, regs, cb);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int p = kP - 1; p >= 0; --p) {
                mma16<false, false>(kP > 1 ? add[q][0][nt] : o[q][0][nt], ca[0], ca[1], cb[0], cb[1], b[nt][i][0][p], b[nt][i][1][p]);
                mma16<false, false>(kP > 1 ? add[q][1][nt] : o[q][1][nt], ca[2], ca[3], cb[2], cb[3], b[nt][i][0][p], b[nt][i][1][p]);
              }
          }
      } else {
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
            uint32_t b0[kP], b1[kP];
            split2<kP>(s[mt][nt][0] * fa, s[mt][nt][1] * fa, b0);
            split2<kP>(s[mt][nt][2] * fb, s[mt][nt][3] * fb, b1);
#pragma unroll
            for (int p = 0; p < kP; ++p) {
              b0[p] = transpose8x8(b0[p]);
              b1[p] = transpose8x8(b1[p]);
            }
#pragma unroll
            for (int p = kP - 1; p >= 0; --p) {
              mma16<false, false>(kP > 1 ? add[q][0][nt] : o[q][0][nt], ca[0], ca[1], cb[0], cb[1], b0[p], b1[p]);
              mma16<false, false>(kP > 1 ? add[q][1][nt] : o[q][1][nt], ca[2], ca[3], cb[2], cb[3], b0[p], b1[p]);
            }
          }
        }
      }
      if (kP > 1 && (mt == kTiles - 1 || (kSplit && (mt & 1)))) {
#pragma unroll
        for (int i = 0; i < kG * 2 * NT * 4; ++i) {
          (&o[0][0][0][0])[i] += (&add[0][0][0][0])[i];
          (&add[0][0][0][0])[i] = 0.f;
        }
      }
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
            make_float4(up ? o[1][0][nt][c] : o[0][0][nt][c], up ? o[1][0][nt][c + 2] : o[0][0][nt][c + 2],
                        up ? o[1][1][nt][c] : o[0][1][nt][c], up ? o[1][1][nt][c + 2] : o[0][1][nt][c + 2]);
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

// Parts -> rows, a warp each: up to 24 parts are under way at once (12 had taken 9.7 us for 1792 rows of 20).
constexpr int kJoinThr = 128;
template <typename T>
__global__ void __launch_bounds__(kJoinThr) attn4_join(const __grid_constant__ AttnArgs a, const __grid_constant__ Attn4Plan plan) {
  pdl_wait_prior();
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * (kJoinThr / 32) + (threadIdx.x >> 5), n_rows = (long long)a.B * a.H_q;
  if (row >= n_rows) return;
  const int b = (int)(row / a.H_q);
  int len = a.k_len[b];
  if (len < 0 || len > a.k_len_max || len > (long long)a.max_pages * a.page_size) len = 0;
  if (a.prefix_len == 0 && len <= plan.own_keys) return;  // written by its only part
  const int n_own = len > 0 ? (len - 1) / plan.own_keys + 1 : 0;
  Joined s = {{0.f, 0.f, 0.f, 0.f}, 0.f, -INFINITY};
  join_parts<24>(
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

template <typename T>
cudaError_t run(const AttnArgs& a, const Attn4Plan& plan, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (plan.n_pre > 0)
    e = plan.pre_rows == 256 ? attn4_prefix_tc_launch(a, plan, s) : go_by_columns<T, true>(plan.pre_rows, a, plan, s);
  if (e == cudaSuccess) e = go_by_columns<T, false>(plan.own_rows, a, plan, s);
  if (e != cudaSuccess || plan.n_pre + plan.n_own <= 1) return e;
  return launch_pdl(attn4_join<T>, dim3((unsigned)(((long long)a.B * a.H_q + kJoinThr / 32 - 1) / (kJoinThr / 32))), dim3(kJoinThr), 0, s, a, plan);
}

}  // namespace

cudaError_t attn4_launch(const AttnArgs& a, const Attn4Plan& plan, int dtype, cudaStream_t s) {
  return dtype == 0 ? run<float>(a, plan, s) : run<__nv_bfloat16>(a, plan, s);
}

}  // namespace provip
