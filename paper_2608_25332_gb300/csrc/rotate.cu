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
// A warp handles four heads of a row at a time: eight lanes a head, lane l with values 8 l .. + 7 and
// 64 + 8 l .. + 7, which are pairs. A row's 64 sines are worked out two a lane and passed round. Each value is
// read and written once; what bounds that beyond a thousand rows is the SMs' issue slots and integer units rather than
// HBM where heads are normed or brought to 4 bits. In a graph over inputs in turn: 9379 rows of 32 heads with norms 27 us
// (5.7 TB/s), 8725 of 64 heads to 4 bits 38 (4.8). 8725 rows of 96 heads into pages take 72 us (5.9 TB/s; 66 alone, with
// nothing of a pass before to be written back), 8725 of 64 heads out of 4 bits 33 (5.5). Below that it is the launch.
#include "common.cuh"
#include "kernels.h"

namespace provip {
namespace {

constexpr int kThr = 256;
// Rotation: rows ahead a warp, bytes of a row's piece at most, blocks an SM (the registers' limit; without rotation
// three: 700 rows of 64 heads to 4 bits 10 us, with two 12), rows from which pieces are that large. (A video's 9379 rows
// of 32 heads, normed, blocks shared out evenly: pieces of 2 KiB 38 us, 4 KiB 31, 8 KiB 37; three blocks an SM 33; four
// rows ahead instead of two, no change.)
constexpr int kRing = 2, kPieceBytes = 4096, kRotateBlocks = 2, kStoreBlocks = 3, kRotateWide = 512;
// Reading: blocks, an SM's.
constexpr int kReadBlocks = 12;

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

__device__ __forceinline__ float max_nan(float x, float y) {  // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
// A group's scale from its largest magnitude, the positive one of two.
__device__ __forceinline__ float scale_of(float most, bool positive, uint16_t& bits) {
  const __nv_bfloat16 h = __float2bfloat16_rn(positive ? most * -0.125f : most * 0.125f);
  bits = *reinterpret_cast<const uint16_t*>(&h);
  if (!(most < 0x1p100f)) bits = 0x7fff;
  if (most < 0x1p-123f) bits = 0;
  return __uint_as_float((uint32_t)bits << 16);
}
// The scale of group k of two (0: values 0 .. 7 of each lane) over the four lanes that hold it.
__device__ __forceinline__ float group_scale(const Raw<float>& raw, int k, uint16_t& bits) {
  float x[16];
  raw.get(x);
  float most = fabsf(x[8 * k]), top = x[8 * k];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    most = max_nan(most, fabsf(x[8 * k + i]));
    top = fmaxf(top, x[8 * k + i]);
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  }
  return scale_of(most, top == most, bits);
}
// bf16 as 16-bit integers: the largest unsigned one is the negative value of largest magnitude, where there is one,
// the largest signed one the positive value of largest magnitude, where there is one (NaN above all). Both go round
// in one word, the signed one shifted to be unsigned.
__device__ __forceinline__ float group_scale(const Raw<__nv_bfloat16>& raw, int k, uint16_t& bits) {
  const uint32_t w[4] = {raw.u[k].x, raw.u[k].y, raw.u[k].z, raw.u[k].w};
  uint32_t neg = __vmaxu2(__vmaxu2(w[0], w[1]), __vmaxu2(w[2], w[3]));
  uint32_t pos = __vmaxs2(__vmaxs2(w[0], w[1]), __vmaxs2(w[2], w[3]));
  neg = __vmaxu2(neg, neg >> 16);
  pos = __vmaxs2(pos, __byte_perm(pos, pos, 0x1032)) ^ 0x80008000u;
  uint32_t both = __byte_perm(neg, pos, 0x5410);
  both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 1));
  both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 2));
  both = __vmaxu2(both, 0x80008000u) & 0x7fff7fffu;  // magnitudes, 0 where there is none of that sign
  const uint32_t up = both & 0xffff0000u, down = both << 16;
  return scale_of(__uint_as_float(max(up, down)), up >= down, bits);
}
// 1 / d rounded to nearest, for a normal d of eight bits whose reciprocal is normal: a step of Newton's iteration,
// r + r (1 - d r), on the hardware's approximation (all 256 such fractions give __frcp_rn's result).
__device__ __forceinline__ float reciprocal(float d) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
  return fmaf(r, fmaf(-d, r, 1.f), r);
}
// Codes of eight values: four of them in each half of the result. No quotient is below -8.1, which rounds
// to -8. A sum with 2^23 + 264 has a unit of 1, and so 256 and the code in its lower half, nothing else up to bit 24.
// Two such sums side by side are cut off at 15 together; the next two, times 16, leave two codes in a byte of each half.
__device__ __forceinline__ uint32_t group_codes(const float* x, float d) {
  constexpr uint32_t most = 0x4c0f010fu;
  const float r = d == 0.f ? 0.f : reciprocal(d);
  uint32_t w[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    uint32_t n[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) n[i] = __float_as_uint(__fadd_rn(__fmul_rn(x[4 * k + i], r), 8388872.f));
    // (upper halves: 2^23 as a float is 0x4b00 there, and the lower sum's 0x4b00.... moves out)
    w[k] = __vminu2(n[0] + n[2] * 65536u, most) + __vminu2(n[1] + n[3] * 65536u, most) * 16u;
  }
  return __byte_perm(w[0], w[1], 0x6420);
}

// A head's row (eight lanes with 16 values each) into its place in 4-bit pages.
template <typename T>
__device__ __forceinline__ void store4bit(const Raw<T>& raw, uint8_t* codes, uint8_t* scales, int l, bool on) {
  uint16_t b0, b1;
  const float d0 = group_scale(raw, 0, b0), d1 = group_scale(raw, 1, b1);
  float x[16];
  raw.get(x);
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

// What a kind of rows (queries, keys, values) is cut into: pieces of `heads` heads, and blocks that share a piece's rows.
struct Share {
  int pieces, blocks;
};
struct Shares {
  Share of[3];
  int heads;
};

// Blocks: queries' pieces first, then keys', then values'; a row a warp at a time. A warp keeps what its piece needs of every row (frequencies, axes, norm weights) in registers;
// the rows' values come through a ring of its own in shared memory, kRing rows ahead, by bulk copies (heads of a
// row lie next to each other). Waits are bounded; one that gives up sets the error word and ends the warp once
// its copies are done.
template <typename T, bool kTurn>
__global__ void __launch_bounds__(kThr, kTurn ? kRotateBlocks : kStoreBlocks) rotate_kernel(const __grid_constant__ RotateArgs a, const __grid_constant__ Shares shares) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t full[kThr / 32][kRing];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane & 7;
  int n = a.T;
  if (a.n_rows) {
    const int m = *a.n_rows;
    if (blockIdx.x == 0 && threadIdx.x == 0 && (m < 0 || m > a.T)) set_error(a.err, kErrBadDeviceArg);
    n = min(m, a.T);
  }
  // 0: queries, 1: keys, 2: values
  int block = blockIdx.x;
  const int q_blocks = shares.of[0].pieces * shares.of[0].blocks, k_blocks = shares.of[1].pieces * shares.of[1].blocks;
  const int kind = block < q_blocks ? 0 : block < q_blocks + k_blocks ? 1 : 2;
  block -= kind == 0 ? 0 : kind == 1 ? q_blocks : q_blocks + k_blocks;
  const int blocks = kind == 0 ? shares.of[0].blocks : kind == 1 ? shares.of[1].blocks : shares.of[2].blocks;
  const int piece = block / blocks, step = blocks * (kThr / 32);
  int t = (block - piece * blocks) * (kThr / 32) + warp;
  if (t >= n) return;
  const int h_lo = piece * shares.heads, n_heads = min(shares.heads, (kind == 0 ? a.H_q : a.H_kv) - h_lo);
  const long long stride = (kind == 0 ? a.q_stride : kind == 1 ? a.k_stride : a.v_stride) * (long long)sizeof(T);
  const uint8_t* src = static_cast<const uint8_t*>(kind == 0 ? a.Q : kind == 1 ? a.K : a.V) + (size_t)h_lo * kHeadDim * sizeof(T);
  const uint32_t bytes = n_heads * kHeadDim * (int)sizeof(T);
  uint8_t* ring = smem + warp * (kRing * kPieceBytes);
  auto load = [&](int row, int stage) {  // (one lane)
    mbar_arrive_expect_tx(&full[warp][stage], bytes);
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     smem_u32(ring + stage * kPieceBytes)),
                 "l"(src + row * stride), "r"(bytes), "r"(smem_u32(&full[warp][stage]))
                 : "memory");
  };
  if (lane == 0) {
    for (int i = 0; i < kRing; ++i) mbar_init(&full[warp][i], 1);
    fence_mbar_init();
    for (int i = 0; i < kRing; ++i)
      if ((long long)t + (long long)i * step < n) load(t + i * step, i);
  }
  __syncwarp();
  T* out = kind == 0 ? static_cast<T*>(a.q_out) : kind == 1 ? static_cast<T*>(a.k_out) : nullptr;
  const long long o_stride = kind == 0 ? a.qo_stride : a.ko_stride;
  if (out) out += (size_t)h_lo * kHeadDim;
  const bool paged = kind != 0 && a.slot_map != nullptr, turn = kTurn && kind != 2;
  void* pages = kind == 1 ? a.k_pages : a.v_pages;
  // pairs 2 lane, 2 lane + 1: this lane's sines and cosines
  unsigned long long turns[2] = {0, 0};
  const int* pos[2] = {nullptr, nullptr};
  if (turn) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      turns[i] = a.turns[2 * lane + i];
      pos[i] = a.pos + a.axis[2 * lane + i] * a.pos_stride;
    }
  }
  const T* w = turn ? static_cast<const T*>(kind == 0 ? a.wq : a.wk) : nullptr;
  Raw<T> weights;
  if (w) weights.load(w + l * 8);
  // bytes of a head's row's places: in an output, and in pages from one head to the next
  const uint32_t lane_at = (uint32_t)((lane >> 3) * kHeadDim + l * 8);
  const size_t head4 = (size_t)kRow4 << a.page_shift;
  int p[2] = {0, 0}, slot = -1;
  auto fetch = [&](int row) {
    if (turn) {
      p[0] = __ldg(pos[0] + row);
      p[1] = __ldg(pos[1] + row);
    }
    if (paged) slot = __ldg(a.slot_map + row);
  };
  fetch(t);
  int stage = 0;
  uint32_t phase = 0;
  for (;;) {
    // y_i = x_i c_i - x_{i+64} s_i and y_{i+64} = x_{i+64} c_i + x_i s_i, each x with its norm weight: the four factors
    float c0[8], c1[8], s0[8], s1[8];
    if (turn) {
      float s2[2], c2[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int part = (int)(((unsigned long long)(long long)p[i] * turns[i]) >> 32);  // 2^-32 of a turn, signed
        sincospif((float)part * 0x1p-31f, &s2[i], &c2[i]);
        s2[i] *= a.factor;
        c2[i] *= a.factor;
      }
      float g[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) g[e] = 1.f;
      if (w) weights.get(g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float s = __shfl_sync(0xffffffffu, s2[i & 1], 4 * l + (i >> 1)), c = __shfl_sync(0xffffffffu, c2[i & 1], 4 * l + (i >> 1));
        c0[i] = c * g[i];
        s1[i] = s * g[i];
        c1[i] = c * g[i + 8];
        s0[i] = s * g[i + 8];
      }
    }
    const int row = t;
    long long at = slot;
    if (at >= a.n_slots) {
      if (paged && lane == 0) set_error(a.err, kErrBadDeviceArg);
      at = -1;
    }
    t += step;
    if (t < n) fetch(t);
    if (__any_sync(0xffffffffu, !mbar_wait(&full[warp][stage], phase, a.err))) {
      // the copies still in flight, from this row's on, once more with a limit
      int st = stage;
      uint32_t ph = phase;
      for (int i = 0; i < kRing && (long long)row + (long long)i * step < n; ++i) {
        mbar_wait(&full[warp][st], ph, a.err);
        if (++st == kRing) {
          st = 0;
          ph ^= 1;
        }
      }
      return;
    }
    const T* from = reinterpret_cast<const T*>(ring + stage * kPieceBytes);
    T* to = out ? out + row * o_stride + lane_at : nullptr;
    // this lane's head in pages: its row, or its codes and its scales
    const bool keep = paged && at >= 0;
    uint8_t* in_page = static_cast<uint8_t*>(pages);
    size_t scales = 0;
    if (keep) {
      if (a.four)
        in_page += place4(at, h_lo + (lane >> 3), a.H_kv, a.page_shift, &scales);
      else
        in_page += (((size_t)at * a.H_kv + h_lo) * kHeadDim + lane_at) * sizeof(T);
    }
#pragma unroll 1
    for (int h4 = 0; h4 < n_heads; h4 += 4) {
      const bool on = h4 + (lane >> 3) < n_heads;
      Raw<T> now;
      now.load(from + (on ? lane_at : (uint32_t)(l * 8)) + h4 * kHeadDim);
      if (turn) {
        float x[16], r = 1.f;
        now.get(x);
        if (w) {
          float ss = 0.f, st = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            ss = fmaf(x[e], x[e], ss);
            st = fmaf(x[e + 8], x[e + 8], st);
          }
          ss += st;
#pragma unroll
          for (int o = 1; o < 8; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
          r = rsqrtf(ss * (1.f / kHeadDim) + a.eps);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = x[e], v = x[e + 8];
          x[e] = u * c0[e] - v * s0[e];
          x[e + 8] = v * c1[e] + u * s1[e];
        }
        if (w) {
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e] *= r;
        }
        now.set(x);
      }
      // (4 bits take in what k_out holds)
      if (keep && a.four) store4bit(now, in_page + (h4 * head4), in_page + (h4 * head4 + scales), l, on);
      if (!on) continue;
      if (to) now.store(to + h4 * kHeadDim);
      if (keep && !a.four) now.store(reinterpret_cast<T*>(in_page) + h4 * kHeadDim);
    }
    __syncwarp();  // every lane has read the stage
    if (lane == 0 && (long long)row + (long long)kRing * step < n) load(row + kRing * step, stage);
    if (++stage == kRing) {
      stage = 0;
      phase ^= 1;
    }
    if (t >= n) break;
  }
}

// Pieces of 4 KiB (sixteen heads in bf16, eight in fp32) where the rows fill the SMs with them, else of four heads.
// All blocks run at once and go through their piece's rows, so pieces get blocks by what a row of theirs costs, in
// turns of four heads: the sines and the norm weights are worth two of them, bringing four heads to 4 bits one and a
// half more, a copy's way through shared memory one. (9379 rows of 28 and 4 heads: rotated 31 us with blocks shared out
// evenly, 27 so; with values into pages 39 and 33. Values' copies at no cost: 41.)
template <typename T, bool kTurn>
cudaError_t rotate_go(const RotateArgs& a, int sms, cudaStream_t s) {
  static std::atomic<bool> configured[64];  // per device, zero-initialised
  constexpr int smem = kThr / 32 * kRing * kPieceBytes;
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 0 && dev < 64 && !configured[dev]) {
    cudaError_t e = cudaFuncSetAttribute(rotate_kernel<T, kTurn>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  Shares n;
  n.heads = a.T >= kRotateWide ? kPieceBytes / (kHeadDim * (int)sizeof(T)) : 4;
  const int all = (a.T + kThr / 32 - 1) / (kThr / 32), most = (kTurn ? kRotateBlocks : kStoreBlocks) * sms;
  long long cost[3], sum = 0;  // of a row, in half turns
  for (int i = 0; i < 3; ++i) {
    const int H = (i == 0 ? a.Q : i == 1 ? a.K : a.V) ? (i == 0 ? a.H_q : a.H_kv) : 0;
    n.of[i].pieces = (H + n.heads - 1) / n.heads;
    cost[i] = (H + 3) / 4 * (i > 0 && a.four ? 5 : 2) + (kTurn && i < 2 ? 4 : a.four ? 0 : 2) * n.of[i].pieces;
    sum += cost[i];
  }
  int blocks = 0;
  for (int i = 0; i < 3; ++i) {
    if (n.of[i].pieces) n.of[i].blocks = (int)min((long long)all, max(cost[i] * most / (sum * n.of[i].pieces), 1ll));
    else n.of[i].blocks = 0;
    blocks += n.of[i].pieces * n.of[i].blocks;
  }
  rotate_kernel<T, kTurn><<<blocks, kThr, smem, s>>>(a, n);
  return cudaGetLastError();
}

// ---------------------------------------------------------------------------
// rows out of 4-bit pages: the same eight lanes a head. Lane l's values lie in 16 bytes of codes,
// which lanes l and l + 4 share.
// ---------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(kThr) read4_kernel(const __grid_constant__ Read4Args a) {
  const int lane = threadIdx.x & 31, l = lane & 7;
  const int h = blockIdx.y * 4 + (lane >> 3);
  if (h >= a.H_kv) return;
  const uint8_t* pages = blockIdx.z ? a.v_pages : a.k_pages;
  const long long stride = blockIdx.z ? a.v_stride : a.k_stride;
  T* out = static_cast<T*>(blockIdx.z ? a.v_out : a.k_out) + (size_t)h * kHeadDim + l * 8;
  const uint32_t half = l & 4 ? 0x7632 : 0x5410;
  for (int t = blockIdx.x * (kThr / 32) + (threadIdx.x >> 5); t < a.T; t += gridDim.x * (kThr / 32)) {
    const long long slot = __ldg(a.slot_map + t);
    if (slot < 0) continue;
    if (slot >= a.n_slots) {
      if (lane == 0) set_error(a.err, kErrBadDeviceArg);
      continue;
    }
    size_t behind;
    const uint8_t* at = pages + place4(slot, h, a.H_kv, a.page_shift, &behind);
    const uint4 codes = *reinterpret_cast<const uint4*>(at + (l & 3) * 16);
    const uint2 scales = *reinterpret_cast<const uint2*>(at + behind);
    const uint32_t c[2] = {__byte_perm(codes.x, codes.z, half), __byte_perm(codes.y, codes.w, half)};
    const uint32_t b[2] = {scales.x, scales.y};
    float x[16];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float d = __uint_as_float(l & 4 ? b[k] & 0xffff0000u : b[k] << 16);
      // (2^23 + n less 2^23 + 8: n - 8 exactly)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[8 * k + e] = d * (__uint_as_float(0x4b000000u | ((c[k] >> (4 * e)) & 15u)) - 8388616.f);
    }
    Raw<T> r;
    r.set(x);
    r.store(out + t * stride);
  }
}

template <typename T>
cudaError_t read4_go(const Read4Args& a, int blocks, cudaStream_t s) {
  const int pieces = (a.H_kv + 3) / 4, all = (a.T + kThr / 32 - 1) / (kThr / 32), most = blocks / (2 * pieces);
  read4_kernel<T><<<dim3((unsigned)min(all, max(most, 1)), pieces, 2), kThr, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t rotate_launch(const RotateArgs& a, int dtype, int sms, cudaStream_t s) {
  if (a.turn) return dtype == 0 ? rotate_go<float, true>(a, sms, s) : rotate_go<__nv_bfloat16, true>(a, sms, s);
  return dtype == 0 ? rotate_go<float, false>(a, sms, s) : rotate_go<__nv_bfloat16, false>(a, sms, s);
}

cudaError_t read4_launch(const Read4Args& a, int dtype, int sms, cudaStream_t s) {
  const int blocks = kReadBlocks * sms;
  return dtype == 0 ? read4_go<float>(a, blocks, s) : read4_go<__nv_bfloat16>(a, blocks, s);
}

}  // namespace provip
