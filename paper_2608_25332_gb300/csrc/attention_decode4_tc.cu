// The shared prefix of a batch in pages of 4 bits, on the tensor cores (bf16 queries).
//
// Every request's query rows see the same keys, so there are rows enough for tcgen05.mma: a CTA takes two
// tiles of 128 packed (request, head of the group) rows of one key/value head against a part of the prefix,
// 128 keys at a time. A value d c (eight significant bits times four) has eleven: it is the sum of two bf16
// values, hi = d c rounded and lo = d c - hi, each exact from one packed multiply and one multiply-add, whatever
// the scales' range. So codes and scales become two bf16 operands of K and of V in shared memory, once for all
// rows, and
//   S = Q K_hi^T + Q K_lo^T    16 MMAs (M = N = 128, K = 16), S in tensor memory
//   P = 2^(s - m)              a thread per row, to bf16 over S's own columns
//   O += P V_hi + P V_lo       16 MMAs, P from tensor memory
// lose nothing but P's rounding. (Queries of 2^20 and more go in with a power of two of their row, so that S stays a
// float whatever the scales.) The eight elements of a 16-byte chunk lie in the order 0 4 1 5 2 6 3 7, as the
// codes give them: queries are staged in that order too, and the output's columns are read in it.
// The maximum is raised only where a tile's sum passes 2^10, or where a row has none yet (every score so far -inf),
// as for bf16 keys (attention_tc.cu).
//
// What bounds it: 64 requests of 28 heads over 4 (448 rows a head), 9251 keys, 23 us: 12 of them set-up, first loads
// and the last tile's way out, the rest 2.7 us for two tiles of rows and 128 keys, of which the MMAs are 2.1; the
// softmax and the expansion share the issue slots beside them. (With the scores of a row tile issued behind its own
// values' product, before the other tile's, K's operands were waited for: 4.0 us a tile; with a thread storing its row
// by itself, 26 in all; queries staged by half a warp a row, no change.) On mma.sync the whole call took 76 us with
// the codes taken apart for every 16 rows, 51 with operands expanded once for 128, and takes 35 here (31 in a graph). What
// the registers do not hold is 48 bytes a thread in places (416 instructions a CTA go there, of tens of thousands).
//
// Roles (640 threads): warps 0-7 softmax, a tile of rows to each four; warp 8 issues the MMAs; warps 12-15 expand
// K's codes, warps 16-19 V's, a key's row a thread, K for the next tile while the softmax works, V when the product
// before has read the buffer; the first of each four loads, by bulk copies. Two row tiles share every operand
// and keep the tensor cores busy for one while the other's softmax runs. Every wait is bounded; one that gives up
// sets the error word and ends its role, the other roles' waits then run out likewise, and the block ends when what it
// has issued is done.
#include "attention_tc.cuh"

namespace provip {
namespace {

constexpr int kSoftWarps = 8, kMmaWarp = 8, kExpandWarp = 12;
constexpr int kThr = 640;
// registers a thread: what the softmax takes more than the launch's 96, the others leave
constexpr int kLaunchRegs = 96, kSoftRegs = 152, kMmaRegs = 40, kExpandRegs = 64;
static_assert(kSoftRegs * 256 + kMmaRegs * 128 + kExpandRegs * 256 <= kLaunchRegs * kThr, "register split");
constexpr int kRawBytes = kT * (kCodes4 + 8);  // K's or V's codes and scales of a tile
constexpr size_t kSmem = 6 * (size_t)kStage + 2 * kRawBytes + 1024;
constexpr uint32_t kIdescS = idesc_bf16_f32(kT, kT);
constexpr uint32_t kIdescO = idesc_bf16_f32(kT, kT) | (1u << 16);  // B's rows run along N
constexpr float kMostSum = 1024.f;

struct Ctl {
  uint64_t raw_full[2];            // codes and scales: K, V
  uint64_t full[2], empty[2];      // operands: K, V
  uint64_t s_full[2], p_full[2], o_full[2];
  uint64_t mma_done;               // (drain)
  uint32_t tmem;
  volatile int fail;
  float scale[2 * kT];             // of a row's scores (kept here over the roles' split: in registers it cost 0.5 us)
};

__device__ __forceinline__ bool wait_all(uint64_t* bar, uint32_t parity, unsigned* err) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, err));
}
// the four warps that expand K (v = 0) or V
__device__ __forceinline__ void expand_sync(int v) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(1 + v) : "memory"); }
__device__ __forceinline__ __nv_bfloat162 as_bf16(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
__device__ __forceinline__ uint32_t as_word(__nv_bfloat162 v) { return *reinterpret_cast<const uint32_t*>(&v); }
__device__ __forceinline__ void scale_o(uint32_t to, float f) {
  for (int z = 0; z < kHeadDim / 32; ++z) {
    uint32_t w[32];
    tmem_ld32(to + z * 32, reinterpret_cast<float*>(w));
    tc_wait_ld();
#pragma unroll
    for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) * f);
    tmem_st32(to + z * 32, w);
  }
}

// This thread's key: its 16 pieces of eight values, hi and lo, into the two operand tiles.
__device__ __forceinline__ void expand_row(const uint8_t* raw, int r, bool on, uint32_t magic, uint8_t* to) {
  uint2 d = *reinterpret_cast<const uint2*>(raw + kT * kCodes4 + r * 8);
  if (!on) d = make_uint2(0u, 0u);  // past the end: zeros, whatever lies there
  const __nv_bfloat162 scale[4] = {as_bf16(__byte_perm(d.x, d.x, 0x1010)), as_bf16(__byte_perm(d.x, d.x, 0x3232)),
                                   as_bf16(__byte_perm(d.y, d.y, 0x1010)), as_bf16(__byte_perm(d.y, d.y, 0x3232))};
  const __nv_bfloat162 bias = __bfloat162bfloat162(__float2bfloat16_rn(136.f));
#pragma unroll 1
  for (int p = 0; p < 4; ++p) {
    const uint4 w = *reinterpret_cast<const uint4*>(raw + r * kCodes4 + 16 * p);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint32_t x = __byte_perm(q < 2 ? w.x : w.y, q < 2 ? w.z : w.w, q & 1 ? 0x7632 : 0x5410);
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        uint32_t v;  // 128 + n
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(v) : "r"(x >> (4 * t)), "n"(0x000f000fu), "r"(magic));
        const __nv_bfloat162 c = __hsub2(as_bf16(v), bias), h = __hmul2(c, scale[q]);
        hi[t] = as_word(h);
        lo[t] = as_word(__hfma2(c, scale[q], __hneg2(h)));
      }
      // elements 32 q + 8 p .. + 7: chunk 4 q + p of the row, swizzled by the row
      const int chunk = 4 * q + p;
      uint8_t* at = to + (chunk >> 3) * kHalf + r * 128 + (((chunk & 7) ^ (r & 7)) << 4);
      *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(at + kStage) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
  }
}

__global__ void __launch_bounds__(kThr, 1)
    attn4_prefix_tc(int part_keys, const __grid_constant__ AttnArgs a, uint32_t magic) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ Ctl ctl;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(smem_raw);
  uint8_t* qs = smem_raw + (((base + 1023u) & ~1023u) - base);
  uint8_t* kb = qs + 2 * kStage;  // K_hi, K_lo
  uint8_t* vb = kb + 2 * kStage;  // V_hi, V_lo
  uint8_t* raw = vb + 2 * kStage;
  const int R = a.group, kv_head = blockIdx.z, part = blockIdx.y;
  const int k_lo = part * part_keys, n_keys = min(a.prefix_len - k_lo, part_keys);
  const int nt = (n_keys + kT - 1) / kT;
  const int row0 = (int)blockIdx.x * 2 * kT, n_rows = (int)min((long long)a.B * R - row0, 2ll * kT);  // rows of the block
  const int n_live = n_rows > kT ? 2 : 1;  // row tiles
  // codes and scales of a tile, K's (v = 0) or V's, by one warp: a lane a copy
  const int v_role = warp >= kExpandWarp + 4 ? 1 : 0;
  const bool loader = warp == kExpandWarp || warp == kExpandWarp + 4;
  const int box = min(a.page_size, kT), box_row = (lane >> 1) * box;
  const bool codes = !(lane & 1);
  const uint32_t unit = codes ? kCodes4 : 8;
  auto page_of = [&](int t) {
    const int k = t * kT + box_row;
    return box_row < kT && k < n_keys ? __ldg(a.prefix_table + ((k_lo + k) >> a.page_shift)) : 0;
  };
  int page = 0, loads = 0;
  auto load = [&]() {
    const int t = loads, rows = min(kT, n_keys - t * kT), k = k_lo + t * kT + box_row;
    int p = page;
    page = page_of(t + 1);
    if (lane == 0) mbar_arrive_expect_tx(&ctl.raw_full[v_role], (uint32_t)(((rows + box - 1) & ~(box - 1)) * kRow4));
    __syncwarp();
    if (box_row < rows) {
      if ((unsigned)p >= (unsigned)a.n_pages) {
        set_error(a.err, kErrBadDeviceArg);
        p = 0;
      }
      const uint8_t* src = static_cast<const uint8_t*>(v_role ? a.V : a.K) + (size_t)p * ((uint32_t)(a.H_kv * kRow4) << a.page_shift) +
                           (((size_t)kv_head * kRow4 + (codes ? 0 : kCodes4)) << a.page_shift) + (size_t)(k & (a.page_size - 1)) * unit;
      uint8_t* dst = raw + v_role * kRawBytes + (codes ? 0 : kT * kCodes4) + box_row * unit;
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                   "l"(src), "r"(box * unit), "r"(smem_u32(&ctl.raw_full[v_role]))
                   : "memory");
    }
    __syncwarp();
    ++loads;
  };
  if (loader) {  // the first tile's are asked for while the block is set up
    page = page_of(0);
    if (lane == 0) {
      mbar_init(&ctl.raw_full[v_role], 1);
      fence_mbar_init();
    }
    __syncwarp();
    load();
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ctl.full[i], 4);
      mbar_init(&ctl.empty[i], 1);
      mbar_init(&ctl.s_full[i], 1);
      mbar_init(&ctl.p_full[i], 4);
      mbar_init(&ctl.o_full[i], 1);
    }
    mbar_init(&ctl.mma_done, 1);
    ctl.fail = 0;
    fence_mbar_init();
  }
  if (warp == 0) {
    tmem_alloc(&ctl.tmem, 512);
    tmem_relinquish();
  }
  // queries: a thread a row, in the chunks' order; rows past the last are zeros
  const int qi = warp >> 2, r = (warp & 3) * 32 + lane;  // (softmax warps) row tile, row of it
  const bool row_live = warp < kSoftWarps && qi * kT + r < n_rows;
  int b = 0, h = 0;
  if (row_live) {
    const unsigned row = (unsigned)(row0 + qi * kT + r);
    b = (int)(row / (unsigned)R);
    h = kv_head * R + (int)(row - (unsigned)b * (unsigned)R);
  }
  if (warp < kSoftWarps) {
    float sc = a.scale_log2;
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.Q) + (size_t)b * a.q_stride + (size_t)h * kHeadDim);
    auto stage = [&](int ch, uint4 x) {
      const uint4 y = make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410),
                                 __byte_perm(x.y, x.w, 0x7632));
      *reinterpret_cast<uint4*>(qs + qi * kStage + (ch >> 3) * kHalf + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = y;
    };
    uint32_t most = 0;  // largest magnitude, as bits, in each half
#pragma unroll 4
    for (int ch = 0; ch < 16; ++ch) {
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (row_live) x = __ldg(src + ch);
      stage(ch, x);
      most = __vmaxu2(most, __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
    }
    // 128 products of less than 2^20 and 2^100 sum up to a float. A row with larger queries is staged again, times a
    // power of two (exact but for what then lies below 2^-133), which its scores' scale makes up for.
    const int over = (int)(max(most & 0xffffu, most >> 16) >> 7) - (127 + 19);
    if (over > 0) {
      const __nv_bfloat162 down = __bfloat162bfloat162(__ushort_as_bfloat16((unsigned short)((127 - over) << 7)));
      auto times = [&](uint32_t w) { return as_word(__hmul2(as_bf16(w), down)); };
#pragma unroll 1
      for (int ch = 0; ch < 16; ++ch) {
        const uint4 x = __ldg(src + ch);
        stage(ch, make_uint4(times(x.x), times(x.y), times(x.z), times(x.w)));
      }
      sc *= __uint_as_float((uint32_t)(127 + over) << 23);
    }
    ctl.scale[qi * kT + r] = sc;
    fence_proxy_async_smem();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_allow_next();  // the own keys' kernel and the joining one, which hold no tensor memory, may be scheduled
  const uint32_t tmem = ctl.tmem;

  if (warp >= kExpandWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kExpandRegs));
    // ---- codes and scales to operands ----
    const int key = ((int)threadIdx.x - kExpandWarp * 32) & 127;
    const uint8_t* from = raw + v_role * kRawBytes;
    uint8_t* to = v_role ? vb : kb;
    bool live = true;
    for (int t = 0; t < nt; ++t) {
      // the operands before are read: K's by tile t - 1's scores, V's by its product
      if (live && t > 0) live = wait_all(&ctl.empty[v_role], (uint32_t)(t - 1) & 1u, a.err);
      if (live) live = wait_all(&ctl.raw_full[v_role], (uint32_t)t & 1u, a.err);
      expand_row(from, key, key < n_keys - t * kT, magic, to);
      fence_proxy_async_smem();
      expand_sync(v_role);  // (met by all four warps, whatever their waits gave; the codes are read)
      if (live && lane == 0) mbar_arrive(&ctl.full[v_role]);
      if (loader && live && t + 1 < nt) load();
    }
    if (!live) ctl.fail = 1;
    if (loader && !live) {
      // copies that may still be in flight: waited for once more, with a limit
      mbar_wait(&ctl.raw_full[v_role], (uint32_t)(loads - 1) & 1u, a.err);
      __syncwarp();
    }
  } else if (warp >= kMmaWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kMmaRegs));
    if (warp == kMmaWarp) {
      // ---- MMA issuer: the whole warp walks through the tiles, one lane issues ----
      const bool lead = elect_one();
      const uint64_t qd = smem_desc_sw128(smem_u32(qs)), kd = smem_desc_sw128(smem_u32(kb)), vd = smem_desc_mn_sw128(smem_u32(vb));
      bool live = true;
      // the values' products of tile t - 1 before the scores of tile t: K's next operands are still being written then
      for (int t = 0; live && t <= nt; ++t) {
        if (t > 0) {
          live = wait_all(&ctl.full[1], (uint32_t)(t - 1) & 1u, a.err);
          for (int i = 0; live && i < n_live; ++i) {
            live = wait_all(&ctl.p_full[i], (uint32_t)(t - 1) & 1u, a.err);
            tc_fence_after();
            if (lead && live) {
#pragma unroll
              for (int ks = 0; ks < 16; ++ks)  // hi, then lo
                tc_mma_bf16_ts(tmem + (2 + i) * kT, tmem + i * kT + (ks & 7) * 8,
                               vd + (uint64_t)(((ks >> 3) * kStage + (ks & 7) * 2048) >> 4), kIdescO, ks > 0 || t > 1 ? 1u : 0u);
              if (t == nt) tc_commit(&ctl.o_full[i]);
            }
          }
          // (only where a tile follows that waits for it, here and below: nothing arrives at the block's end)
          if (lead && live && t < nt) tc_commit(&ctl.empty[1]);
        }
        if (live && t < nt) {
          live = wait_all(&ctl.full[0], (uint32_t)t & 1u, a.err);
          tc_fence_after();
          if (lead && live) {
            for (int i = 0; i < n_live; ++i) {
#pragma unroll
              for (int ks = 0; ks < 16; ++ks) {
                const uint32_t off = ((ks >> 2) & 1) * kHalf + (ks & 3) * 32;
                tc_mma_bf16(tmem + i * kT, qd + (uint64_t)((i * kStage + off) >> 4), kd + (uint64_t)(((ks >> 3) * kStage + off) >> 4),
                            kIdescS, ks > 0 ? 1u : 0u);
              }
              tc_commit(&ctl.s_full[i]);
            }
            if (t + 1 < nt) tc_commit(&ctl.empty[0]);
          }
        }
        __syncwarp();
      }
      if (!live) {
        ctl.fail = 1;
        if (lead) {  // products under way
          tc_commit(&ctl.mma_done);
          mbar_wait(&ctl.mma_done, 0, a.err);
        }
        __syncwarp();
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    // ---- softmax: a thread per row ----
    const uint32_t ts = tmem + qi * kT + ((uint32_t)((warp & 3) * 32) << 16), to = ts + 2 * kT;
    const float sc = ctl.scale[qi * kT + r];
    float m = -INFINITY, l = 0.f;
    bool live = true;
    for (int t = 0; live && t < nt && qi < n_live; ++t) {
      live = wait_all(&ctl.s_full[qi], (uint32_t)t & 1u, a.err);
      if (!live) break;
      tc_fence_after();
      const int seen = n_keys - t * kT;
      float sum;
      uint32_t w[kT / 2];
      // as for bf16 keys: P against the maximum so far, which is raised where the tile's sum is too large, and looked
      // for where a row has none (the first tile's; later ones' where all scores before were -inf)
#pragma unroll 1
      for (bool raise = __any_sync(0xffffffffu, row_live && m == -INFINITY), raised = false;;) {
        if (raise) {
          raised = true;
          float mx = -INFINITY;
#pragma unroll 1
          for (int z = 0; z < kT; z += 64) {
            float v[64], top[8];
            tmem_ld64(ts + z, v);
            tc_wait_ld();
            if (seen < kT) {
#pragma unroll
              for (int e = 0; e < 64; ++e) v[e] = z + e < seen ? v[e] : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) top[e] = fmaxf(v[e], v[8 + e]);
#pragma unroll
            for (int e = 16; e < 64; e += 16)
#pragma unroll
              for (int k = 0; k < 8; ++k) top[k] = max3(top[k], v[e + k], v[e + 8 + k]);
            mx = fmaxf(mx, fmaxf(max3(top[0], top[1], top[2]), max3(max3(top[3], top[4], top[5]), top[6], top[7])));
          }
          const float mn = fmaxf(m, mx * sc);  // sc > 0: the maximum commutes with it
          const float f = m == mn ? 1.f : ex2_approx(m - mn);
          m = mn;
          if (t > 0) {
            l *= f;
            scale_o(to, f);
            tc_wait_st();
          }
        }
        const float mb = m == -INFINITY ? 0.f : m;
        // (scores are rounded before the maximum is subtracted, as that is: with the two in one fma, scores past 2^28
        // would pass their own maximum by more than the exponent holds)
        const uint64_t sc2 = pack2(sc, sc), mb2 = pack2(-mb, -mb);
        uint64_t s2[2] = {0, 0};
#pragma unroll
        for (int z = 0; z < 2; ++z) {  // (64 scores at a time, for the registers)
          float v[64];
          tmem_ld64(ts + z * 64, v);
          tc_wait_ld();
          if (seen < kT) {
#pragma unroll
            for (int e = 0; e < 64; ++e) v[e] = z * 64 + e < seen ? v[e] : -INFINITY;
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            float p0, p1;
            unpack2(add2(fma2(pack2(v[2 * e], v[2 * e + 1]), sc2, 0), mb2), p0, p1);
            p0 = ex2_approx(p0);
            p1 = ex2_approx(p1);
            s2[e & 1] = add2(s2[e & 1], pack2(p0, p1));
            w[z * 32 + e] = pack_bf16(p0, p1);
          }
        }
        float s0, s1;
        unpack2(add2(s2[0], s2[1]), s0, s1);
        sum = s0 + s1;
        raise = !raised && __any_sync(0xffffffffu, row_live && sum > kMostSum);
        if (!raise) break;
      }
      l += sum;
      tmem_st32(ts, w);
      tmem_st32(ts + 32, w + 32);
      tc_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.p_full[qi]);
    }
    if (live && qi < n_live) live = wait_all(&ctl.o_full[qi], 0, a.err);
    if (!live) ctl.fail = 1;
    if (live && qi < n_live) {
      tc_fence_after();
      // this thread's row of the parts (~0: none)
      const unsigned long long row = row_live ? ((size_t)part * a.B + b) * a.H_q + h : ~0ull;
      // (every score -inf: no weight)
      const float inv = l == 0.f ? 0.f : 1.f / l;
      // 64 columns of the warp's 32 rows at a time go through shared memory, where this tile's queries have been
      // read for the last time, so that half a warp stores a row's 256 bytes side by side
      float4* st = reinterpret_cast<float4*>(qs + qi * kStage) + (warp & 3) * 512;
#pragma unroll 1
      for (int z = 0; z < kHeadDim; z += 64) {
#pragma unroll
        for (int y = 0; y < 64; y += 32) {
          float o[32];
          tmem_ld32(to + z + y, o);
          tc_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            const int c = (y + e) / 4;
            st[lane * 16 + (c ^ (lane & 7))] = make_float4(o[e] * inv, o[e + 2] * inv, o[e + 4] * inv, o[e + 6] * inv);
            st[lane * 16 + ((c + 1) ^ (lane & 7))] = make_float4(o[e + 1] * inv, o[e + 3] * inv, o[e + 5] * inv, o[e + 7] * inv);
          }
        }
        __syncwarp();
#pragma unroll 4
        for (int i = 0; i < 32; i += 2) {
          const int at = i + (lane >> 4), c = lane & 15;
          const unsigned long long to_row = __shfl_sync(0xffffffffu, row, at);
          if (to_row != ~0ull) *reinterpret_cast<float4*>(a.part_o + to_row * kHeadDim + z + c * 4) = st[at * 16 + (c ^ (at & 7))];
        }
        __syncwarp();
      }
      if (row_live) a.part_lse[row] = l == 0.f ? -INFINITY : m == -INFINITY ? NAN : m + lg2_approx(l);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tmem_dealloc(tmem, 512);
}

}  // namespace

cudaError_t attn4_prefix_tc_launch(const AttnArgs& a, const Attn4Plan& plan, cudaStream_t s) {
  static std::atomic<bool> configured[64];  // per device, zero-initialised
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 0 && dev < 64 && !configured[dev]) {
    cudaError_t e = cudaFuncSetAttribute(attn4_prefix_tc, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    cudaFuncAttributes at;
    if (e == cudaSuccess) e = cudaFuncGetAttributes(&at, attn4_prefix_tc);
    if (e != cudaSuccess) return e;
    // a register split that the launch does not cover would wait for ever
    if (at.numRegs != kLaunchRegs) return cudaErrorInvalidConfiguration;
    configured[dev] = true;
  }
  const long long rows = (long long)a.B * a.group;
  attn4_prefix_tc<<<dim3((unsigned)((rows + 2 * kT - 1) / (2 * kT)), plan.n_pre, a.H_kv), kThr, kSmem, s>>>(plan.pre_keys, a, plan.regs[1]);
  return cudaGetLastError();
}

}  // namespace provip
