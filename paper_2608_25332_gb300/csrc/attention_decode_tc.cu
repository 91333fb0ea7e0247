// One token per request against its own pages (bf16, up to eight query heads a group): the
// keys are the rows of the tensor-core tiles.
//
// Bound by HBM: every key and value row of a request is read once for the R heads of its
// group, and there are only R query rows to multiply it with. So the products are transposed,
// with the tile of 128 keys as the 128 rows of the MMA and the heads as its columns (N = 16,
// the fewest; columns past R hold anything and are never read):
//   S^T = K Q^T    8 tcgen05.mma (M = 128 keys, N = 16, K = 16), a thread per key then has R
//                  scores to weigh, instead of one thread 128;
//   P^T            2^(s - m) in fp32, to bf16 in shared memory [head][key] (the second
//                  product's only 16-bit operand type); per thread and head the sum of the
//                  values in fp32 for the log-sum-exp, and that of the rounded ones, by which
//                  O is divided so that its weights add up to one;
//   O^T += V^T P^T 8 tcgen05.mma (M = 128 elements, N = 16, K = 16 keys), V as it lies.
// No maximum is looked for while no value of P passes 2^10 (a vote of the tile's threads);
// at a unit's first tile and past that it is found and P formed again.
//
// Work. The tiles of all (request, key/value head) units lie end to end; CTA c of G takes
// tiles [c T / G, (c + 1) T / G), whatever the requests' lengths, so all CTAs end together (a
// few short requests: a unit each, which needs no scan of the lengths and no join). A
// unit inside one CTA's span is finished by it; one that a span's border cuts is written in
// pieces, at most two a CTA, which a second kernel joins. Two CTAs an SM, each with a ring
// of three 32 KiB stages that TMA fills across units.
// Roles: warps 0-3 softmax (thread = key, then element), warp 4 MMAs, warp 5 TMA.
// Every wait is bounded, from the last sign of elements computed again on (mbar_wait_beat); a timeout
// sets the device error word, the roles end, and the block when what it has issued is done (drain).
#include "attention_tc.cuh"

namespace provip {
namespace {

constexpr int kHeads = 8;      // query heads of a group, at most
constexpr int kCols = 16;      // columns of the MMAs
constexpr int kStages = 3;
constexpr int kQBytes = 2 * kHeads * 128;  // a unit's queries: two halves of 64 elements
constexpr int kPBytes = 2 * kHeads * 128;  // a tile's P^T: two halves of 64 keys
// an MMA reads 16 rows of an operand of 8: 1 KiB past it, which the layout keeps inside
constexpr size_t kSmem = (size_t)kStages * kStage + 2 * kQBytes + 2 * kPBytes + 1024 + 1024;
constexpr int kThr = 192;
constexpr uint32_t kTmemCols = 64;  // S twice, O
constexpr float kMostP = 1024.f;
constexpr uint32_t kIdescS = idesc_bf16_f32(kT, kCols);
constexpr uint32_t kIdescO = idesc_bf16_f32(kT, kCols) | (1u << 15);  // A's (V's) rows run along M
constexpr int kBoard = 4;

// a unit's tiles in this CTA's span
struct Piece {
  int b, g;          // request, key/value head (-1: none is left)
  int t_lo, nt;      // tiles of the unit
  int n_keys;        // keys from the first tile on
  bool whole;        // every tile of the unit
  uint32_t tile0;    // number of its first tile in the CTA
};

struct Ctl {
  Piece board[kBoard];
  uint64_t u_full[kBoard], u_empty[kBoard];
  uint64_t q_full[2], q_empty[2];
  uint64_t kv_full[kStages], kv_empty[kStages];
  uint64_t s_full[2], p_full[2];
  uint64_t o_done[2];  // by the tile's parity
  uint64_t mma_done;   // (drain)
  unsigned long long beat;  // when elements were last known to be computed again (mbar_wait_beat)
  float red[4][kHeads], red_w[4][kHeads], inv[kHeads];
  uint32_t tmem;
  uint32_t n_ld, n_q;  // loads issued
  volatile int fail;   // a wait has given up
};

__device__ __forceinline__ int unit_tiles(int k_len) { return max((k_len + kT - 1) / kT, 1); }
__device__ __forceinline__ int fitting_len(const AttnArgs& a, int n) {
  return n >= 0 && n <= a.k_len_max && n <= (long long)a.max_pages * a.page_size ? n : -1;
}
__device__ __forceinline__ int checked_len(const AttnArgs& a, int b) { return fitting_len(a, a.k_len[b]); }

__device__ __forceinline__ void soft_sync() { asm volatile("barrier.cta.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ bool soft_any(bool v) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.pred q, 1, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"((uint32_t)v)
      : "memory");
  return any != 0;
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float* v) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const float* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
               "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])),
               "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])),
               "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7]))
               : "memory");
}

// first tile of span c of G over T tiles
__device__ __forceinline__ long long span_start(long long T, int c, int G) {
  // (a 64-bit division takes a few hundred instructions)
  if (T < (1 << 22)) return (long long)((unsigned)T * (unsigned)c / (unsigned)G);
  return T * c / G;
}
// the last span that starts at or before tile f
__device__ __forceinline__ int span_of(long long f, long long T, int G) {
  if (T < (1 << 22)) return (int)((((unsigned)f + 1u) * (unsigned)G - 1u) / (unsigned)T);
  return (int)(((f + 1) * G - 1) / T);
}

// The warp's reduction of eight values a lane, in nine exchanges instead of forty: afterwards
// lane 4 h has that of value h.
template <typename Op>
__device__ __forceinline__ float reduce8(const float* x, Op op) {
  const int lane = threadIdx.x & 31;
  float v[4], u[2], w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool up = lane & 16;
    v[i] = op(up ? x[i + 4] : x[i], __shfl_xor_sync(0xffffffffu, up ? x[i] : x[i + 4], 16));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bool up = lane & 8;
    u[i] = op(up ? v[i + 2] : v[i], __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + 2], 8));
  }
  const bool up = lane & 4;
  w = op(up ? u[1] : u[0], __shfl_xor_sync(0xffffffffu, up ? u[0] : u[1], 4));
  w = op(w, __shfl_xor_sync(0xffffffffu, w, 2));
  return op(w, __shfl_xor_sync(0xffffffffu, w, 1));
}

// the warp's sum of the requests' tiles before each of 32 requests, and of all 32
__device__ __forceinline__ int tiles_before(int t, int lane, int& all) {
  int s = t;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  all = __shfl_sync(0xffffffffu, s, 31);
  return s - t;
}

// Where a wait has given up, loads into the block's shared memory and products in its tensor memory
// may still be under way. The warps that issued them (role 0 the products, 1 the loads) wait for them
// before the block ends, once more with a limit.
__device__ __forceinline__ void drain(Ctl& ctl, unsigned* err) {
  const int role = (int)(threadIdx.x >> 5) - 4;
  if (role == 0) {
    if (elect_one()) {  // the lane that issued the products
      tc_commit(&ctl.mma_done);
      mbar_wait(&ctl.mma_done, 0, err);
    }
  } else if (role == 1 && (threadIdx.x & 31) == 0) {
    for (uint32_t i = ctl.n_q > 2 ? ctl.n_q - 2 : 0; i < ctl.n_q; ++i) mbar_wait(&ctl.q_full[i & 1], (i >> 1) & 1u, err);
    for (uint32_t i = ctl.n_ld > kStages ? ctl.n_ld - kStages : 0; i < ctl.n_ld; ++i)
      mbar_wait(&ctl.kv_full[i % kStages], (i / kStages) & 1u, err);
  }
}

// Elements of a finished piece that are infinite or NaN though their weights are finite: again
// (attn_element_again). Reads them back from where this thread has stored them, which keeps all of
// it out of the unit's loop (inside, 64 requests of 32 heads on 4 had taken 26.4 us instead of 25.9).
template <int R>
__device__ __noinline__ void elements_again(const AttnArgs& a, const AttnSpans& sp, const Piece& x, const float* inv,
                                            unsigned long long* beat) {
  const int r = threadIdx.x, lo = x.t_lo * kT, hi = lo + min(x.nt * kT, x.n_keys);
  const bool last = x.whole && a.prefix_len == 0;
  const size_t row0 = (size_t)x.b * a.H_q + x.g * R, slot = 2 * (size_t)blockIdx.x + (x.t_lo == 0 ? 1 : 0);
  for (int h = 0; h < R; ++h) {
    __nv_bfloat16* op = static_cast<__nv_bfloat16*>(a.out) + (size_t)x.b * a.o_stride + (size_t)(x.g * R + h) * kHeadDim + r;
    float* po = x.whole ? sp.whole_o + (row0 + h) * kHeadDim + r : sp.piece_o + (slot * R + h) * kHeadDim + r;
    const bool odd = isfinite(inv[h]) && !isfinite(last ? __bfloat162float(*op) : *po);
    if (!__any_sync(0xffffffffu, odd)) continue;
    const float v = attn_element_again<__nv_bfloat16>(a, x.b, x.g * R + h, lo, hi, r, odd, beat);
    if (odd && last) *op = __float2bfloat16_rn(v);
    if (odd && !last) *po = v;
  }
}

template <int R>
__global__ void __launch_bounds__(kThr, 2)
    attn_keys_tc(int G, const __grid_constant__ AttnArgs a, const __grid_constant__ AttnSpans sp,
                 const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                 const __grid_constant__ CUtensorMap map_v) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ Ctl ctl;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(smem_raw);
  uint8_t* kv = smem_raw + (((base + 1023u) & ~1023u) - base);
  uint8_t* ps = kv + kStages * kStage;
  uint8_t* qs = ps + 2 * kPBytes;
  // lengths of 256 requests in the producer's registers, asked for while the block is set up
  constexpr int kHeld = 8;
  int held[kHeld];
  if (warp == 5 && !sp.by_unit) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = i * 32 + lane < a.B ? a.k_len[i * 32 + lane] : 0;
  }
  if (threadIdx.x == 0) {
    prefetch_tmap(&map_q);
    prefetch_tmap(&map_k);
    prefetch_tmap(&map_v);
    for (int n = 0; n < kBoard; ++n) {
      mbar_init(&ctl.u_full[n], 1);
      mbar_init(&ctl.u_empty[n], 5);
    }
    for (int n = 0; n < 2; ++n) {
      mbar_init(&ctl.q_full[n], 1);
      mbar_init(&ctl.q_empty[n], 1);
      mbar_init(&ctl.s_full[n], 1);
      mbar_init(&ctl.p_full[n], 4);
      mbar_init(&ctl.o_done[n], 1);
    }
    mbar_init(&ctl.mma_done, 1);
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&ctl.kv_full[s], 1);
      mbar_init(&ctl.kv_empty[s], 1);
    }
    ctl.fail = 0;
    ctl.beat = 0;
    fence_mbar_init();
  }
  if (warp == 0) {
    tmem_alloc(&ctl.tmem, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_allow_next();  // the joining kernel, which holds no tensor memory, may be scheduled
  const uint32_t tmem = ctl.tmem;

  if (warp == 4) {
    // ---- MMA issuer. A tile's product with V goes before the next one's with Q: with three
    // stages, the next K is only asked for once the last V but one is done with, and to wait
    // for it first had made the time of a tile the latency of a load ----
    const bool lead = elect_one();
    const uint64_t kd0 = smem_desc_sw128(smem_u32(kv)), vd0 = smem_desc_mn_sw128(smem_u32(kv));
    const uint64_t qd0 = smem_desc_sw128(smem_u32(qs)), pd0 = smem_desc_sw128(smem_u32(ps));
    uint32_t n = 0;  // tiles done
    bool live = true;
    // S^T of tile n from unit buffer qb
    auto scores = [&](uint32_t t, uint32_t qb) {
      const uint32_t ld = 2 * t, st = ld % kStages;
      live = live && warp_wait(&ctl.kv_full[st], (ld / kStages) & 1u, a.err, &ctl.beat);
      tc_fence_after();
      if (lead) {
        const uint64_t kd = kd0 + (uint64_t)(st * (kStage >> 4)), qd = qd0 + (uint64_t)(qb * (kQBytes >> 4));
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
          tc_mma_bf16(tmem + (t & 1) * kCols, kd + (uint64_t)(((ks >> 2) * kHalf + (ks & 3) * 32) >> 4),
                      qd + (uint64_t)(((ks >> 2) * (kQBytes / 2) + (ks & 3) * 32) >> 4), kIdescS, ks > 0 ? 1u : 0u);
        tc_commit(&ctl.s_full[t & 1]);
        tc_commit(&ctl.kv_empty[st]);
      }
    };
    auto values = [&](uint32_t t, bool first) {
      const uint32_t ld = 2 * t + 1, st = ld % kStages;
      live = live && warp_wait(&ctl.kv_full[st], (ld / kStages) & 1u, a.err, &ctl.beat);
      live = live && warp_wait(&ctl.p_full[t & 1], (t >> 1) & 1u, a.err, &ctl.beat);
      tc_fence_after();
      if (lead) {
        const uint64_t vd = vd0 + (uint64_t)(st * (kStage >> 4)), pd = pd0 + (uint64_t)((t & 1) * (kPBytes >> 4));
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
          tc_mma_bf16(tmem + 2 * kCols, vd + (uint64_t)(ks * 2048 >> 4),
                      pd + (uint64_t)(((ks >> 2) * (kPBytes / 2) + (ks & 3) * 32) >> 4), kIdescO,
                      first && ks == 0 ? 0u : 1u);
        tc_commit(&ctl.kv_empty[st]);
        tc_commit(&ctl.o_done[t & 1]);
      }
    };
    for (uint32_t u = 0; live; ++u) {
      live = warp_wait(&ctl.u_full[u % kBoard], (u / kBoard) & 1u, a.err, &ctl.beat);
      const Piece& x = ctl.board[u % kBoard];
      if (!live || x.g < 0) break;
      const int nt = x.nt;
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.u_empty[u % kBoard]);
      live = warp_wait(&ctl.q_full[u & 1], (u >> 1) & 1u, a.err, &ctl.beat);
      for (int j = 0; live && j <= nt; ++j) {
        if (j > 0) values(n + j - 1, j == 1);
        if (j < nt) {
          scores(n + j, u & 1);
          if (j == nt - 1 && lead) tc_commit(&ctl.q_empty[u & 1]);
        }
      }
      n += nt;
    }
    if (!live) ctl.fail = 1;
  } else if (warp == 5) {
    // ---- producer: the CTA's span, cut into pieces, and their loads ----
    const int box = min(a.page_size, kT);
    bool live = true;
    uint32_t n_ld = 0, n_q = 0, u = 0, tile0 = 0;
    long long f = 0, f_end = 1, f_b = 0, T = 0;  // this CTA's tiles; the first of request b
    int b = 0, k_len = 0, nt_b = 1;
    if (sp.by_unit) {
      // a unit each: nothing to share out
      b = (int)blockIdx.x / a.H_kv;
      k_len = checked_len(a, b);
      if (k_len < 0 && lane == 0) set_error(a.err, kErrBadDeviceArg);
      k_len = max(k_len, 0);
      nt_b = unit_tiles(k_len);
      f = (long long)((int)blockIdx.x - b * a.H_kv) * nt_b;
      f_end = f + nt_b;
    } else {
      // (past 256 requests the lengths are read twice)
#pragma unroll
      for (int i = 0; i < kHeld; ++i) held[i] = fitting_len(a, held[i]);
      auto len_of = [&](int i) { return i * 32 + lane < a.B ? checked_len(a, i * 32 + lane) : 0; };
      // all tiles, and the tiles of the requests before each
      auto count = [&](int i, int k) {
        int all;
        const int t = i * 32 + lane < a.B ? unit_tiles(k) : 0, before = tiles_before(t, lane, all);
        if (blockIdx.x == 0 && i * 32 + lane < a.B) {
          sp.before[i * 32 + lane] = T + before;
          if (k < 0) set_error(a.err, kErrBadDeviceArg);
        }
        T += all;
      };
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (i * 32 < a.B) count(i, held[i]);
      for (int i = kHeld; i * 32 < a.B; ++i) count(i, len_of(i));
      if (blockIdx.x == 0 && lane == 0) sp.before[a.B] = T;
      T *= a.H_kv;
      f = span_start(T, (int)blockIdx.x, G);
      f_end = span_start(T, (int)blockIdx.x + 1, G);
      // the request that holds tile f: its tiles, and those before it
      long long done = 0;
      auto look = [&](int i, int k) {
        int all;
        const int t = i * 32 + lane < a.B ? unit_tiles(k) : 0, before = tiles_before(t, lane, all);
        const bool here = (done + all) * a.H_kv > f;
        if (here) {
          const int src = 31 - __clz(__ballot_sync(0xffffffffu, t > 0 && (done + before) * a.H_kv <= f));
          b = i * 32 + src;
          k_len = max(__shfl_sync(0xffffffffu, k, src), 0);
          nt_b = __shfl_sync(0xffffffffu, t, src);
          f_b = (done + __shfl_sync(0xffffffffu, before, src)) * a.H_kv;
        }
        done += all;
        return here;
      };
      bool here = f >= f_end;  // a span without tiles looks for nothing
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (!here && i * 32 < a.B) here = look(i, held[i]);
      for (int i = kHeld; !here && i * 32 < a.B; ++i) here = look(i, len_of(i));
    }
    const long long f0 = f, f0_b = f_b;
    const int b0 = b, nt0_b = nt_b;
    // One tile, K or V, into the next stage. A lane's page is looked up once for both, a tile
    // ahead.
    int row = 0, next = 0;
    auto row_of = [&](const Piece& x, int j) {
      if (j >= x.nt || lane * box >= min(kT, x.n_keys - j * kT)) return 0;
      return (int)attn_slot(a, a.block_table + (size_t)x.b * a.max_pages, (x.t_lo + j) * kT + lane * box);
    };
    auto load = [&](const Piece& x, int j, bool v) {
      const uint32_t st = n_ld % kStages, ph = (n_ld / kStages) & 1u;
      ++n_ld;
      const int n = min(kT, x.n_keys - j * kT), boxes = n > 0 ? (n + box - 1) / box : 0;
      if (!v) {
        row = next;
        next = row_of(x, j + 1);
      }
      bool ok = true;
      if (lane == 0) {
        ok = !ctl.fail && mbar_wait_beat(&ctl.kv_empty[st], ph ^ 1u, a.err, &ctl.beat);
        if (ok) mbar_arrive_expect_tx(&ctl.kv_full[st], (uint32_t)(boxes * box * 256));
      }
      __syncwarp();
      if (!__shfl_sync(0xffffffffu, ok ? 1 : 0, 0)) {
        --n_ld;
        return false;
      }
      uint8_t* dst = kv + st * kStage;
      const CUtensorMap* map = v ? &map_v : &map_k;
      if (lane < boxes) {
        tma_load_2d(dst + lane * box * 128, map, x.g * kHeadDim, row, &ctl.kv_full[st]);
        tma_load_2d(dst + kHalf + lane * box * 128, map, x.g * kHeadDim + 64, row, &ctl.kv_full[st]);
      }
      __syncwarp();
      return true;
    };
    for (; live; ++u) {
      Piece x;
      x.g = -1;
      if (f < f_end) {
        const int in = (int)(f - f_b);
        x.b = b;
        x.g = in / nt_b;
        x.t_lo = in % nt_b;
        x.nt = (int)min((long long)(nt_b - x.t_lo), f_end - f);
        x.n_keys = k_len - x.t_lo * kT;
        x.whole = x.nt == nt_b;
        x.tile0 = tile0;
        tile0 += x.nt;
        f += x.nt;
        if (f - f_b == (long long)nt_b * a.H_kv && f < f_end) {
          // the next request (never past the last: f < f_end <= T)
          f_b = f;
          ++b;
          k_len = max(checked_len(a, b), 0);
          nt_b = unit_tiles(k_len);
        }
      }
      live = warp_wait(&ctl.u_empty[u % kBoard], ((u / kBoard) & 1u) ^ 1u, a.err, &ctl.beat);
      if (!live) break;
      if (lane == 0) {
        ctl.board[u % kBoard] = x;
        mbar_arrive(&ctl.u_full[u % kBoard]);
      }
      __syncwarp();
      if (x.g < 0) break;
      next = row_of(x, 0);
      live = load(x, 0, false);
      if (!live) break;
      bool ok = true;
      if (lane == 0) {
        ok = mbar_wait_beat(&ctl.q_empty[u & 1], ((u >> 1) & 1u) ^ 1u, a.err, &ctl.beat);
        if (ok) {
          mbar_arrive_expect_tx(&ctl.q_full[u & 1], R * 256);
          uint8_t* q = qs + (u & 1) * kQBytes;
          tma_load_3d(q, &map_q, 0, x.g * R, x.b, &ctl.q_full[u & 1]);
          tma_load_3d(q + kQBytes / 2, &map_q, 64, x.g * R, x.b, &ctl.q_full[u & 1]);
        }
      }
      __syncwarp();
      live = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
      n_q += live;
      for (int j = 0; live && j < x.nt; ++j) {
        live = load(x, j, true);
        if (live && j + 1 < x.nt) live = load(x, j + 1, false);
      }
    }
    // what a border cuts: the first border inside a unit tells the joining kernel
    if (!sp.by_unit && lane == 0) {
      int unit = -1, last = -1;  // a span without tiles
      if (f0 < f_end) {
        last = 0;
        const int in = (int)(f0 - f0_b);
        const long long F = f0_b + in / nt0_b * nt0_b;
        // no other span starts inside the unit before this one: the tile before it lies in a
        // span that starts at or before the unit
        if (f0 > F && span_start(T, span_of(f0 - 1, T, G), G) <= F) {
          unit = b0 * a.H_kv + in / nt0_b;
          last = span_of(F + nt0_b - 1, T, G);  // the span that holds the unit's last tile
        }
      }
      sp.cut[blockIdx.x] = make_int2(unit, last);
    }
    if (!live) ctl.fail = 1;
    if (lane == 0) {
      ctl.n_ld = n_ld;
      ctl.n_q = n_q;
    }
  } else {
    // ---- softmax: a thread per key; in the epilogue a thread per element ----
    const int r = threadIdx.x;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const uint32_t to = tmem + 2 * kCols + lanes;
    const float sc = a.scale_log2;
    // this key's place in a row of P^T: 16-byte chunks swizzled by the row
    const uint32_t p_half = (uint32_t)(r >> 6) * (kPBytes / 2), p_chunk = (uint32_t)(r >> 3) & 7u, p_in = (uint32_t)(r & 7) * 2;
    // a wait that gave up: no more waits in the unit, but every barrier of the four warps is
    // met, and all of them leave before the next one
    bool failed = false;
    for (uint32_t u = 0;; ++u) {
      if (!failed) failed = !mbar_wait_beat(&ctl.u_full[u % kBoard], (u / kBoard) & 1u, a.err, &ctl.beat);
      failed = soft_any(failed);
      const Piece& x = ctl.board[u % kBoard];
      if (failed || x.g < 0) break;
      const int nt = x.nt;
      float m[R], l[R], lw[R];
#pragma unroll
      for (int h = 0; h < R; ++h) {
        m[h] = -INFINITY;
        l[h] = lw[h] = 0.f;
      }
      bool none = false;  // a head without a finite maximum so far
      for (int j = 0; j < nt; ++j) {
        const uint32_t n = x.tile0 + j, buf = n & 1;
        const bool key = r < x.n_keys - j * kT;
        if (!failed) failed = !mbar_wait_beat(&ctl.s_full[buf], (n >> 1) & 1u, a.err, &ctl.beat);
        __syncwarp();
        tc_fence_after();
        float s[8], p[R];
        // (rounded before the maximum is subtracted: with the two in one fma, scores past 2^28 would
        // pass their own maximum by more than the loop below allows)
        tmem_ld8(tmem + buf * kCols + lanes, s);
        tc_wait_ld();
#pragma unroll
        for (int h = 0; h < 8; ++h) s[h] = key && h < R ? __fmul_rn(s[h], sc) : -INFINITY;
        bool raise = j == 0 || none;
        for (;;) {
          if (raise) {
            // each head's largest score of the tile, over its 128 threads
            {
              const float w = reduce8(s, [](float x, float y) { return fmaxf(x, y); });
              if ((lane & 3) == 0) ctl.red[warp][lane >> 2] = w;
            }
            soft_sync();
            float f[8];
            bool any = false;
            none = false;
#pragma unroll
            for (int h = 0; h < R; ++h) {
              const float mx = fmaxf(fmaxf(ctl.red[0][h], ctl.red[1][h]), fmaxf(ctl.red[2][h], ctl.red[3][h]));
              const float mn = fmaxf(m[h], mx);
              f[h] = m[h] == mn ? 1.f : ex2_approx(m[h] - mn);
              any = any || f[h] != 1.f;
              m[h] = mn;
              none = none || mn == -INFINITY;
              l[h] *= f[h];
              lw[h] *= f[h];
            }
#pragma unroll
            for (int h = R; h < 8; ++h) f[h] = 1.f;
            if (j > 0 && any) {
              // O^T times f, once the product before is complete (the next waits for this P)
              if (!failed) failed = !mbar_wait_beat(&ctl.o_done[buf ^ 1], ((n - 1) >> 1) & 1u, a.err, &ctl.beat);
              __syncwarp();
              tc_fence_after();
              float o[8];
              tmem_ld8(to, o);
              tc_wait_ld();
#pragma unroll
              for (int h = 0; h < 8; ++h) o[h] *= f[h];
              tmem_st8(to, o);
              tc_wait_st();
            }
          }
          bool far = false;
#pragma unroll
          for (int h = 0; h < R; ++h) {
            p[h] = ex2_approx(s[h] - (m[h] == -INFINITY ? 0.f : m[h]));
            far = far || p[h] > kMostP;
          }
          // against the tile's own maximum no value passes 1, so this ends
          raise = soft_any(far);
          if (!raise) break;
        }
        uint8_t* pb = ps + buf * kPBytes + p_half + p_in;
#pragma unroll
        for (int h = 0; h < R; ++h) {
          const __nv_bfloat16 w = __float2bfloat16_rn(p[h]);
          l[h] += p[h];
          lw[h] += __bfloat162float(w);
          *reinterpret_cast<__nv_bfloat16*>(pb + h * 128 + ((p_chunk ^ (uint32_t)h) & 7u) * 16) = w;
        }
        if (x.n_keys - j * kT < kT) {
          // value rows past the end: zero before the product reads them (neighbours in a warp
          // write neighbouring 16 bytes: a row each had cost a microsecond of bank conflicts)
          const uint32_t ld = 2 * n + 1, st = ld % kStages;
          if (!failed) failed = !mbar_wait_beat(&ctl.kv_full[st], (ld / kStages) & 1u, a.err, &ctl.beat);
          uint8_t* vs = kv + st * kStage;
          for (int q = max(x.n_keys - j * kT, 0) * 8 + r; q < kT * 8; q += 128) {
            *reinterpret_cast<uint4*>(vs + q * 16) = make_uint4(0u, 0u, 0u, 0u);
            *reinterpret_cast<uint4*>(vs + kHalf + q * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.p_full[buf]);
      }
      // ---- epilogue: O^T / l, element r of every head ----
      {
        auto add = [](float x, float y) { return x + y; };
        float l8[8], w8[8];
#pragma unroll
        for (int h = 0; h < 8; ++h) {
          l8[h] = h < R ? l[h] : 0.f;
          w8[h] = h < R ? lw[h] : 0.f;
        }
        const float t = reduce8(l8, add), w = reduce8(w8, add);
        if ((lane & 3) == 0) {
          ctl.red[warp][lane >> 2] = t;
          ctl.red_w[warp][lane >> 2] = w;
        }
      }
      soft_sync();
      const size_t row0 = (size_t)x.b * a.H_q + x.g * R;
      const bool last = x.whole && a.prefix_len == 0;
      const size_t slot = x.whole ? 0 : 2 * (size_t)blockIdx.x + (x.t_lo == 0 ? 1 : 0);
      // The sums over the warps, the divisor and the log-sum-exp of each head, a thread a head,
      // while the last product runs. No weight: 0, or where every score is -inf 0 / 0, as
      // the formula has it.
      if (r < R) {
        const float t = (ctl.red[0][r] + ctl.red[1][r]) + (ctl.red[2][r] + ctl.red[3][r]);
        const float w = (ctl.red_w[0][r] + ctl.red_w[1][r]) + (ctl.red_w[2][r] + ctl.red_w[3][r]);
        float mh = m[0];
#pragma unroll
        for (int h = 1; h < R; ++h) mh = r == h ? m[h] : mh;
        const bool nil = last && x.n_keys > 0;
        const float lse = t != 0.f ? mh + lg2_approx(t) : nil ? NAN : -INFINITY;
        ctl.inv[r] = t != 0.f ? 1.f / w : nil ? NAN : 0.f;
        if (!last)
          (x.whole ? sp.whole_lse[row0 + r] : sp.piece_lse[slot * R + r]) = lse;
        else if (a.lse)
          a.lse[row0 + r] = lse * kLn2;
      }
      const uint32_t last_n = x.tile0 + nt - 1;
      if (!failed) failed = !mbar_wait_beat(&ctl.o_done[last_n & 1], (last_n >> 1) & 1u, a.err, &ctl.beat);
      __syncwarp();
      tc_fence_after();
      soft_sync();
      float o[8];
      tmem_ld8(to, o);
      tc_wait_ld();
      tc_fence_before();  // O^T is read before the next unit's first product, which waits for p_full
      float not_fine = 0.f;  // NaN once a value is not finite
#pragma unroll
      for (int h = 0; h < R; ++h) {
        // (an element without weight may hold anything)
        const float inv = ctl.inv[h], val = inv == 0.f ? 0.f : o[h] * inv;
        not_fine = fmaf(val, 0.f, not_fine);
        if (last) {
          __nv_bfloat16* op = static_cast<__nv_bfloat16*>(a.out) + (size_t)x.b * a.o_stride + (size_t)(x.g * R + h) * kHeadDim;
          op[r] = __float2bfloat16_rn(val);
        } else {
          float* po = x.whole ? sp.whole_o + (row0 + h) * kHeadDim : sp.piece_o + (slot * R + h) * kHeadDim;
          po[r] = val;
        }
      }
      if (__any_sync(0xffffffffu, isnan(not_fine))) elements_again<R>(a, sp, x, ctl.inv, &ctl.beat);
      __syncwarp();  // every lane has read the unit
      if (lane == 0) mbar_arrive(&ctl.u_empty[u % kBoard]);
    }
    if (failed) ctl.fail = 1;
  }
  tc_fence_before();
  __syncthreads();
  if (ctl.fail) {
    drain(ctl, a.err);
    __syncthreads();
  }
  if (warp == 0) tmem_dealloc(tmem, kTmemCols);
  // where this kernel runs beside the prefix's, it does not complete before it: the joining
  // kernel waits for this one alone
  if (blockIdx.x == 0 && threadIdx.x == 0) pdl_wait_prior();
}

// ---------------------------------------------------------------------------
// pieces and prefix parts -> rows: a warp per row
// ---------------------------------------------------------------------------
// with a prefix: a warp per (request, head); without: per border of two spans and head, for
// the unit that the border is the first to cut
__global__ void __launch_bounds__(256) attn_join_spans(const __grid_constant__ AttnArgs a, const __grid_constant__ AttnSpans sp) {
  pdl_wait_prior();
  const int lane = threadIdx.x & 31, R = a.H_q / a.H_kv, G = sp.n_spans;
  const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long n_rows = (long long)a.T_q * a.H_q;
  long long row;
  int b, h, hd, c0 = 0, c1 = 0;  // c0, c1: the spans that hold the unit's first and last tile
  if (a.prefix_len > 0) {
    if (w >= n_rows) return;
    row = w;
    b = (int)((unsigned)w / (unsigned)a.H_q);  // (B H_q fits 31 bits)
    h = (int)w - b * a.H_q;
    hd = h % R;
  } else {
    const int c = 1 + (int)((unsigned)w / (unsigned)R);
    if (c >= G) return;
    const int2 cut = sp.cut[c];
    if (cut.x < 0) return;
    hd = (int)w - (c - 1) * R;
    b = cut.x / a.H_kv;
    h = cut.x % a.H_kv * R + hd;
    row = (long long)b * a.H_q + h;
    // (the border cuts the unit, so the tile before it lies in the nearest span that has any)
    c0 = c - 1;
    while (c0 > 0 && sp.cut[c0].y < 0) --c0;
    c1 = cut.y;
  }
  // what is needed later is asked for now
  const int k_len = checked_len(a, b);
  const bool scan = a.prefix_len > 0 && !sp.by_unit;
  const long long all = scan ? sp.before[a.B] : 0, first = scan ? sp.before[b] : 0, next = scan ? sp.before[b + 1] : 0;
  Joined s = {{0.f, 0.f, 0.f, 0.f}, 0.f, -INFINITY};
  join_parts(
      s, sp.n_prefix, [&](int p) { return a.part_lse[p * n_rows + row]; },
      [&](int p) { return a.part_o + (p * n_rows + row) * kHeadDim; });
  if (scan) {
    const long long T = all * a.H_kv, nt = next - first, F = first * a.H_kv + h / R * nt;
    c0 = span_of(F, T, G);
    c1 = span_of(F + nt - 1, T, G);
  }
  if (c0 == c1) {
    join_parts(
        s, 1, [&](int) { return sp.whole_lse[row]; }, [&](int) { return sp.whole_o + row * kHeadDim; });
  } else {
    auto slot = [&](int p) { return (size_t)(2 * (c0 + p) + (p == 0 ? 1 : 0)) * R + hd; };
    auto empty = [&](int p) { return p > 0 && sp.cut[c0 + p].y < 0; };  // a span without tiles (its slot: anything)
    join_parts(
        s, c1 - c0 + 1, [&](int p) { return empty(p) ? -INFINITY : sp.piece_lse[slot(p)]; },
        [&](int p) { return sp.piece_o + slot(p) * kHeadDim; });
  }
  const int n_keys = a.prefix_len + max(k_len, 0);
  const float den = s.w == 0.f ? (n_keys > 0 ? NAN : 1.f) : s.w;  // every score -inf: 0 / 0, as the formula has it
  float o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = s.o[e] / den;
  store4(static_cast<__nv_bfloat16*>(a.out) + (size_t)b * a.o_stride + (size_t)h * kHeadDim + lane * 4, o);
  if (lane == 0 && a.lse) a.lse[row] = s.w == 0.f ? (n_keys > 0 ? NAN : -INFINITY) : s.lse() * kLn2;
}

template <int R>
cudaError_t launch(const AttnArgs& a, const AttnSpans& sp, const CUtensorMap& q, const CUtensorMap& k,
                   const CUtensorMap& v, cudaStream_t s) {
  static std::atomic<bool> configured[64];  // per device, zero-initialised
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 0 && dev < 64 && !configured[dev]) {
    cudaError_t e = cudaFuncSetAttribute(attn_keys_tc<R>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  // beside the prefix's kernel, where there is one (whose results it does not read)
  if (sp.n_prefix > 0) return launch_pdl(attn_keys_tc<R>, dim3(sp.n_spans), dim3(kThr), kSmem, s, sp.n_spans, a, sp, q, k, v);
  attn_keys_tc<R><<<sp.n_spans, kThr, kSmem, s>>>(sp.n_spans, a, sp, q, k, v);
  return cudaGetLastError();
}

}  // namespace

cudaError_t attn_keys_launch(const AttnArgs& a, const AttnSpans& sp, cudaStream_t s) {
  CUtensorMap q, k, v;
  const int R = a.H_q / a.H_kv;
  const uint32_t box = (uint32_t)(a.page_size < kT ? a.page_size : kT);
  const uint64_t rows = (uint64_t)a.n_pages * a.page_size;
  if (make_tmap_bf16_heads(&q, a.Q, (uint64_t)a.T_q, (uint64_t)a.H_q, (uint64_t)a.q_stride * 2, (uint32_t)R, 1) ||
      make_tmap_bf16_2d(&k, a.K, rows, (uint64_t)a.H_kv * kHeadDim, (uint64_t)a.k_stride * 2, box) ||
      make_tmap_bf16_2d(&v, a.V, rows, (uint64_t)a.H_kv * kHeadDim, (uint64_t)a.v_stride * 2, box))
    return cudaErrorInvalidValue;
  cudaError_t e;
  switch (R) {
    case 1: e = launch<1>(a, sp, q, k, v, s); break;
    case 2: e = launch<2>(a, sp, q, k, v, s); break;
    case 3: e = launch<3>(a, sp, q, k, v, s); break;
    case 4: e = launch<4>(a, sp, q, k, v, s); break;
    case 5: e = launch<5>(a, sp, q, k, v, s); break;
    case 6: e = launch<6>(a, sp, q, k, v, s); break;
    case 7: e = launch<7>(a, sp, q, k, v, s); break;
    case 8: e = launch<8>(a, sp, q, k, v, s); break;
    default: return cudaErrorInvalidValue;
  }
  if (e != cudaSuccess) return e;
  const long long warps = a.prefix_len > 0 ? (long long)a.B * a.H_q : sp.by_unit ? 0 : (long long)(sp.n_spans - 1) * R;
  if (warps == 0) return cudaSuccess;
  return launch_pdl(attn_join_spans, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0, s, a, sp);
}

}  // namespace provip
