// Attention behind the pruning on the tensor cores (bf16, fp32 accumulation).
//
// A persistent CTA takes units: NQ tiles of 128 packed rows (attention.cuh) of one
// key/value head against a run of 128-key tiles. Per key tile and row tile:
//   S = Q K^T   8 tcgen05.mma (M = N = 128, K = 16), both operands in shared memory, S in
//               tensor memory;
//   P = 2^(s - m), a thread per row: the 128 scores in registers, running maximum and sum
//               in fp32, P to bf16 over S's own columns;
//   O += P V    8 tcgen05.mma, P read from tensor memory, V as it lies in memory (keys by
//               elements, an operand whose rows run along N), O in tensor memory.
// P is rounded to bf16 for its product (the only 16-bit operand type that V allows); the
// sum of a row adds the unrounded values. The maximum that P is taken against is raised, to
// the true one (whose P is then 1 and rounds to itself), only where a tile's values add up to
// more than 2^10: larger values of P cost no accuracy in floating point, O is rescaled a few
// times a row instead of at every tile, and the other tiles need no maximum at all, whose 64
// three-way comparisons had taken a third of a tile's time. S of a tile is complete after the
// product of the tile before (one thread issues both, and a commit covers all that it issued),
// so a rescale needs no further wait.
// Roles: warps 0 .. 4 NQ - 1 softmax, then one warp issues the MMAs, one the TMA loads, and one
// works the units out.
// K and V tiles share a ring of 32 KiB stages. While the softmax works on one row tile, the
// tensor cores multiply for the other (NQ = 2, one CTA an SM), or for the other CTA of the
// SM (NQ = 1, two CTAs).
// Value rows of a tile past the sequence's end (another sequence's, padding, a page's unused
// slots, a page not loaded) are zeroed in shared memory before the product.
// Every wait is bounded, from the last sign of rows computed again on (mbar_wait_beat); one that gives
// up sets the device error word and ends its role, the other roles' waits then run out likewise, and
// the block ends when what it has issued is done (drain).
#include "attention_tc.cuh"

namespace provip {
namespace {

constexpr float kMostSum = 1024.f;     // of a row's 128 values of P before its maximum is raised

template <int NQ>
struct Form {
  static constexpr int kStages = NQ == 2 ? 5 : 2;
  static constexpr int kSoft = 128 * NQ;               // softmax threads
  static constexpr int kThreads = kSoft + 128;         // + MMA, TMA and unit warps, an idle one
  static constexpr int kCtas = NQ == 2 ? 1 : 2;
  // registers a thread: a row's 128 scores live in the softmax warps'; the sum over the block
  // is what it is launched with (168 a thread and 128)
  static constexpr int kSoftRegs = NQ == 2 ? 224 : 208, kRestRegs = NQ == 2 ? 56 : 48;
  static constexpr size_t kSmem = (size_t)(NQ + kStages) * kStage + 1024;
  static constexpr uint32_t kCols = 256 * NQ;          // S and O of every row tile
};

struct Maps {
  CUtensorMap q, k, v, kp, vp;
};

// One unit, as its warp works it out and the other roles read it (a board of kBoard units in
// shared memory, which keeps the decoding out of their registers and way).
template <int NQ>
struct Unit {
  AttnSeq s;
  int g, part;       // key/value head (-1: no unit is left); slot of the partial results
  int tok0;          // first token of the first row tile
  int n_tok[NQ];     // tokens of each row tile
  int n_prefix;      // prefix keys of the list, their tiles
  int n_pt;
  int t_lo;          // the unit's first tile of the list
  int nt[NQ];        // tiles of each row tile
  int ntm;           // the most of them
  uint32_t load0, step0;  // numbers of its first K load and of its first step
};
constexpr int kBoard = 4;
// The MMAs' step j of a unit multiplies P of tile j - 1 with V and Q with K of tile j: the two
// loads it needs share a barrier, and so do the two stages it hands back. (A step has one load
// at least, so the producer is at most a ring of stages, five, ahead.)
constexpr int kSteps = 8;

template <int NQ>
struct Ctl {
  Unit<NQ> board[kBoard];
  uint64_t u_full[kBoard], u_empty[kBoard];
  uint64_t q_full, q_empty;
  uint64_t full[kSteps], empty[kSteps];
  uint64_t s_full[NQ], p_full[NQ], o_full[NQ];
  uint64_t mma_done;  // (drain)
  unsigned long long beat;  // when rows were last known to be computed again (mbar_wait_beat)
  uint32_t tmem;
  uint32_t armed, n_q;  // steps and queries that loads were issued for
  volatile int fail;    // a wait has given up
};

constexpr uint32_t kIdescS = idesc_bf16_f32(kT, kT);
constexpr uint32_t kIdescO = idesc_bf16_f32(kT, kT) | (1u << 16);  // B's rows run along N

// n scores, with those from number `from` on hidden
template <int N>
__device__ __forceinline__ void mask_from(float* x, int from) {
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = e < from ? x[e] : -INFINITY;
}
// the largest of 128 in eight chains
__device__ __forceinline__ float max128(const float* x) {
  float b[8];
#pragma unroll
  for (int z = 0; z < 8; ++z) b[z] = max3(x[z], x[8 + z], x[16 + z]);
#pragma unroll
  for (int e = 24; e < 120; e += 16) {
#pragma unroll
    for (int z = 0; z < 8; ++z) b[z] = max3(b[z], x[e + z], x[e + 8 + z]);
  }
#pragma unroll
  for (int z = 0; z < 8; ++z) b[z] = fmaxf(b[z], x[120 + z]);
  return fmaxf(max3(b[0], b[1], b[2]), max3(max3(b[3], b[4], b[5]), b[6], b[7]));
}
// this thread's row of O times f
__device__ __noinline__ void scale_o(uint32_t to, float f) {
  for (int z = 0; z < kHeadDim / 32; ++z) {
    uint32_t w[32];
    tmem_ld32(to + z * 32, reinterpret_cast<float*>(w));
    tc_wait_ld();
#pragma unroll
    for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) * f);
    tmem_st32(to + z * 32, w);
  }
}

// ---------------------------------------------------------------------------
// units
// ---------------------------------------------------------------------------
// the tiles of a unit whose sequence, head, part and first token are known
template <int NQ>
__device__ __forceinline__ void set_tiles(const AttnArgs& a, Unit<NQ>& x, int part, int n_parts) {
  const int TT = a.tile_tokens;
  x.n_pt = (x.n_prefix + kT - 1) / kT;
  int most = 0, tiles[NQ];
#pragma unroll
  for (int i = 0; i < NQ; ++i) {
    x.n_tok[i] = min(max(x.s.q_len - x.tok0 - i * TT, 0), TT);
    tiles[i] = 0;
    if (x.n_tok[i] > 0) {
      const int vis = attn_visible(a, x.s.q_len, x.s.k_len, x.tok0 + i * TT + x.n_tok[i] - 1);
      tiles[i] = x.n_pt + (vis + kT - 1) / kT;
    }
    most = max(most, tiles[i]);
  }
  const int per = (most + n_parts - 1) / n_parts;
  x.t_lo = min(part * per, most);
  x.ntm = min(x.t_lo + per, most) - x.t_lo;
#pragma unroll
  for (int i = 0; i < NQ; ++i) x.nt[i] = min(max(tiles[i] - x.t_lo, 0), x.ntm);
}

// paged: the units of the prefix (the tokens of every request against it), then those of the
// requests' own keys
template <int NQ>
__device__ __forceinline__ Unit<NQ> paged_unit(const AttnArgs& a, const AttnPlan& p, int u) {
  Unit<NQ> x;
  int part, n_parts;
  if (u < p.n_prefix_units) {
    n_parts = p.n_prefix_parts;
    part = u % n_parts;
    u /= n_parts;
    x.g = u % a.H_kv;
    x.tok0 = u / a.H_kv * NQ * a.tile_tokens;
    x.part = p.n_own_parts + part;
    x.s.q0 = 0;
    x.s.q_len = a.B;
    x.s.k_len = 0;
    x.s.k0 = 0;
    x.s.pages = nullptr;
    x.s.ok = true;
    x.n_prefix = a.prefix_len;
  } else {
    u -= p.n_prefix_units;
    n_parts = p.n_own_parts;
    x.g = u % a.H_kv;
    u /= a.H_kv;
    part = u % n_parts;
    x.s = attn_seq(a, u / n_parts);
    x.tok0 = 0;
    x.part = part;
    x.n_prefix = 0;
  }
  set_tiles(a, x, part, n_parts);
  return x;
}

// Contiguous keys: the units that have rows, in an order that their warp walks through. The
// sequences (and, where one's keys are too many, its heads) come in chunks whose keys and
// values stay in L2; within a chunk level by level, level l holding the l-th block of rows from
// each sequence's end, which sees the most keys, so that long units come first. The blocks of a
// chunk's sequences (256 at most) lie in the lanes' registers.
struct Walk {
  static constexpr int kHeld = 8;
  int nb[kHeld];   // blocks of sequence b0 + 32 i + lane
  int b0, n_seq;   // the chunk's sequences
  int g0, n_g;     // and heads
  int level, more; // the level, and how many like it follow (sequences of the same number of blocks)
  int base, cnt;   // units before this level, and of it
};
__device__ __forceinline__ void walk_level(const AttnArgs& a, Walk& w) {
  int n = 0;
  unsigned least = 0x7fffffffu;
#pragma unroll
  for (int i = 0; i < Walk::kHeld; ++i) {
    if (i * 32 >= w.n_seq) break;
    const bool has = w.nb[i] > w.level;
    n += __popc(__ballot_sync(0xffffffffu, has));
    if (has) least = min(least, (unsigned)w.nb[i]);
  }
  w.cnt = n * w.n_g * a.n_part;
  w.more = n ? (int)__reduce_min_sync(0xffffffffu, least) - w.level - 1 : 0;
}
template <int NQ>
__device__ __forceinline__ void walk_chunk(const AttnArgs& a, const AttnPlan& p, Walk& w) {
  const int lane = threadIdx.x & 31, rows = NQ * a.tile_tokens;
  w.n_seq = min(p.chunk_seqs, a.B - w.b0);
  w.n_g = min(p.chunk_heads, a.H_kv - w.g0);
#pragma unroll
  for (int i = 0; i < Walk::kHeld; ++i) {
    w.nb[i] = 0;
    if (i * 32 + lane < w.n_seq) {
      const AttnSeq s = attn_seq(a, w.b0 + i * 32 + lane);
      if (!s.ok) set_error(a.err, kErrBadDeviceArg);
      w.nb[i] = (s.q_len + rows - 1) / rows;
    }
  }
  w.level = 0;
  walk_level(a, w);
}
// unit u, which comes after the one asked for before; false: there is none
template <int NQ>
__device__ __forceinline__ bool walk_to(const AttnArgs& a, const AttnPlan& p, Walk& w, int u, Unit<NQ>& x) {
  while (u >= w.base + w.cnt) {
    if (w.cnt > 0) {
      const int skip = min((u - w.base) / w.cnt, w.more + 1);
      w.base += skip * w.cnt;
      w.level += skip;
      w.more -= skip;
      if (w.more < 0) walk_level(a, w);
    } else {
      w.g0 += w.n_g;
      if (w.g0 >= a.H_kv) {
        w.g0 = 0;
        w.b0 += w.n_seq;
        if (w.b0 >= a.B) return false;
      }
      walk_chunk<NQ>(a, p, w);
    }
  }
  int in = u - w.base;
  const int part = in % a.n_part;
  in /= a.n_part;
  x.g = w.g0 + in % w.n_g;
  in /= w.n_g;  // the in-th sequence that has this level
  int b = 0, nb = 0;
#pragma unroll
  for (int i = 0; i < Walk::kHeld; ++i) {
    if (i * 32 >= w.n_seq) break;
    const unsigned has = __ballot_sync(0xffffffffu, w.nb[i] > w.level);
    const int n = __popc(has);
    if (in >= 0 && in < n) {
      const int src = (int)__fns(has, 0, in + 1);
      b = w.b0 + i * 32 + src;
      nb = __shfl_sync(0xffffffffu, w.nb[i], src);
    }
    in -= n;
  }
  x.s = attn_seq(a, b);
  x.n_prefix = a.prefix_len;
  x.part = part;
  x.tok0 = (nb - 1 - w.level) * NQ * a.tile_tokens;
  set_tiles(a, x, part, a.n_part);
  return true;
}

// key of the list that tile t starts with
template <int NQ>
__device__ __forceinline__ int list_key(const Unit<NQ>& x, int t) {
  return t < x.n_pt ? t * kT : x.n_prefix + (t - x.n_pt) * kT;
}

// the k-th unit of this CTA: every other round runs backwards, so that the long units of
// one round meet the short ones of the next
__device__ __forceinline__ int unit_index(int k) {
  const int G = (int)gridDim.x, i = (int)blockIdx.x;
  return k * G + ((k & 1) ? G - 1 - i : i);
}

// 32 bytes of a thread's row: one store where the rows allow it
__device__ __forceinline__ void store32(char* p, const uint32_t* r, bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(r[0], r[1], r[2], r[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(r[4], r[5], r[6], r[7]);
  }
}

// O / l of a thread's row, its log-sum-exp: to memory, as the result or as a part. Kept out
// of line: its addresses would cost the tile loop registers. (One copy a kernel: shared by two, the
// compiler made stores of four bytes of its 32-byte ones.) Bound by the instructions of a
// single warp a scheduler; stores of whole 32-byte sectors need no exchange between lanes, and
// as pairs of 16 bytes they had made the pass of 8 prompts 3% longer.
template <int NQ>
__device__ __noinline__ void finish_rows(const AttnArgs& a, const Unit<NQ>& x, int i, int tok_in, int hid, float m,
                                         float l, uint32_t to, unsigned long long* beat) {
  const int lane = threadIdx.x & 31, r = threadIdx.x & 127;
  const int R = a.group, hd = r - tok_in * R;
  const int nt = x.nt[i];
  const bool row_live = tok_in < x.n_tok[i];
  const int h = x.g * R + hd, tok = x.tok0 + i * a.tile_tokens + tok_in;
  const size_t n_rows = (size_t)a.T_q * a.H_q, row = (size_t)(x.s.q0 + tok) * a.H_q + h;
  const bool partial = a.n_part > 1;
  // the part's keys of the list that this row sees
  const int lo = list_key(x, x.t_lo), hi = min(list_key(x, x.t_lo + nt), x.n_prefix + x.s.k_len - hid);
  const float inv = 1.f / l, lse = m + lg2_approx(l);
  char* dst = partial ? reinterpret_cast<char*>(a.part_o + ((size_t)x.part * n_rows + row) * kHeadDim)
                      : reinterpret_cast<char*>(static_cast<__nv_bfloat16*>(a.out) + (size_t)(x.s.q0 + tok) * a.o_stride +
                                                (size_t)h * kHeadDim);
  const bool wide = !__any_sync(0xffffffffu, (reinterpret_cast<uintptr_t>(dst) & 31u) != 0);
  float sum = 0.f;
  if (nt == 0) {
    // no keys at all for the tile (in this part)
    if (row_live) {
      const uint32_t zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      for (int e = 0; e < kHeadDim * (partial ? 4 : 2); e += 32) store32(dst + e, zero, wide);
      if (partial)
        a.part_lse[(size_t)x.part * n_rows + row] = -INFINITY;
      else if (a.lse)
        a.lse[row] = -INFINITY;
    }
    return;
  } else {
    const uint64_t inv2 = pack2(inv, inv);
    uint64_t s2[2] = {0, 0};
#pragma unroll 1
    for (int c = 0; c < 2; ++c) {
      float o[64];
      tmem_ld64(to + c * 64, o);
      tc_wait_ld();
#pragma unroll
      for (int e = 0; e < 64; e += 2) {
        const uint64_t v = fma2(pack2(o[e], o[e + 1]), inv2, 0);
        s2[(e >> 1) & 1] = add2(s2[(e >> 1) & 1], v);  // not finite once an element is not
        unpack2(v, o[e], o[e + 1]);
      }
      if (row_live) {
        if (partial) {
#pragma unroll
          for (int e = 0; e < 64; e += 8) store32(dst + (c * 64 + e) * 4, reinterpret_cast<const uint32_t*>(o) + e, wide);
        } else {
#pragma unroll
          for (int e = 0; e < 64; e += 16) {
            uint32_t w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = pack_bf16(o[e + 2 * k], o[e + 2 * k + 1]);
            store32(dst + (c * 64 + e) * 2, w, wide);
          }
        }
      }
      __syncwarp();  // the next round's load is the whole warp's
    }
    float s0, s1;
    unpack2(add2(s2[0], s2[1]), s0, s1);
    sum = s0 + s1;
  }
  tc_fence_before();  // O is read before the next unit's first product, which waits for p_full
  // a NaN sum is the row's own: no masked score, rescaling or overflow makes one (O times 1 / l is NaN throughout)
  const bool fine = isnan(l) || (l != 0.f && isfinite(sum) && isfinite(lse));
  if (row_live && fine) {
    if (partial)
      a.part_lse[(size_t)x.part * n_rows + row] = lse;
    else if (a.lse)
      a.lse[row] = lse * kLn2;
  }
  // rows that are not finite or have no weight: again by the definition
  __syncwarp();
  unsigned again = __ballot_sync(0xffffffffu, row_live && !fine);
  while (again) {
    const int src = __ffs(again) - 1;
    again &= again - 1;
    const int tk = __shfl_sync(0xffffffffu, tok, src), hh = __shfl_sync(0xffffffffu, h, src);
    const int khi = __shfl_sync(0xffffffffu, hi, src);
    float o[4];
    float le = attn_row_plain<__nv_bfloat16>(a, x.s, x.n_prefix, tk, hh, lo, khi, lane * 4, o, beat);
    const size_t rw = (size_t)(x.s.q0 + tk) * a.H_q + hh;
    if (partial) {
      store4(a.part_o + ((size_t)x.part * n_rows + rw) * kHeadDim + lane * 4, o);
      if (lane == 0) a.part_lse[(size_t)x.part * n_rows + rw] = le;
    } else {
      // every score is -inf: 0 / 0, as the formula has it (a row without keys is 0)
      if (le == -INFINITY && khi > lo) le = o[0] = o[1] = o[2] = o[3] = NAN;
      store4(static_cast<__nv_bfloat16*>(a.out) + (size_t)(x.s.q0 + tk) * a.o_stride + (size_t)hh * kHeadDim + lane * 4, o);
      if (lane == 0 && a.lse) a.lse[rw] = le * kLn2;
    }
  }
}

// Where a wait has given up, loads into the block's shared memory and products in its tensor memory
// may still be under way. The warps that issued them (role 0 the products, 1 the loads) wait for them
// before the block ends, once more with a limit. (A step whose loads were not all issued takes all
// of it.)
template <int NQ>
__device__ __forceinline__ void drain(Ctl<NQ>& ctl, unsigned* err) {
  const int role = (int)(threadIdx.x >> 5) - 4 * NQ;
  if (role == 0) {
    if (elect_one()) {  // the lane that issued the products
      tc_commit(&ctl.mma_done);
      mbar_wait(&ctl.mma_done, 0, err);
    }
  } else if (role == 1 && (threadIdx.x & 31) == 0) {
    if (ctl.n_q > 0) mbar_wait(&ctl.q_full, (ctl.n_q - 1) & 1u, err);
    for (uint32_t i = ctl.armed > kSteps ? ctl.armed - kSteps : 0; i < ctl.armed; ++i)
      mbar_wait(&ctl.full[i % kSteps], (i / kSteps) & 1u, err);
  }
}

// ---------------------------------------------------------------------------
// the kernel
// ---------------------------------------------------------------------------
template <int NQ>
__global__ void __launch_bounds__(Form<NQ>::kThreads, Form<NQ>::kCtas)
    attn_tc(int n_units, const __grid_constant__ AttnArgs a, const __grid_constant__ AttnPlan plan,
            const __grid_constant__ Maps maps) {
  using F = Form<NQ>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Ctl<NQ> ctl;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int R = a.group, TT = a.tile_tokens;
  const uint32_t base = smem_u32(smem_raw);
  uint8_t* qs = smem_raw + (((base + 1023u) & ~1023u) - base);
  uint8_t* kv = qs + NQ * kStage;
  if (threadIdx.x == 0) {
    prefetch_tmap(&maps.q);
    prefetch_tmap(&maps.k);
    prefetch_tmap(&maps.v);
    for (int n = 0; n < kBoard; ++n) {
      mbar_init(&ctl.u_full[n], 1);
      mbar_init(&ctl.u_empty[n], 4 * NQ + 2);
    }
    mbar_init(&ctl.q_full, 1);
    mbar_init(&ctl.q_empty, 1);
    mbar_init(&ctl.mma_done, 1);
    for (int s = 0; s < kSteps; ++s) {
      mbar_init(&ctl.full[s], 1);
      mbar_init(&ctl.empty[s], 1);
    }
    for (int i = 0; i < NQ; ++i) {
      mbar_init(&ctl.s_full[i], 1);
      mbar_init(&ctl.p_full[i], 4);
      mbar_init(&ctl.o_full[i], 1);
    }
    ctl.fail = 0;
    ctl.beat = 0;
    fence_mbar_init();
  }
  if (warp == 0) {
    tmem_alloc(&ctl.tmem, F::kCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_allow_next();  // the joining kernel, which holds no tensor memory, may be scheduled
  const uint32_t tmem = ctl.tmem;

  if (warp >= 4 * NQ) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(F::kRestRegs));
    if (warp == 4 * NQ) {
      // ---- MMA issuer: the whole warp walks through the tiles, one lane issues ----
      const bool lead = elect_one();
      const uint64_t qd = smem_desc_sw128(smem_u32(qs));
      const uint64_t kd0 = smem_desc_sw128(smem_u32(kv)), vd0 = smem_desc_mn_sw128(smem_u32(kv));
      // loads come in the order K_0 V_0 K_1 V_1 ..: stages of the next K and of the next V
      uint32_t sk = 0, sv = 1, step = 0, pq = 0, pp[NQ];
#pragma unroll
      for (int i = 0; i < NQ; ++i) pp[i] = 0;
      auto two_on = [](uint32_t& st) { st = st + 2 < F::kStages ? st + 2 : st + 2 - F::kStages; };
      bool live = true;
      for (uint32_t n = 0; live; ++n) {
        live = warp_wait(&ctl.u_full[n % kBoard], (n / kBoard) & 1u, a.err, &ctl.beat);
        const Unit<NQ>& x = ctl.board[n % kBoard];
        if (!live || x.g < 0) break;
        const int ntm = x.ntm;
        int nt[NQ];
#pragma unroll
        for (int i = 0; i < NQ; ++i) nt[i] = x.nt[i];
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.u_empty[n % kBoard]);
        if (ntm == 0) continue;
        live = warp_wait(&ctl.q_full, pq, a.err, &ctl.beat);
        pq ^= 1u;
        for (int j = 0; live && j <= ntm; ++j, ++step) {
          live = warp_wait(&ctl.full[step % kSteps], (step / kSteps) & 1u, a.err, &ctl.beat);
          const uint64_t kd = kd0 + (uint64_t)(sk * (kStage >> 4)), vd = vd0 + (uint64_t)(sv * (kStage >> 4));
#pragma unroll
          for (int i = 0; i < NQ; ++i) {
            const uint32_t ts = tmem + i * kT, to = tmem + (NQ + i) * kT;
            if (j > 0 && j <= nt[i]) {
              if (live) live = warp_wait(&ctl.p_full[i], pp[i], a.err, &ctl.beat);
              pp[i] ^= 1u;
              tc_fence_after();
              if (lead) {
                const uint32_t first = j > 1 ? 1u : 0u;
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                  tc_mma_bf16_ts(to, ts + ks * 8, vd + (uint64_t)(ks * 2048 >> 4), kIdescO, ks > 0 ? 1u : first);
                if (j == nt[i]) tc_commit(&ctl.o_full[i]);
              }
            }
            if (j < nt[i]) {
              tc_fence_after();
              if (lead) {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                  const uint64_t off = (uint64_t)((ks >> 2) * kHalf + (ks & 3) * 32) >> 4;
                  tc_mma_bf16(ts, qd + (uint64_t)(i * kStage >> 4) + off, kd + off, kIdescS, ks > 0 ? 1u : 0u);
                }
                tc_commit(&ctl.s_full[i]);
              }
            }
          }
          if (lead) {
            tc_commit(&ctl.empty[step % kSteps]);
            if (j == ntm - 1) tc_commit(&ctl.q_empty);
          }
          if (j > 0) two_on(sv);
          if (j < ntm) two_on(sk);
        }
      }
      if (!live) ctl.fail = 1;
    } else if (warp == 4 * NQ + 1) {
      // ---- TMA producer (the lanes share a tile's pages) ----
      uint32_t n_q = 0, st = 0, step = 0, armed = 0;  // armed: steps whose barrier expects loads
      uint32_t user[F::kStages];  // the step that the stage's tile is for, and one more
#pragma unroll
      for (int i = 0; i < F::kStages; ++i) user[i] = 0;
      bool live = true;
      const int box = a.paged ? min(a.page_size, kT) : kT;
      auto bytes_of = [&](const Unit<NQ>& x, int t) {
        if (!a.paged) return kStage;
        const int n = min(kT, t < x.n_pt ? x.n_prefix - t * kT : x.s.k_len - (t - x.n_pt) * kT);
        return (n + box - 1) / box * box * 256;
      };
      // one tile of the list, K or V, into the next stage, for the step under way
      auto load = [&](const Unit<NQ>& x, int t, bool v) {
        bool ok = true;
        uint32_t before = 0;
#pragma unroll
        for (int i = 0; i < F::kStages; ++i)
          if (st == i) {
            before = user[i];
            user[i] = step + 1;
          }
        if (lane == 0 && before > 0)
          ok = mbar_wait_beat(&ctl.empty[(before - 1) % kSteps], ((before - 1) / kSteps) & 1u, a.err, &ctl.beat);
        __syncwarp();
        if (!__shfl_sync(0xffffffffu, ok ? 1 : 0, 0)) return false;
        uint64_t* full = &ctl.full[step % kSteps];
        uint8_t* dst = kv + st * kStage;
        st = st + 1 < F::kStages ? st + 1 : 0;
        const bool pre = t < x.n_pt;
        const int key = pre ? t * kT : (t - x.n_pt) * kT;
        const CUtensorMap* map = pre ? (v ? &maps.vp : &maps.kp) : (v ? &maps.v : &maps.k);
        if (lane * box * 256 < bytes_of(x, t)) {
          int row;
          if (a.paged)
            row = (int)attn_slot(a, pre ? a.prefix_table : x.s.pages, key + lane * box);
          else
            row = pre ? key : (int)(x.s.k0 + key);
          tma_load_2d(dst + lane * box * 128, map, x.g * kHeadDim, row, full);
          tma_load_2d(dst + kHalf + lane * box * 128, map, x.g * kHeadDim + 64, row, full);
        }
        __syncwarp();
        return true;
      };
      for (uint32_t n = 0; live; ++n) {
        live = warp_wait(&ctl.u_full[n % kBoard], (n / kBoard) & 1u, a.err, &ctl.beat);
        if (!live) break;
        const Unit<NQ> x = ctl.board[n % kBoard];
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.u_empty[n % kBoard]);
        if (x.g < 0) break;
        if (x.ntm == 0) continue;
        // (a step's barrier is free: the stages handed over so far come from later steps than its last)
        armed = step + 1;
        if (lane == 0) mbar_arrive_expect_tx(&ctl.full[step % kSteps], bytes_of(x, x.t_lo));
        __syncwarp();
        live = load(x, x.t_lo, false);
        if (!live) break;
        ++step;
        bool ok = true;
        if (lane == 0) {
          ok = mbar_wait_beat(&ctl.q_empty, (n_q & 1u) ^ 1u, a.err, &ctl.beat);
          if (ok) {
            int tiles = 0;
#pragma unroll
            for (int i = 0; i < NQ; ++i) tiles += x.n_tok[i] > 0;
            mbar_arrive_expect_tx(&ctl.q_full, (uint32_t)(tiles * TT * R * 256));
#pragma unroll
            for (int i = 0; i < NQ; ++i)
              if (x.n_tok[i] > 0) {
                const int tok = x.s.q0 + x.tok0 + i * TT;
                tma_load_3d(qs + i * kStage, &maps.q, 0, x.g * R, tok, &ctl.q_full);
                tma_load_3d(qs + i * kStage + kHalf, &maps.q, 64, x.g * R, tok, &ctl.q_full);
              }
          }
        }
        __syncwarp();
        live = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
        n_q += live;
        for (int j = 0; live && j < x.ntm; ++j, ++step) {
          const bool more = j + 1 < x.ntm;
          armed = step + 1;
          if (lane == 0)
            mbar_arrive_expect_tx(&ctl.full[step % kSteps], bytes_of(x, x.t_lo + j) + (more ? bytes_of(x, x.t_lo + j + 1) : 0));
          __syncwarp();
          live = load(x, x.t_lo + j, true);
          if (live && more) live = load(x, x.t_lo + j + 1, false);
        }
      }
      if (lane == 0) {
        ctl.armed = armed;
        ctl.n_q = n_q;
      }
      if (!live) ctl.fail = 1;
    } else if (warp == 4 * NQ + 2) {
      // ---- units of this CTA onto the board, ahead of those who work on them ----
      Walk w;
      if (!a.paged) {
        w.b0 = w.g0 = w.base = 0;
        walk_chunk<NQ>(a, plan, w);
      }
      uint32_t loads = 0, steps = 0;
      bool live = true;
      for (int k = 0; live; ++k) {
        const int u = unit_index(k), slot = k % kBoard;
        Unit<NQ> x;
        bool more = u < n_units;  // (contiguous keys: at most)
        if (more && a.paged) {
          x = paged_unit<NQ>(a, plan, u);
          if (lane == 0 && !x.s.ok) set_error(a.err, kErrBadDeviceArg);
        } else if (more) {
          more = walk_to<NQ>(a, plan, w, u, x);
        }
        if (!more) x.g = -1;
        x.load0 = loads;
        x.step0 = steps;
        if (more && x.ntm > 0) {
          loads += 2 * x.ntm;
          steps += x.ntm + 1;
        }
        live = warp_wait(&ctl.u_empty[slot], ((k / kBoard) & 1u) ^ 1u, a.err, &ctl.beat);
        if (live && lane == 0) {
          ctl.board[slot] = x;
          mbar_arrive(&ctl.u_full[slot]);
        }
        __syncwarp();
        if (!more) break;
      }
      if (!live) ctl.fail = 1;
    }
  } else {
    // ---- softmax: a thread per row ----
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(F::kSoftRegs));
    const int i = NQ == 2 ? warp >> 2 : 0, r = (warp & 3) * 32 + lane;
    const uint32_t ts = tmem + i * kT + ((uint32_t)(r & ~31) << 16), to = ts + NQ * kT;
    const int tok_in = (r * a.group_inv) >> 16, tok_first = ((r & ~31) * a.group_inv) >> 16;  // / R
    const float sc = a.scale_log2;
    uint32_t n_s = 0, n_o = 0;
    bool failed = false;
    for (uint32_t n = 0;; ++n) {
      if (!warp_wait(&ctl.u_full[n % kBoard], (n / kBoard) & 1u, a.err, &ctl.beat)) failed = true;
      const Unit<NQ>& x = ctl.board[n % kBoard];
      if (failed || x.g < 0) break;
      const int nt = x.nt[i];
      const bool row_live = tok_in < x.n_tok[i], warp_live = tok_first < x.n_tok[i];
      // hidden own keys, of this row and of the warp's first one, which sees the fewest
      int hid = 0, hid_first;
      {
        const int q_len = x.s.q_len, k_len = x.s.k_len, tok = x.tok0 + i * TT;
        if (row_live) hid = k_len - attn_visible(a, q_len, k_len, tok + tok_in);
        hid_first = k_len - attn_visible(a, q_len, k_len, tok + tok_first);
      }
      int pre_left = x.n_pt - x.t_lo;  // tiles of the prefix from the unit's first tile on
      int n_keys = pre_left > 0 ? x.n_prefix - x.t_lo * kT : x.s.k_len + pre_left * kT;  // from the tile on
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < nt; ++j) {
        failed = !warp_wait(&ctl.s_full[i], n_s & 1u, a.err, &ctl.beat);
        ++n_s;
        if (failed) break;
        tc_fence_after();
        if (n_keys < kT) {
          // rows past the end: zero before the product reads them
          const uint32_t sv = (x.load0 + 2 * j + 1) % F::kStages, st = x.step0 + j + 1;
          failed = !warp_wait(&ctl.full[st % kSteps], (st / kSteps) & 1u, a.err, &ctl.beat);
          if (failed) break;
          uint8_t* vs = kv + sv * kStage;
          for (int q = n_keys * 16 + r; q < kT * 16; q += 128)
            *reinterpret_cast<uint4*>(vs + ((q >> 3) & 1) * kHalf + (q >> 4) * 128 + (q & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
          fence_proxy_async_smem();
          __syncwarp();
        }
        if (warp_live) {
          // P is formed against the maximum so far. No maximum is looked for: a tile's sum shows
          // whether one of its terms is too large (and at a row's first keys there is no
          // maximum yet); only then it is found and P formed again from the scores, which
          // are still there
          const int lim = n_keys - (pre_left > 0 ? 0 : hid);  // keys that this row sees
          const bool masked = n_keys - (pre_left > 0 ? 0 : hid_first) < kT;  // the warp's first row sees the fewest
          float t;
          uint32_t w[kT / 2];
#pragma unroll 1
          for (bool raise = __any_sync(0xffffffffu, m == -INFINITY && lim > 0 && row_live), raised = false;;) {
            float v[kT];
            tmem_ld64(ts, v);
            tmem_ld64(ts + 64, v + 64);
            tc_wait_ld();
            if (masked) mask_from<kT>(v, lim);
            if (raise) {
              raised = true;
              const float mn = fmaxf(m, max128(v) * sc);  // sc > 0: the maximum commutes with it
              const float f = m == mn ? 1.f : ex2_approx(m - mn);
              m = mn;
              if (j > 0) {
                l = l == INFINITY ? l : l * f;  // (NaN is kept for a row that sees a NaN score)
                scale_o(to, f);
                raise = false;
                continue;  // the scores are read again rather than kept over the call
              }
            }
            const float mb = m == -INFINITY ? 0.f : m;
            const uint64_t sc2 = pack2(sc, sc), mb2 = pack2(-mb, -mb);
            uint64_t s2[2] = {0, 0};
#pragma unroll
            for (int e = 0; e < kT / 2; ++e) {
              float p0, p1;
              unpack2(fma2(pack2(v[2 * e], v[2 * e + 1]), sc2, mb2), p0, p1);
              p0 = ex2_approx(p0);
              p1 = ex2_approx(p1);
              s2[e & 1] = add2(s2[e & 1], pack2(p0, p1));
              w[e] = pack_bf16(p0, p1);
            }
            float s0, s1;
            unpack2(add2(s2[0], s2[1]), s0, s1);
            t = s0 + s1;
            // Against the tile's own maximum the sum is about kT at most. (Where scores pass 2^28 the
            // rounding of m alone may make more of it, up to infinity: not raised again. Such
            // a sum cancels with O's, or the row is not finite and computed again.)
            raise = !raised && __any_sync(0xffffffffu, row_live && t > kMostSum);
            if (!raise) break;
          }
          l += t;
          tmem_st32(ts, w);
          tmem_st32(ts + 32, w + 32);
          tc_wait_st();
        }
        n_keys = --pre_left == 0 ? x.s.k_len : n_keys - kT;  // of the next tile
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl.p_full[i]);
      }
      if (failed) break;
      // ---- epilogue: O / l to memory ----
      if (nt > 0) {
        failed = !warp_wait(&ctl.o_full[i], n_o & 1u, a.err, &ctl.beat);
        ++n_o;
        if (failed) break;
        tc_fence_after();
      }
      if (warp_live) finish_rows<NQ>(a, x, i, tok_in, hid, m, l, to, &ctl.beat);
      __syncwarp();
      if (lane == 0) mbar_arrive(&ctl.u_empty[n % kBoard]);
    }
    if (failed) ctl.fail = 1;
  }
  tc_fence_before();
  __syncthreads();
  if (ctl.fail) {
    drain<NQ>(ctl, a.err);
    __syncthreads();
  }
  if (warp == 0) tmem_dealloc(tmem, F::kCols);
}

int map_of(CUtensorMap* m, const void* base, uint64_t rows, int H, long long stride, uint32_t box_rows) {
  return make_tmap_bf16_2d(m, base, rows, (uint64_t)H * kHeadDim, (uint64_t)stride * 2, box_rows);
}

template <int NQ>
cudaError_t launch(const AttnArgs& a, const AttnPlan& plan, const Maps& maps, int sms, cudaStream_t s) {
  using F = Form<NQ>;
  static std::atomic<bool> configured[64];  // per device, zero-initialised
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev >= 0 && dev < 64 && !configured[dev]) {
    cudaError_t e = cudaFuncSetAttribute(attn_tc<NQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)F::kSmem);
    cudaFuncAttributes at;
    if (e == cudaSuccess) e = cudaFuncGetAttributes(&at, attn_tc<NQ>);
    if (e != cudaSuccess) return e;
    // a register split that the launch does not cover would wait for ever
    if (at.numRegs * F::kThreads < F::kSoftRegs * F::kSoft + F::kRestRegs * (F::kThreads - F::kSoft))
      return cudaErrorInvalidConfiguration;
    configured[dev] = true;
  }
  const long long most = (long long)sms * F::kCtas;
  const int grid = (int)(plan.n_units < most ? plan.n_units : most);
  attn_tc<NQ><<<grid, F::kThreads, F::kSmem, s>>>((int)plan.n_units, a, plan, maps);
  return cudaGetLastError();
}

}  // namespace

cudaError_t attn_tc_launch(const AttnArgs& a, const AttnPlan& plan, int sms, cudaStream_t s) {
  Maps m;
  const int R = a.H_q / a.H_kv;
  const uint32_t box = a.paged ? (uint32_t)(a.page_size < kT ? a.page_size : kT) : (uint32_t)kT;
  const uint64_t rows = a.paged ? (uint64_t)a.n_pages * a.page_size : (uint64_t)(a.T_k > 0 ? a.T_k : 1);
  if (make_tmap_bf16_heads(&m.q, a.Q, (uint64_t)a.T_q, (uint64_t)a.H_q, (uint64_t)a.q_stride * 2, (uint32_t)R,
                           (uint32_t)(kT / R)) ||
      map_of(&m.k, a.K, rows, a.H_kv, a.k_stride, box) || map_of(&m.v, a.V, rows, a.H_kv, a.v_stride, box))
    return cudaErrorInvalidValue;
  m.kp = m.k;
  m.vp = m.v;
  if (!a.paged && a.prefix_len > 0 &&
      (map_of(&m.kp, a.Kp, (uint64_t)a.prefix_len, a.H_kv, a.kp_stride, box) ||
       map_of(&m.vp, a.Vp, (uint64_t)a.prefix_len, a.H_kv, a.vp_stride, box)))
    return cudaErrorInvalidValue;
  return plan.nq == 2 ? launch<2>(a, plan, m, sms, s) : launch<1>(a, plan, m, sms, s);
}

}  // namespace provip
