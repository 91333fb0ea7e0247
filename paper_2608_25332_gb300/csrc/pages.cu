// Paged key/value cache behind the pruning: block tables and slot maps from the requests'
// lengths, and rows into the pages.
#include <cooperative_groups.h>

#include "common.cuh"
#include "kernels.h"

namespace provip {
namespace {

// ---------------------------------------------------------------------------
// block tables and slot maps
//
// One cluster. Its CTAs all scan the requests (a block of them at a time, in order) and share
// out the writes, so one launch does both passes: ended requests' pages onto the free stack,
// then, past a cluster barrier, pages off it in request order (those of a request that no
// longer fits are not taken), the tables' new entries and a slot for every new token. Lengths
// and the free count may be updated in place, so they are written past a last barrier. Bound
// by latency: two block scans and the barriers, with the requests read once where one block
// holds them all. A decode step (256 requests, a token each) runs on one CTA of 256 threads.
// ---------------------------------------------------------------------------
constexpr int kThr = 1024;  // at most

struct Scan {
  int pages[32];
  long long rows[32];
};

// exclusive sums over the block of (pages, rows), and the block's totals
__device__ __forceinline__ void block_scan(Scan& sc, int& pages, long long& rows, int& pages_all, long long& rows_all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int p = pages;
  long long r = rows;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int pu = __shfl_up_sync(0xffffffffu, p, o);
    const long long ru = __shfl_up_sync(0xffffffffu, r, o);
    if (lane >= o) {
      p += pu;
      r += ru;
    }
  }
  __syncthreads();  // the arrays' last use
  if (lane == 31) {
    sc.pages[warp] = p;
    sc.rows[warp] = r;
  }
  __syncthreads();
  const bool has = lane < (int)(blockDim.x >> 5);
  int wp = has ? sc.pages[lane] : 0;
  long long wr = has ? sc.rows[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int pu = __shfl_up_sync(0xffffffffu, wp, o);
    const long long ru = __shfl_up_sync(0xffffffffu, wr, o);
    if (lane >= o) {
      wp += pu;
      wr += ru;
    }
  }
  pages_all = __shfl_sync(0xffffffffu, wp, 31);
  rows_all = __shfl_sync(0xffffffffu, wr, 31);
  const int p0 = __shfl_sync(0xffffffffu, wp, max(warp - 1, 0));
  const long long r0 = __shfl_sync(0xffffffffu, wr, max(warp - 1, 0));
  pages = p - pages + (warp ? p0 : 0);
  rows = r - rows + (warp ? r0 : 0);
}

__device__ __forceinline__ long long pages_of(long long n, int shift) { return (n + (1ll << shift) - 1) >> shift; }

// last i of first[0 .. n) with first[i] <= x (first[0] <= x)
template <typename V>
__device__ __forceinline__ int last_at_most(const V* first, int n, V x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

struct Request {
  int kv, add, held, need;  // tokens held, new ones, pages held, pages wanted
  bool end, bad;
};
__device__ __forceinline__ Request request(const PageTablesArgs& a, int b) {
  Request q = {0, 0, 0, 0, false, false};
  if (b >= a.B) return q;
  q.kv = a.kv_len[b];
  const int n = a.new_len[b];
  q.end = n < 0;
  q.add = max(n, 0);
  const long long held = pages_of(max(q.kv, 0), a.page_shift);
  const long long all = pages_of((long long)max(q.kv, 0) + q.add, a.page_shift);
  q.bad = q.kv < 0 || held > a.max_pages || (!q.end && all > a.max_pages) || (long long)q.kv + q.add > 0x7fffffffll;
  if (!q.bad) {
    q.held = (int)held;
    q.need = q.end ? 0 : (int)(all - held);
  }
  return q;
}

// a barrier over the cluster; one CTA needs only its own
__device__ __forceinline__ void all_sync(int n_cta) {
  if (n_cta > 1)
    cooperative_groups::this_cluster().sync();
  else
    __syncthreads();
}

__global__ void __launch_bounds__(kThr) page_tables_kernel(const PageTablesArgs a) {
  const int n_cta = (int)gridDim.x, rank = (int)blockIdx.x, thr = (int)blockDim.x;  // the grid is one cluster
  const int gtid = rank * thr + (int)threadIdx.x, gthr = n_cta * thr;
  const bool single = a.B <= thr;
  __shared__ Scan sc;
  __shared__ int s_pages[kThr], s_held[kThr], s_kv[kThr], s_take[kThr];
  __shared__ long long s_rows[kThr];
  __shared__ int s_used;

  // ended requests' pages onto the stack
  int count = *a.free_count;
  Request q = request(a, (int)threadIdx.x);
  if (threadIdx.x == 0) s_used = 0;
  if (count < 0 || count > a.n_free_max) {
    if (gtid == 0) set_error(a.err, kErrBadDeviceArg);
    count = min(max(count, 0), a.n_free_max);
  }
  long long back = 0;
  for (int b0 = 0; b0 < a.B; b0 += thr) {
    if (b0 > 0) q = request(a, b0 + (int)threadIdx.x);
    const int mine = q.end ? q.held : 0;
    if (!__syncthreads_or(mine)) continue;
    int at = mine, all;
    long long r = 0, r_all;
    block_scan(sc, at, r, all, r_all);
    s_pages[threadIdx.x] = at;
    __syncthreads();
    for (int i = gtid; i < all; i += gthr) {
      const int j = last_at_most(s_pages, thr, i);
      const long long to = count + back + i;
      if (to < a.n_free_max)
        a.free_pages[to] = a.block_table[(size_t)(b0 + j) * a.max_pages + (i - s_pages[j])];
      else
        set_error(a.err, kErrBadDeviceArg);
    }
    back += all;
  }
  const int total = (int)min((long long)a.n_free_max, count + back);
  all_sync(n_cta);  // the stack is whole

  // pages off its top
  long long pages_done = 0, rows_done = 0;  // of the requests before the chunk
  int used = 0;                             // pages of granted requests
  bool ok = false;
  long long row = 0;
  // request b0 + threadIdx.x: its first new row, whether it is granted; its first page
  auto place = [&](int b0) {
    if (!single) q = request(a, b0 + (int)threadIdx.x);
    int p = q.need, p_all;
    long long r_all;
    row = q.add;
    block_scan(sc, p, row, p_all, r_all);
    row += rows_done;
    const long long first = pages_done + p;
    ok = !q.end && !q.bad && row + q.add <= a.T_max && (q.need == 0 || first + q.need <= total);
    pages_done += p_all;
    rows_done += r_all;
    return first;
  };
  for (int b0 = 0; b0 < a.B; b0 += thr) {
    const long long p0 = pages_done, r0 = rows_done;
    const long long first = place(b0);
    if (b0 + (int)threadIdx.x < a.B && rank == 0 && (q.bad || row + q.add > a.T_max)) set_error(a.err, kErrBadDeviceArg);
    s_pages[threadIdx.x] = (int)min(first, 0x7fffffffll);
    s_rows[threadIdx.x] = row;
    s_held[threadIdx.x] = q.held;
    s_kv[threadIdx.x] = q.kv;
    s_take[threadIdx.x] = ok ? q.need : -1;
    // requests with pages are granted in order, so the last one's end is what was used
    used = max(used, ok && q.need ? (int)(first + q.need) : 0);
    __syncthreads();
    // the tables' new entries
    for (long long i = p0 + gtid; i < min(pages_done, (long long)total); i += gthr) {
      const int j = last_at_most(s_pages, thr, (int)i), k = (int)i - s_pages[j];
      if (k < s_take[j]) a.block_table[(size_t)(b0 + j) * a.max_pages + s_held[j] + k] = a.free_pages[total - 1 - i];
    }
    // a slot for every new token
    for (long long t = r0 + gtid; t < min(rows_done, (long long)a.T_max); t += gthr) {
      const int j = last_at_most(s_rows, thr, t);
      int slot = -1;
      if (s_take[j] >= 0) {
        const int pos = s_kv[j] + (int)(t - s_rows[j]), pi = pos >> a.page_shift;
        const int page = pi < s_held[j] ? a.block_table[(size_t)(b0 + j) * a.max_pages + pi]
                                        : a.free_pages[total - 1 - (s_pages[j] + pi - s_held[j])];
        slot = (page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
      }
      a.slot_map_out[t] = slot;
    }
    if (!single) __syncthreads();  // the arrays may change
  }
  for (long long t = rows_done + gtid; t < a.T_max; t += gthr) a.slot_map_out[t] = -1;
  if (rank == 0) {
    used = __reduce_max_sync(0xffffffffu, used);
    if ((threadIdx.x & 31) == 0 && used) atomicMax(&s_used, used);
  }
  const long long rows_all = rows_done;

  // lengths and the free count, which calls may keep in one place: past everybody's reads
  all_sync(n_cta);
  if (rank != 0) return;
  pages_done = rows_done = 0;
  for (int b0 = 0; b0 < a.B; b0 += thr) {
    const int b = b0 + (int)threadIdx.x;
    if (!single) place(b0);  // this chunk's requests again
    if (b < a.B) {
      a.kv_len_out[b] = q.end && !q.bad ? 0 : ok ? q.kv + q.add : q.kv;
      a.row_start_out[b] = (int)min(row, 0x7fffffffll);
    }
  }
  if (threadIdx.x == 0) {
    a.row_start_out[a.B] = (int)min(rows_all, 0x7fffffffll);
    *a.free_count_out = total - s_used;
  }
}

// ---------------------------------------------------------------------------
// rows into pages: 16-byte pieces, four loads of a thread in flight. A block takes as
// many whole rows as make 1024 pieces (one row at least). Bound by HBM (each row is read
// and written once).
// ---------------------------------------------------------------------------
constexpr int kAppThr = 256, kAppUnroll = 4;

__global__ void __launch_bounds__(kAppThr) kv_append_kernel(const KvAppendArgs a, int rows_per_block) {
  const int pieces = (int)(a.row_bytes >> 4);
  const long long row0 = (long long)blockIdx.x * rows_per_block;
  const int n = (int)min((long long)rows_per_block, a.T - row0) * pieces;
  const char* src = blockIdx.y ? a.V : a.K;
  char* dst = blockIdx.y ? a.v_pages : a.k_pages;
  const long long stride = blockIdx.y ? a.v_stride : a.k_stride;
  for (int u0 = threadIdx.x; u0 < n; u0 += kAppThr * kAppUnroll) {
    uint4 v[kAppUnroll];
    char* to[kAppUnroll];
#pragma unroll
    for (int i = 0; i < kAppUnroll; ++i) {
      const int u = u0 + i * kAppThr;
      to[i] = nullptr;
      if (u < n) {
        const int r = u / pieces, piece = u - r * pieces;
        const int slot = __ldg(a.slot_map + row0 + r);
        if (slot >= 0 && slot < a.n_slots) {
          v[i] = __ldg(reinterpret_cast<const uint4*>(src + (row0 + r) * stride) + piece);
          to[i] = dst + slot * a.row_bytes + (long long)piece * 16;
        } else if (slot >= 0) {
          set_error(a.err, kErrBadDeviceArg);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kAppUnroll; ++i)
      if (to[i]) *reinterpret_cast<uint4*>(to[i]) = v[i];
  }
}

}  // namespace

cudaError_t page_tables_launch(const PageTablesArgs& a, cudaStream_t s) {
  // few requests and slots: one small CTA, whose barriers are quick; else eight large ones
  // (the portable cluster's most) from four slots a thread on
  const int thr = a.B <= 256 && a.T_max <= 1024 ? 256 : kThr;
  if (a.T_max <= 4 * thr) {
    page_tables_kernel<<<1, thr, 0, s>>>(a);
    return cudaGetLastError();
  }
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 8;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3(8);
  cfg.blockDim = dim3(kThr);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, page_tables_kernel, a);
}

cudaError_t kv_append_launch(const KvAppendArgs& a, cudaStream_t s) {
  const long long pieces = a.row_bytes >> 4;
  const int rpb = (int)(pieces >= 1024 ? 1 : 1024 / pieces);
  kv_append_kernel<<<dim3((unsigned)((a.T + rpb - 1) / rpb), 2), kAppThr, 0, s>>>(a, rpb);
  return cudaGetLastError();
}

}  // namespace provip
