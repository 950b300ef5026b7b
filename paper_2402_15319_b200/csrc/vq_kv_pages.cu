// The cache's books and the pages they move: vq_kv_reserve, vq_kv_fork, vq_kv_free, vq_kv_compact, vq_kv_copy_pages.
//
// Books are whole numbers on the device.  What depends on order - which free page a sequence gets - is decided by one CTA
// that counts free pages with ballots (the reference counts are read twice, coalesced; 65,536 of them are 256 KB) and
// ranks them by a scan, so equal books give equal books.  What does not - page data, table rows, counts of shared
// pages - is left to a second kernel on the whole GPU, which finds the list of pages in the workspace.
#include "vq_device.cuh"
#include "vq_kv.cuh"

namespace vq {
namespace {

using namespace dev;

constexpr int kBookThreads = 1024;
constexpr int kMaxForks = 1024;
constexpr int kCopyThreads = 256;

// Workspace: 64 words of header, then the lists (32-bit words each).
struct Lists {
  int* count;      // [0] pages to copy (or forks), [1] pages in use
  int* src;        // [n_pages] pages to move
  int* dst;        // [n_pages] where to / free pages in order
  int* remap;      // [n_pages] new number of a moved page
  int* first;      // [n_seqs + 1] pages in front of a sequence's share
  int* fork;       // [kMaxForks][6] parent, child, full pages, tokens behind them, their page, its copy
};
__host__ __device__ inline Lists lists_of(void* ws, int n_pages, int n_seqs) {
  Lists l;
  l.count = static_cast<int*>(ws);
  l.fork = l.count + 64;
  l.src = l.fork + 6 * kMaxForks;
  l.dst = l.src + n_pages;
  l.remap = l.dst + n_pages;
  l.first = l.remap + n_pages;
  (void)n_seqs;
  return l;
}

__device__ __forceinline__ int clamp_len(const KvBooks& b, int n) { return n < 0 ? 0 : n > b.max_len ? b.max_len : n; }

// Exclusive sum over the CTA's threads, and the total.
template <class T>
__device__ __forceinline__ T block_scan(T v, T* total, T* s_scan) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  T incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T up = __shfl_up_sync(~0u, incl, o);
    if (lane >= o) incl += up;
  }
  __syncthreads();
  if (lane == 31) s_scan[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    T w = s_scan[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T up = __shfl_up_sync(~0u, w, o);
      if (lane >= o) w += up;
    }
    s_scan[lane] = w;
  }
  __syncthreads();
  *total = s_scan[31];
  return incl - v + (warp ? s_scan[warp - 1] : 0);
}

// Visits the pages in order: each warp a run of them, 32 a step; f(page, is_free, rank among the pages for which `want`
// holds) after the warps' counts have been scanned.  Returns how many there are.  `want(page, is_free)`.
template <class Want, class Each>
__device__ __forceinline__ int rank_pages(const int* refs, int n_pages, int* s_scan, Want want, Each each) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int run = ((n_pages + 31) / 32 + 31) / 32 * 32;   // per warp (32 warps), whole steps
  const int lo = min(n_pages, warp * run), hi = min(n_pages, lo + run);
  int mine = 0;
#pragma unroll 8
  for (int p = lo + lane; p < lo + run; p += 32) {
    const bool free_page = p < hi && __ldcg(refs + p) == 0;
    mine += p < hi && want(p, free_page);
  }
  int total;
  const int before_thread = block_scan(mine, &total, s_scan);
  int before = __shfl_sync(~0u, before_thread, 0);   // pages of the warps in front
#pragma unroll 8
  for (int p = lo + lane; p < lo + run; p += 32) {
    const bool free_page = p < hi && __ldcg(refs + p) == 0;
    const bool is = p < hi && want(p, free_page);
    const unsigned all = __ballot_sync(~0u, is);
    if (is) each(p, before + __popc(all & ((1u << lane) - 1)));
    before += __popc(all);
  }
  return total;
}

// ---- vq_kv_reserve ------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(kBookThreads) reserve_kernel(KvGeometry g, KvBooks b, int* refs, const int* grow, int* status, void* ws) {
  __shared__ int s_scan[32];
  __shared__ long long s_need[32];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x;
  const Lists l = lists_of(ws, g.n_pages, b.n_seqs);
  const int per = (b.n_seqs + kBookThreads - 1) / kBookThreads, s0 = tid * per;
  auto shares = [&](int s, int* n, long long* more) {   // pages that sequence s needs
    *n = clamp_len(b, __ldcg(b.len + s));
    *more = grow ? __ldcg(grow + s) : 1;
    if (*more < 0) *more = 0;
    const long long to = *n + *more;
    if (to > b.max_len) return -1;
    return static_cast<int>(((to + g.page_tokens - 1) >> g.page_shift) - ((*n + g.page_tokens - 1) >> g.page_shift));
  };
  long long need = 0;
  int too_long = 0, n;
  long long more;
  for (int s = s0; s < min(b.n_seqs, s0 + per); ++s) {
    const int p = shares(s, &n, &more);
    if (p < 0) ++too_long;
    else need += p;
  }
  long long total;
  int any_long;
  long long at = block_scan(need, &total, s_need);
  block_scan(too_long, &any_long, s_scan);
  if (any_long) {
    if (tid == 0) {
      status[0] = 0;
      status[1] = any_long;
    }
    return;
  }
  if (total > 0) {
    const int have = rank_pages(refs, g.n_pages, s_scan, [](int, bool is_free) { return is_free; },
                                [&](int page, int rank) {
                                  if (rank < total) l.dst[rank] = page;
                                });
    if (have < total) {
      if (tid == 0) {
        status[0] = total - have < 0x7fffffff ? static_cast<int>(total - have) : 0x7fffffff;
        status[1] = 0;
      }
      return;
    }
    for (int s = s0; s < min(b.n_seqs, s0 + per); ++s) {   // (there are no more than the pool has: 32 bits)
      l.first[s] = static_cast<int>(at);
      at += shares(s, &n, &more);
    }
    __syncthreads();
    for (int r = tid; r < total; r += kBookThreads) {
      int lo = 0, hi = b.n_seqs;   // last sequence whose share begins at or in front of r
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (l.first[mid] <= r) lo = mid;
        else hi = mid;
      }
      const int len = clamp_len(b, __ldcg(b.len + lo));
      const int page = l.dst[r];
      b.table[static_cast<long long>(lo) * b.table_stride + ((len + g.page_tokens - 1) >> g.page_shift) + r - l.first[lo]] = page;
      refs[page] = 1;
    }
  }
  __syncthreads();
  for (int s = s0; s < min(b.n_seqs, s0 + per); ++s) {
    shares(s, &n, &more);
    b.len[s] = static_cast<int>(n + more);
  }
  if (tid == 0) status[0] = status[1] = 0;
}

// ---- vq_kv_fork: the list of forks, pages for their last tokens ---------------------------------------------------------
__global__ void __launch_bounds__(kBookThreads) fork_kernel(KvGeometry g, KvBooks b, int* refs, const int* pairs, int n_pairs, int* status,
                                                           void* ws) {
  __shared__ int s_scan[32];
  __shared__ int s_child[kMaxForks];
  pdl_launch_dependents();
  pdl_wait();
  const int i = threadIdx.x;
  const Lists l = lists_of(ws, g.n_pages, b.n_seqs);
  int parent = -1, child = -1;
  if (i < n_pairs) {
    parent = __ldcg(pairs + 2 * i);
    child = __ldcg(pairs + 2 * i + 1);
  }
  s_child[i] = child;
  __syncthreads();
  bool ok = i < n_pairs && static_cast<unsigned>(parent) < static_cast<unsigned>(b.n_seqs) &&
            static_cast<unsigned>(child) < static_cast<unsigned>(b.n_seqs) && __ldcg(b.len + child) <= 0;
  for (int j = 0; j < n_pairs; ++j)
    if (j < i && s_child[j] == child) ok = false;
  const int len = ok ? clamp_len(b, __ldcg(b.len + parent)) : 0;
  const int full = len >> g.page_shift, rest = len & (g.page_tokens - 1);
  int kept, total;
  const int at = block_scan(static_cast<int>(ok), &kept, s_scan);
  const int rank = block_scan(static_cast<int>(rest > 0), &total, s_scan);
  if (total > 0) {
    const int have = rank_pages(refs, g.n_pages, s_scan, [](int, bool is_free) { return is_free; },
                                [&](int page, int r) {
                                  if (r < total) l.dst[r] = page;
                                });
    if (have < total) {
      if (i == 0) {
        status[0] = total - have;
        status[1] = n_pairs - kept;
        l.count[0] = 0;
      }
      return;
    }
  }
  __syncthreads();
  if (ok) {
    int* f = l.fork + 6 * at;
    f[0] = parent;
    f[1] = child;
    f[2] = full;
    f[3] = rest;
    f[4] = rest ? __ldcg(b.table + static_cast<long long>(parent) * b.table_stride + full) : -1;
    f[5] = rest ? l.dst[rank] : -1;
    if (rest) refs[l.dst[rank]] = 1;
    b.len[child] = len;   // (every parent's length has been read)
  }
  if (i == 0) {
    status[0] = 0;
    status[1] = n_pairs - kept;
    l.count[0] = kept;
  }
}

// ---- vq_kv_free ---------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) free_kernel(KvGeometry g, KvBooks b, int* refs, const int* slots, int n_slots) {
  pdl_launch_dependents();
  pdl_wait();
  const int i = blockIdx.x;   // a CTA per entry
  const int seq = __ldcg(slots + i);
  if (static_cast<unsigned>(seq) >= static_cast<unsigned>(b.n_seqs)) return;
  __shared__ int s_len;
  if (threadIdx.x == 0) s_len = clamp_len(b, atomicExch(b.len + seq, 0));   // of repeated entries one finds the length
  __syncthreads();
  const int pages = (s_len + g.page_tokens - 1) >> g.page_shift;
  const int* row = b.table + static_cast<long long>(seq) * b.table_stride;
  for (int j = threadIdx.x; j < pages; j += blockDim.x) {
    const int page = __ldcg(row + j);
    if (static_cast<unsigned>(page) < static_cast<unsigned>(g.n_pages)) atomicSub(refs + page, 1);
  }
}

// ---- vq_kv_compact: which page goes where ---------------------------------------------------------------------------
__global__ void __launch_bounds__(kBookThreads) compact_kernel(KvGeometry g, KvBooks b, int* refs, int* status, void* ws) {
  __shared__ int s_scan[32];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x;
  const Lists l = lists_of(ws, g.n_pages, b.n_seqs);
  int mine = 0;
#pragma unroll 8
  for (int p = tid; p < g.n_pages; p += kBookThreads) mine += __ldcg(refs + p) != 0;
  int used;
  block_scan(mine, &used, s_scan);
  const int moved = rank_pages(refs, g.n_pages, s_scan, [&](int p, bool is_free) { return !is_free && p >= used; },
                               [&](int p, int r) { l.src[r] = p; });
  rank_pages(refs, g.n_pages, s_scan, [&](int p, bool is_free) { return is_free && p < used; }, [&](int p, int r) { l.dst[r] = p; });
  __syncthreads();
  for (int r = tid; r < moved; r += kBookThreads) {
    const int from = l.src[r], to = l.dst[r];
    l.remap[from] = to;
    refs[to] = refs[from];
    refs[from] = 0;
  }
  if (tid == 0) {
    l.count[0] = moved;
    l.count[1] = used;
    status[0] = used;
    status[1] = moved;
  }
}

// ---- page data, table rows --------------------------------------------------------------------------------------------
enum CopyKind { kPairs, kMoves, kForks };

// A warp copies up to 4 KB at a time, eight 16-byte pieces of each lane in flight.
__device__ __forceinline__ void copy_run(const uint8_t* src, uint8_t* dst, long long bytes, int lane) {
  const int n = static_cast<int>(bytes / 16);
  uint4 v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i * 32 + lane < n) v[i] = __ldcg(reinterpret_cast<const uint4*>(src) + i * 32 + lane);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i * 32 + lane < n) reinterpret_cast<uint4*>(dst)[i * 32 + lane] = v[i];
}

template <CopyKind KIND>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(KvGeometry g, const __grid_constant__ KvPools pools, KvBooks b, int* refs,
                                                           const int* pairs, int n_pairs, void* ws) {
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const Lists l = lists_of(ws, g.n_pages, b.n_seqs);
  const int count = KIND == kPairs ? n_pairs : __ldcg(l.count);
  const long long warps = static_cast<long long>(gridDim.x) * (kCopyThreads / 32);
  const long long warp0 = static_cast<long long>(blockIdx.x) * (kCopyThreads / 32) + (threadIdx.x >> 5);

  // page data: (entry, layer, keys | values, run of 4 KB)
  const long long page_bytes = static_cast<long long>(g.heads) * g.page_tokens * g.row_bytes;
  const int runs = static_cast<int>((page_bytes + 4095) / 4096);
  const long long scale_words = static_cast<long long>(g.heads) * g.page_tokens;
  const long long items = static_cast<long long>(count) * pools.n_layers * 2 * runs;
  for (long long it = warp0; it < items; it += warps) {
    const int run = static_cast<int>(it % runs);
    const long long rest_it = it / runs;
    const int kv = static_cast<int>(rest_it & 1), layer = static_cast<int>((rest_it >> 1) % pools.n_layers);
    const int e = static_cast<int>((rest_it >> 1) / pools.n_layers);
    int src, dst, tokens = g.page_tokens;
    if (KIND == kPairs) {
      src = __ldcg(pairs + 2 * e);
      dst = __ldcg(pairs + 2 * e + 1);
    } else if (KIND == kMoves) {
      src = __ldcg(l.src + e);
      dst = __ldcg(l.dst + e);
    } else {
      tokens = __ldcg(l.fork + 6 * e + 3);
      src = __ldcg(l.fork + 6 * e + 4);
      dst = __ldcg(l.fork + 6 * e + 5);
    }
    if (static_cast<unsigned>(src) >= static_cast<unsigned>(g.n_pages) || static_cast<unsigned>(dst) >= static_cast<unsigned>(g.n_pages)) continue;
    const KvPool& p = pools.p[layer];
    uint8_t* base = kv ? p.v : p.k;
    const uint8_t* from = base + src * page_bytes;
    uint8_t* to = base + dst * page_bytes;
    if (tokens == g.page_tokens) {
      const long long off = static_cast<long long>(run) * 4096;
      copy_run(from + off, to + off, page_bytes - off < 4096 ? page_bytes - off : 4096, lane);
    } else {   // the first `tokens` of every head
      const int per_head = tokens * g.row_bytes / 16, head_units = g.page_tokens * g.row_bytes / 16;
      const int units = g.heads * per_head;
      for (int u = run * 256 + lane; u < min(units, run * 256 + 256); u += 32) {
        const int head = u / per_head, at = head * head_units + u - head * per_head;
        reinterpret_cast<uint4*>(to)[at] = __ldcg(reinterpret_cast<const uint4*>(from) + at);
      }
    }
    if (g.int8 && run == 0) {
      const float* sf = (kv ? p.vs : p.ks) + src * scale_words;
      float* st = (kv ? p.vs : p.ks) + dst * scale_words;
      for (int i = lane; i < scale_words; i += 32)
        if ((i & (g.page_tokens - 1)) < tokens) st[i] = __ldcg(sf + i);
    }
  }

  // the books that follow: 1024 table entries to a CTA's step
  if (KIND == kPairs) return;
  const int pieces = (b.table_stride + 1023) / 1024;
  const long long rows = KIND == kForks ? count : b.n_seqs;
  for (long long it = blockIdx.x; it < rows * pieces; it += gridDim.x) {
    const int e = static_cast<int>(it / pieces), j0 = static_cast<int>(it % pieces) * 1024;
    if (KIND == kForks) {
      const int* f = l.fork + 6 * e;
      const int full = __ldcg(f + 2), has_rest = __ldcg(f + 3) > 0;
      const int* above = b.table + static_cast<long long>(__ldcg(f)) * b.table_stride;
      int* row = b.table + static_cast<long long>(__ldcg(f + 1)) * b.table_stride;
      for (int j = j0 + threadIdx.x; j < min(j0 + 1024, full); j += kCopyThreads) {
        const int page = __ldcg(above + j);
        row[j] = page;
        if (static_cast<unsigned>(page) < static_cast<unsigned>(g.n_pages)) atomicAdd(refs + page, 1);
      }
      if (has_rest && full >= j0 && full < j0 + 1024 && threadIdx.x == 0) row[full] = __ldcg(f + 5);
    } else {
      const int used = __ldcg(l.count + 1);
      const int pages = (clamp_len(b, __ldcg(b.len + e)) + g.page_tokens - 1) >> g.page_shift;
      int* row = b.table + static_cast<long long>(e) * b.table_stride;
      for (int j = j0 + threadIdx.x; j < min(j0 + 1024, pages); j += kCopyThreads) {
        const int page = __ldcg(row + j);
        if (page >= used && page < g.n_pages) row[j] = __ldcg(l.remap + page);
      }
    }
  }
}

template <CopyKind KIND>
vq_status launch_copy(const KvGeometry& g, const KvPools& pools, const KvBooks& b, int* refs, const int* pairs, int n_pairs, void* ws,
                      cudaStream_t s) {
  int sms = 0;
  const vq_status st = device_sms(&sms);
  if (st != VQ_OK) return st;
  return launch_dependent(copy_kernel<KIND>, dim3(static_cast<unsigned>(sms * 8)), dim3(kCopyThreads), 0, s, g, pools, b, refs, pairs, n_pairs, ws);
}

}  // namespace

size_t kv_pages_workspace_bytes(const KvGeometry& g, int n_seqs) {
  return sizeof(int) * (64 + 6 * static_cast<size_t>(kMaxForks) + 3 * static_cast<size_t>(g.n_pages) + n_seqs + 1);
}

vq_status launch_kv_reserve(const KvGeometry& g, const KvBooks& books, int* refs, const int* grow, int* status, void* ws, cudaStream_t s) {
  return launch_dependent(reserve_kernel, dim3(1), dim3(kBookThreads), 0, s, g, books, refs, grow, status, ws);
}

vq_status launch_kv_fork(const KvGeometry& g, const KvPools& pools, const KvBooks& books, int* refs, const int* pairs, int n_pairs,
                         int* status, void* ws, cudaStream_t s) {
  const vq_status st = launch_dependent(fork_kernel, dim3(1), dim3(kBookThreads), 0, s, g, books, refs, pairs, n_pairs, status, ws);
  if (st != VQ_OK) return st;
  return launch_copy<kForks>(g, pools, books, refs, nullptr, 0, ws, s);
}

vq_status launch_kv_free(const KvGeometry& g, const KvBooks& books, int* refs, const int* slots, int n_slots, cudaStream_t s) {
  return launch_dependent(free_kernel, dim3(static_cast<unsigned>(n_slots)), dim3(256), 0, s, g, books, refs, slots, n_slots);
}

vq_status launch_kv_compact(const KvGeometry& g, const KvPools& pools, const KvBooks& books, int* refs, int* status, void* ws,
                            cudaStream_t s) {
  const vq_status st = launch_dependent(compact_kernel, dim3(1), dim3(kBookThreads), 0, s, g, books, refs, status, ws);
  if (st != VQ_OK) return st;
  return launch_copy<kMoves>(g, pools, books, refs, nullptr, 0, ws, s);
}

vq_status launch_kv_copy_pages(const KvGeometry& g, const KvPools& pools, const int* pairs, int n_pairs, cudaStream_t s) {
  KvBooks none = {};
  return launch_copy<kPairs>(g, pools, none, nullptr, pairs, n_pairs, nullptr, s);
}

}  // namespace vq
