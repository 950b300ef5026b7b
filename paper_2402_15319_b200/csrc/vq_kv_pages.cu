// The cache's books and the pages they move: vq_kv_reserve, vq_kv_fork, vq_kv_free, vq_kv_compact, vq_kv_copy_pages.
//
// Books are whole numbers on the device.  What depends on order - which free page a sequence gets - is decided by one CTA.
// It gets the reference counts as bits: a cluster of eight CTAs reads them (one SM alone drew 16 bytes a clock from L2:
// 65,536 pages took 8.5 us), ballots make words of them that go to the first CTA's shared memory, and scans of the words'
// counts rank the pages, so equal books give equal books.  What does not depend on order - page data, table rows, counts
// of shared pages - is left to a second kernel on the whole GPU, which finds the list of pages in the workspace.
// Counting 65,536 pages and entering 1750 for 256 sequences: 8.3 us with a copy of the books in front (alone 1.6); moving
// 980 pages of 32 KB in 8 layers: 174 us = 5.9 TB/s.
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
  int* fork;       // [kMaxForks][6] parent, child, full pages, tokens behind them, their page, its copy
};
__device__ inline Lists lists_of(void* ws, int n_pages) {
  Lists l;
  l.count = static_cast<int*>(ws);
  l.fork = l.count + 64;
  l.src = l.fork + 6 * kMaxForks;
  l.dst = l.src + n_pages;
  l.remap = l.dst + n_pages;
  return l;
}

__device__ __forceinline__ void st_cluster_u32(uint32_t cluster_addr, unsigned v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
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

// Which of up to kSpan pages from `base` on are in use, as bits: a warp has `words` runs of 32 pages, lane i its words i and i + 32.
constexpr int kSpan = 65536;
struct PageBits {
  unsigned used[2];
  int words, from;     // words of a warp; this warp's first page
  __device__ __forceinline__ int page(int half) const { return from + 32 * ((threadIdx.x & 31) + 32 * half); }   // of bit 0
  // bits of the pages lo <= page < hi
  __device__ __forceinline__ unsigned between(int half, int lo, int hi) const {
    const int p = page(half);
    if (static_cast<int>(threadIdx.x & 31) + 32 * half >= words) return 0;
    const unsigned above = lo <= p ? ~0u : lo - p >= 32 ? 0u : ~0u << (lo - p);
    const unsigned below = hi <= p ? 0u : hi - p >= 32 ? ~0u : (1u << (hi - p)) - 1;
    return above & below;
  }
};
// By all CTAs of the cluster: each reads an eighth, the words meet in CTA 0's `s_words`, and CTA 0 gets its bits.  A store into
// CTA 0's shared memory has to come behind its start, and between two calls behind its use of the words before: every call waits
// in front of its stores (the loads are under way) for an arrival of all CTAs, the kernel's first statement or next_span().
constexpr int kBookCtas = 8;
__device__ __forceinline__ PageBits page_bits(const int* refs, int n_pages, int base, unsigned* s_words) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = static_cast<int>(cluster_ctarank());
  const int n = n_pages - base < kSpan ? n_pages - base : kSpan;
  PageBits b;
  b.words = (n + 32 * 32 - 1) / (32 * 32);
  b.from = base + warp * b.words * 32;
  const int all = (n + 31) / 32, share = 32 * ((all + 32 * kBookCtas - 1) / (32 * kBookCtas));   // words; of a CTA
  const int word0 = rank * share + warp * (share / 32);   // this warp's share / 32 <= 8 words
  int count[8];   // (all requested before the first is looked at; behind the last page: that one again)
#pragma unroll
  for (int k = 0; k < 8; ++k) count[k] = __ldcg(refs + min(base + (word0 + k) * 32 + lane, n_pages - 1));
  const uint32_t dst = map_to_rank(smem_u32(s_words), 0);
  __syncwarp();   // (the barrier is for whole warps)
  cluster_wait_acquire();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const unsigned word = __ballot_sync(~0u, count[k] != 0);
    if (lane == k && k < share / 32 && word0 + k < all) st_cluster_u32(dst + 4 * (word0 + k), word);
  }
  __syncwarp();
  cluster_arrive_release();
  cluster_wait_acquire();
  if (rank == 0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = warp * b.words + lane + 32 * h;
      b.used[h] = lane + 32 * h < b.words && k < all ? s_words[k] & b.between(h, 0, n_pages) : 0;
    }
  }
  return b;
}
__device__ __forceinline__ void next_span() {
  __syncwarp();
  cluster_arrive_release();
}
// Numbers the set bits of w[0], w[1] over the whole CTA in the order of the pages; returns how many there are.  first[]: of
// each word's lowest.
__device__ __forceinline__ int rank_bits(const unsigned (&w)[2], int (&first)[2], int* s_scan) {
  int incl[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    incl[h] = __popc(w[h]);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(~0u, incl[h], o);
      if (static_cast<int>(threadIdx.x & 31) >= o) incl[h] += up;
    }
  }
  const int low = __shfl_sync(~0u, incl[0], 31), high = __shfl_sync(~0u, incl[1], 31);
  int total;
  const int before = block_scan((threadIdx.x & 31) == 0 ? low + high : 0, &total, s_scan);
  const int warp_first = __shfl_sync(~0u, before, 0);
  first[0] = warp_first + incl[0] - __popc(w[0]);
  first[1] = warp_first + low + incl[1] - __popc(w[1]);
  return total;
}
// list[rank] = page for the set bits with base + rank < limit.
__device__ __forceinline__ void write_bits(const PageBits& b, const unsigned (&w)[2], const int (&first)[2], int base, long long limit, int* list) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int rank = base + first[h];
#pragma unroll 1
    for (unsigned m = w[h]; m && rank < limit; m &= m - 1) list[rank++] = b.page(h) + __ffs(m) - 1;
  }
}
// By all CTAs of the cluster; CTA 0: the lowest free pages into list[0 .. need), returns how many there are (or `need` and more).
__device__ __forceinline__ int free_pages(const int* refs, int n_pages, long long need, int* list, int* s_scan, unsigned* s_words) {
  int have = 0;
#pragma unroll 1
  for (int base = 0; base < n_pages; base += kSpan) {
    if (base) next_span();
    const PageBits b = page_bits(refs, n_pages, base, s_words);
    if (cluster_ctarank() == 0 && have < need) {
      const unsigned w[2] = {~b.used[0] & b.between(0, 0, n_pages), ~b.used[1] & b.between(1, 0, n_pages)};
      int first[2];
      const int found = rank_bits(w, first, s_scan);
      write_bits(b, w, first, have, need, list);
      have += found;
    }
    if (base > 0x7fffffff - kSpan) break;
  }
  return have;
}

// ---- vq_kv_reserve ------------------------------------------------------------------------------------------------
__global__ void __cluster_dims__(kBookCtas, 1, 1) __launch_bounds__(kBookThreads) reserve_kernel(KvGeometry g, KvBooks b, int* refs, const int* grow, int* status, void* ws) {
  __shared__ int s_scan[32];
  __shared__ long long s_need[32];
  __shared__ int s_first[kBookThreads];   // pages in front of a thread's sequences
  __shared__ int s_have[kBookThreads];    // pages that its first sequence has
  __shared__ unsigned s_words[kSpan / 32];
  cluster_arrive_release();   // (page_bits waits)
  pdl_launch_dependents();
  pdl_wait();
  if (cluster_ctarank() != 0) {
    free_pages(refs, g.n_pages, 0, nullptr, s_scan, s_words);
    return;
  }
  const int tid = threadIdx.x;
  const Lists l = lists_of(ws, g.n_pages);
  const int per = (b.n_seqs + kBookThreads - 1) / kBookThreads, s0 = tid * per, s1 = min(b.n_seqs, s0 + per);
  struct Share {
    int len, more, pages;   // tokens there are, tokens to come, pages for them (-1: the row is too short)
  };
  auto share_of = [&](int s) {
    Share h;
    h.len = clamp_len(b, __ldcg(b.len + s));
    h.more = grow ? max(0, __ldcg(grow + s)) : 1;
    h.pages = h.more > b.max_len - h.len ? -1 : ((h.len + h.more + g.page_tokens - 1) >> g.page_shift) - ((h.len + g.page_tokens - 1) >> g.page_shift);
    return h;
  };
  const Share mine = s0 < s1 ? share_of(s0) : Share{0, 0, 0};
  long long need = mine.pages;
  int too_long = mine.pages < 0;
#pragma unroll 1
  for (int s = s0 + 1; s < s1; ++s) {
    const Share h = share_of(s);
    need += h.pages;
    too_long += h.pages < 0;
  }
  long long total;
  const long long before = block_scan(need, &total, s_need);
  s_first[tid] = static_cast<int>(min(before, 0x7fffffffll));   // (no more than the pool has are given out: 32 bits)
  s_have[tid] = (mine.len + g.page_tokens - 1) >> g.page_shift;
  const int any_long = __syncthreads_count(too_long);
  const int have = free_pages(refs, g.n_pages, any_long ? 0 : total, l.dst, s_scan, s_words);
  if (any_long) {
    int all;
    block_scan(too_long, &all, s_scan);
    if (tid == 0) {
      status[0] = 0;
      status[1] = all;
    }
    return;
  }
  if (total > 0) {
    if (have < total) {
      if (tid == 0) {
        status[0] = total - have < 0x7fffffff ? static_cast<int>(total - have) : 0x7fffffff;
        status[1] = 0;
      }
      return;
    }
    __syncthreads();
    int page_ahead = tid < total ? l.dst[tid] : 0;
#pragma unroll 1
    for (int r = tid; r < total; r += kBookThreads) {
      const int page = page_ahead;
      if (r + kBookThreads < total) page_ahead = l.dst[r + kBookThreads];
      int lo = 0;   // last thread whose sequences' share begins at or in front of r
#pragma unroll
      for (int step = kBookThreads / 2; step; step >>= 1)
        if (s_first[lo + step] <= r) lo += step;
      int s = lo * per, at = r - s_first[lo], there = s_have[lo];
      if (per > 1) {   // a thread's sequences one by one
        Share h = share_of(s);
        while (at >= h.pages) {
          at -= h.pages;
          h = share_of(++s);
        }
        there = (h.len + g.page_tokens - 1) >> g.page_shift;
      }
      b.table[static_cast<long long>(s) * b.table_stride + there + at] = page;
      refs[page] = 1;
    }
    __syncthreads();   // the lengths have been read
  }
  if (s0 < s1) b.len[s0] = mine.len + mine.more;
#pragma unroll 1
  for (int s = s0 + 1; s < s1; ++s) {
    const Share h = share_of(s);
    b.len[s] = h.len + h.more;
  }
  if (tid == 0) status[0] = status[1] = 0;
}

// ---- vq_kv_fork: the list of forks, pages for their last tokens ---------------------------------------------------------
__global__ void __cluster_dims__(kBookCtas, 1, 1) __launch_bounds__(kBookThreads) fork_kernel(KvGeometry g, KvBooks b, int* refs, const int* pairs, int n_pairs, int* status,
                                                           void* ws) {
  __shared__ int s_scan[32];
  __shared__ int s_child[kMaxForks];
  __shared__ unsigned s_words[kSpan / 32];
  cluster_arrive_release();   // (page_bits waits)
  pdl_launch_dependents();
  pdl_wait();
  if (cluster_ctarank() != 0) {
    free_pages(refs, g.n_pages, 0, nullptr, s_scan, s_words);
    return;
  }
  const int i = threadIdx.x;
  const Lists l = lists_of(ws, g.n_pages);
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
  const int have = free_pages(refs, g.n_pages, total, l.dst, s_scan, s_words);
  if (total > 0) {
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
__global__ void __launch_bounds__(kBookThreads) free_kernel(KvGeometry g, KvBooks b, int* refs, const int* slots, int n_slots) {
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
  for (int j0 = threadIdx.x; j0 < pages; j0 += 4 * blockDim.x) {
    int page[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) page[k] = j0 + k * static_cast<int>(blockDim.x) < pages ? __ldcg(row + j0 + k * blockDim.x) : -1;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (static_cast<unsigned>(page[k]) < static_cast<unsigned>(g.n_pages)) atomicSub(refs + page[k], 1);
  }
}

// ---- vq_kv_compact: which page goes where ---------------------------------------------------------------------------
__global__ void __cluster_dims__(kBookCtas, 1, 1) __launch_bounds__(kBookThreads) compact_kernel(KvGeometry g, KvBooks b, int* refs, int* status, void* ws) {
  __shared__ int s_scan[32];
  __shared__ unsigned s_words[kSpan / 32];
  cluster_arrive_release();   // (page_bits waits)
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x;
  const Lists l = lists_of(ws, g.n_pages);
  const bool lead = cluster_ctarank() == 0;
  PageBits bits = page_bits(refs, g.n_pages, 0, s_words);
  int mine = lead ? __popc(bits.used[0]) + __popc(bits.used[1]) : 0;
  const int spans = (g.n_pages - 1) / kSpan + 1;
#pragma unroll 1
  for (int k = 1; k < spans; ++k) {
    next_span();
    const PageBits more = page_bits(refs, g.n_pages, k * kSpan, s_words);
    if (lead) mine += __popc(more.used[0]) + __popc(more.used[1]);
  }
  int used, moved = 0, holes = 0;
  block_scan(mine, &used, s_scan);
#pragma unroll 1
  for (int k = 0; k < spans; ++k) {
    if (spans > 1) {
      next_span();
      bits = page_bits(refs, g.n_pages, k * kSpan, s_words);
    }
    if (!lead) continue;
    const unsigned from[2] = {bits.used[0] & bits.between(0, used, g.n_pages), bits.used[1] & bits.between(1, used, g.n_pages)};
    const unsigned to[2] = {~bits.used[0] & bits.between(0, 0, used), ~bits.used[1] & bits.between(1, 0, used)};
    int first[2];
    int found = rank_bits(from, first, s_scan);
    write_bits(bits, from, first, moved, g.n_pages, l.src);
    moved += found;
    found = rank_bits(to, first, s_scan);
    write_bits(bits, to, first, holes, g.n_pages, l.dst);
    holes += found;
  }
  if (!lead) return;
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
  const Lists l = lists_of(ws, g.n_pages);
  const int count = KIND == kPairs ? n_pairs : __ldcg(l.count);
  const long long warps = static_cast<long long>(gridDim.x) * (kCopyThreads / 32);
  const long long warp0 = static_cast<long long>(blockIdx.x) * (kCopyThreads / 32) + (threadIdx.x >> 5);

  // page data: (entry, layer, keys | values, run of 4 KB)
  const long long page_bytes = static_cast<long long>(g.heads) * g.page_tokens * g.row_bytes;
  const int runs = static_cast<int>((page_bytes + 4095) / 4096);
  const long long scale_words = static_cast<long long>(g.heads) * g.page_tokens;
  const long long items = static_cast<long long>(count) * pools.n_layers * 2 * runs;
  for (long long it = warp0; it < items; it += warps) {
    // (forks: the first runs of every page before any page's later ones, which are behind the last token more often)
    const long long pieces = static_cast<long long>(count) * pools.n_layers * 2;
    const int run = static_cast<int>(KIND == kForks ? it / pieces : it % runs);
    const long long rest_it = KIND == kForks ? it % pieces : it / runs;
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
      uint4 v[8];
      int at[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int u = run * 256 + 32 * i + lane, head = u / per_head;
        at[i] = u < units ? head * head_units + u - head * per_head : -1;
        if (at[i] >= 0) v[i] = __ldcg(reinterpret_cast<const uint4*>(from) + at[i]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (at[i] >= 0) reinterpret_cast<uint4*>(to)[at[i]] = v[i];
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
  return sizeof(int) * (64 + 6 * static_cast<size_t>(kMaxForks) + 3 * static_cast<size_t>(g.n_pages) + static_cast<size_t>(n_seqs));
}

vq_status launch_kv_reserve(const KvGeometry& g, const KvBooks& books, int* refs, const int* grow, int* status, void* ws, cudaStream_t s) {
  return launch_dependent(reserve_kernel, dim3(kBookCtas), dim3(kBookThreads), 0, s, g, books, refs, grow, status, ws);
}

vq_status launch_kv_fork(const KvGeometry& g, const KvPools& pools, const KvBooks& books, int* refs, const int* pairs, int n_pairs,
                         int* status, void* ws, cudaStream_t s) {
  const vq_status st = launch_dependent(fork_kernel, dim3(kBookCtas), dim3(kBookThreads), 0, s, g, books, refs, pairs, n_pairs, status, ws);
  if (st != VQ_OK) return st;
  return launch_copy<kForks>(g, pools, books, refs, nullptr, 0, ws, s);
}

vq_status launch_kv_free(const KvGeometry& g, const KvBooks& books, int* refs, const int* slots, int n_slots, cudaStream_t s) {
  return launch_dependent(free_kernel, dim3(static_cast<unsigned>(n_slots)), dim3(books.table_stride > 1024 ? kBookThreads : 256), 0, s, g, books,
                          refs, slots, n_slots);
}

vq_status launch_kv_compact(const KvGeometry& g, const KvPools& pools, const KvBooks& books, int* refs, int* status, void* ws,
                            cudaStream_t s) {
  const vq_status st = launch_dependent(compact_kernel, dim3(kBookCtas), dim3(kBookThreads), 0, s, g, books, refs, status, ws);
  if (st != VQ_OK) return st;
  return launch_copy<kMoves>(g, pools, books, refs, nullptr, 0, ws, s);
}

vq_status launch_kv_copy_pages(const KvGeometry& g, const KvPools& pools, const int* pairs, int n_pairs, cudaStream_t s) {
  KvBooks none = {};
  return launch_copy<kPairs>(g, pools, none, nullptr, pairs, n_pairs, nullptr, s);
}

}  // namespace vq
