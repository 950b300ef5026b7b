// Attention of one new token per sequence over a paged cache (vq_kv_attention).
//
//   out[h] = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale * q_h . k_t - m),  m the running maximum,
// one pass over keys and values: maximum and sum run along, accumulators are rescaled when the maximum has grown by a factor
// of 2^kSlack (weights stay in range till then, so most tiles need no exchange between lanes).
//
// Bound by memory: every key and value is read once, 4 * group multiply-adds per pair of stored values, far below what the
// tensor cores need.  So the products run as mma.sync m16n8k16 straight from the tiles in shared memory, the tokens (first
// product) and the dimensions (second) as the 16 rows, eight query heads of one key/value head as the columns: no operand
// passes through tensor memory, and the scores turn into the second product's operand in registers (movmatrix).
//
// Split: the tokens of all sequences and key/value heads form one list of tiles (sequence, head, tile); each CTA takes an
// equal run of it and each warp an equal part of that, wherever sequences end, so lengths need not be known on the host
// and ragged batches stay balanced.  A warp has a ring of tiled TMA copies of its own (a box never crosses a page; lane i
// requests box i, so a tile costs the warp one request) that runs on over the ends of sequences: there is no barrier
// before the end of the run.  A head that lies in one warp's part is finished there.  What is cut between warps is joined
// at the CTA's end, what is cut between CTAs goes to the workspace (accumulators, maximum, sum) and is joined by the CTA
// that arrives last - in the order of the list, so results do not depend on which one that is.
// 16 sequences of 40000 tokens, 64/8 heads of 128: 393 us = 6.7 TB/s, in an 8-bit cache 212 = 6.4; 16 of 4096 tokens, 32/8 heads:
// 46.8 us (a plain read of as many bytes takes 44.8); one of 512: 8.0.
#include <math.h>

#include "vq_device.cuh"
#include "vq_kv.cuh"

namespace vq {
namespace {

using namespace dev;

constexpr int kToll = 2;                // places in front of a head's tiles: what beginning and ending one costs, in tiles
constexpr int kWaitTries = 1 << 18;     // mbarrier polls before a warp gives up and flags an error
constexpr int kMaxHeads = 16;           // query heads that a CTA takes together at most
constexpr int kMaxCtas = 256;           // CTAs of a launch, one per SM (partial sums and counters are sized for them)
constexpr int kMaxWarps = 12;
// Weights are held as 2^kLift * exp(...): up to 2^(kLift + kSlack) fits binary16, and weights down to 2^-21 of the largest are normal
// numbers.  The two binary16 pieces of a weight w (w rounded, and the rest rounded) are off by 2^-23 w at most where the second is a
// normal number, and by 2^-25 where it is not: 2^-32 of the largest weight, which is 2^kLift or more.
constexpr float kLift = 7.0f, kSlack = 8.0f;

struct AttnArgs {
  const float* ks;
  const float* vs;
  const int* table;
  const int* len;
  const __half* q;
  __half* out;
  float* lse;
  float* partial;
  int* counters;
  int* error_flag;
  long long q_stride, out_stride;
  int n_seqs, table_stride, max_len, n_pages, page_shift, run_shift, heads, group, chunks, n_q_heads, window;
  float scale_log2, inv_grid;
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Counts an arrival; what the CTA wrote (in front of its barrier) is there for whoever counts later.
__device__ __forceinline__ int arrive(int* counter) {
  int old;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(old) : "l"(counter) : "memory");
  return old;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ float lds_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float log2_fast(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Transposes an 8 x 8 matrix of binary16 held a row to four lanes.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float inverse(float sum) { return sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f; }   // 0: no token at all
__device__ __forceinline__ float log_sum(float top, float sum) {   // natural, of 2^(top - kLift) * sum
  return ((top == -INFINITY ? 0.0f : top) - kLift + log2f(sum)) * 0.693147180559945309f;
}
__device__ __forceinline__ float2 unpack_half2(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
// Two signed bytes (already offset by 128) into binary16, exactly: 0x6400 | u is 1024 + u.
template <uint32_t SEL>
__device__ __forceinline__ uint32_t bytes_to_half2(uint32_t u) {
  uint32_t r = prmt(u, 0x64646464u, SEL);
  __half2 h = *reinterpret_cast<__half2*>(&r);
  const uint32_t off = 0x64806480u;   // 1152 = 1024 + 128
  h = __hsub2(h, *reinterpret_cast<const __half2*>(&off));
  return *reinterpret_cast<uint32_t*>(&h);
}

// Shapes of one instantiation: head dimension, 8-bit cache, groups of eight query heads taken together.
template <int D, bool I8, int NH>
struct Shape {
  static constexpr int ROW = D * (I8 ? 1 : 2);          // bytes of one token
  // A tile lies in shared memory as column blocks of 128 bytes (64 where a row has no more) by tokens, 16-byte pieces
  // swizzled by the copy: eight rows of a matrix lie in different banks.  Columns beyond the row are filled, not read.
  static constexpr int CBB = ROW <= 64 ? 64 : 128;
  static constexpr int NCB = (ROW + CBB - 1) / CBB;
  // tokens per tile: a stage of a warp holds about 8 KB of keys and values
  static constexpr int R = I8 ? (ROW <= 64 ? 4 : ROW <= 128 ? 2 : 1) : (ROW <= 128 ? 2 : 1);
  static constexpr int TT = 16 * R;
  static constexpr int HALVES = TT / 8;                 // runs of 8 tokens: never across a page
  static constexpr int WIN = 32 / HALVES;               // tiles whose pages a warp's lanes hold
  static constexpr int KV = TT * NCB * CBB;
  static constexpr int STAGE = 2 * KV;
  static constexpr int SCALES = I8 ? 2 * TT * 4 : 0;    // per stage, behind the rings
  static constexpr int HEADS = 8 * NH;
  static constexpr int JROW = D + 4;                    // a row of the join's sums: heads of a lane's neighbours in different banks
  static constexpr int SUMS = HEADS * (D + 2);          // partial sums in the workspace: accumulators, maxima, sums
  // One CTA per SM.  Twelve warps with two stages each where the accumulators leave 168 registers enough (against eight with
  // three: sixteen sequences of 40000 tokens, 64/8 heads of 128, 401 -> 393 us, in an 8-bit cache, whose bytes become binary16
  // for both products, 228 -> 224; one sequence of 512 tokens 8.3 -> 8.8), else eight, else four.
  static constexpr int fit(int warps) { return (226 * 1024 - 8192) / (warps * (STAGE + SCALES)); }
  static constexpr int WARPS = NH == 1 && D <= 128 && fit(12) >= 2 ? 12 : fit(8) >= 3 && 3 * STAGE >= 2 * HEADS * JROW * 4 ? 8 : 4, THREADS = 32 * WARPS;
  static constexpr int NS = fit(WARPS) > 6 ? 6 : fit(WARPS);   // stages of a warp's ring
  static constexpr int RINGS = WARPS * NS * STAGE;
  static constexpr size_t SMEM = 1024 + static_cast<size_t>(RINGS) + WARPS * NS * SCALES;   // (1024: alignment)
  // Costs of a split (see choose()): measured from calls of 1 to 16 sequences, 8 to 128 heads, 100 to 4096 tokens, up to 8 query heads to
  // a key/value head; elsewhere they are carried over.  A join costs more the more CTAs share a head, which no term counts: one
  // sequence of 32768 tokens with one key/value head takes 44 us with 8 query heads of 128, 157 with 16 of 256.
  static constexpr float JOIN_COST = 22.0f * 8192 / STAGE, RUN_COST = 31.0f * 8192 / STAGE, ALONE = I8 ? 1.11f : 0.625f;
  static constexpr int QREGS = D / 16 * 2 * NH;
  static constexpr bool AHEAD = QREGS <= 32;            // the next piece's queries are fetched under this one
  static_assert(NS * STAGE >= 2 * HEADS * JROW * 4, "a warp's two cut pieces fit its ring");
  static_assert(RINGS >= 2 * kMaxCtas * HEADS * 4, "the factors of a join over all CTAs fit the rings");
  static_assert(NS >= 2 && KV % 1024 == 0, "a ring needs two stages, a swizzled block 1024-byte alignment");
};

// 16-byte piece `c` of row `row` in a swizzled tile.
template <class S>
__device__ __forceinline__ uint32_t piece_at(uint32_t tile, int row, int c) {
  if constexpr (S::CBB == 128) return tile + (c >> 3) * (S::TT * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4);
  return tile + row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
}

__device__ __forceinline__ int clamp_len(const AttnArgs& a, int n) { return n < 0 ? 0 : n > a.max_len ? a.max_len : n; }
__device__ __forceinline__ int first_token(const AttnArgs& a, int n) { return a.window > 0 && n > a.window ? n - a.window : 0; }
// Tiles of a sequence of length n: those that hold a token of the window.
template <int TT>
__device__ __forceinline__ int tile_count(const AttnArgs& a, int n) {
  return n <= 0 ? 0 : (n - 1) / TT - first_token(a, n) / TT + 1;
}

// Empty places in front of the nt tiles of a (sequence, head).  `whole` != 0: they fill up the CTAs' runs of `whole` places, so
// that no CTA has tiles of two heads.  Else kToll: what beginning and ending a head costs, in tiles.
__device__ __forceinline__ int lead_places(int nt, int whole) { return whole ? (whole - 1) - (nt + whole - 1) % whole : kToll; }

// Position in the list: a piece is a run of tiles of one (sequence, head), inside one warp's part.
struct Walk {
  int x;                // place of the piece's beginning (a launch's list has fewer than 2^31)
  int seq, hc;          // sequence; key/value head and chunk of its query heads
  int at, nt, lead;     // place within the (sequence, head), its tiles, the places in front of them
  int n, begin;         // the sequence's length and first token
  __device__ __forceinline__ int first() const { return at < lead ? 0 : at - lead; }
  __device__ __forceinline__ int places(int x1) const {
    const int rest = nt + lead - at;
    return x1 - x < rest ? x1 - x : rest;
  }
  __device__ __forceinline__ int count(int x1) const {
    const int end = at + places(x1) - lead;
    return end > first() ? end - first() : 0;
  }
};

// A cut piece: what a warp has of a (sequence, head).  Two per warp, in the order of the list: one that began in front of
// the warp's part and ends in it (its sums are parked in the workspace while the warp goes on), and the last one (its
// sums go to the warp's ring when that has run dry).
struct Part {
  int seq, hc;          // hc < 0: there is none
  int t0, t1, nt;       // tiles of it
  int begin;            // place of the (sequence, head)'s first tile
};

template <int D, bool I8, int NH>
__global__ void __launch_bounds__(Shape<D, I8, NH>::THREADS, 1)
attention_kernel(AttnArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using S = Shape<D, I8, NH>;
  constexpr int TT = S::TT, R = S::R, HALVES = S::HALVES, NS = S::NS, HEADS = S::HEADS, WIN = S::WIN;
  constexpr int KSTEPS = D / 16, MT = D / 16, kWarps = S::WARPS, kThreads = S::THREADS;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  __shared__ __align__(8) unsigned long long s_bar[kWarps][NS];
  __shared__ int s_len[2 * kThreads];
  __shared__ int s_scan[kWarps + 1], s_sums[2][kWarps];
  __shared__ int s_bad[kWarps][NS];
  __shared__ float s_m[2 * kWarps][HEADS], s_l[2 * kWarps][HEADS];
  __shared__ Part s_part[2 * kWarps];
  __shared__ int s_last, s_empty, s_join[2], s_cta[2][2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  const uint32_t bars = smem_u32(s_bar[warp]);
  if (lane < NS) mbar_init(bars + 8 * lane, I8 ? 33 : 1);   // (8-bit: every lane arrives with its part of the scales)
  mbar_init_fence();
  pdl_launch_dependents();
  pdl_wait();
  const int hc_count = a.heads * a.chunks;

  // ---- the list of tiles: total, this CTA's run, this warp's part of it ----
  auto zeros = [&](int s) {   // a sequence without tokens
#pragma unroll 1
    for (int i = tid; i < a.n_q_heads * D / 8; i += kThreads) *reinterpret_cast<uint4*>(a.out + s * a.out_stride + i * 8) = make_uint4(0, 0, 0, 0);
    if (a.lse)
#pragma unroll 1
      for (int h = tid; h < a.n_q_heads; h += kThreads) a.lse[static_cast<long long>(s) * a.n_q_heads + h] = -INFINITY;
  };
  const int cta = blockIdx.x, grid = gridDim.x;
  bool snap = false;
  int whole_run = 0, run = 0, x0 = 0, x1 = 0, wx0 = 0, wx1 = 0;
  // Which split?  In tiles of a CTA at its fair share of the memory's rate (0.19 us for one of 8 KB):
  //   a CTA per head               the longest head at the rate that one SM reaches alone, or the mean and a little if that is more
  //   an equal number of CTAs each  the longest head's part, and the join of CTAs
  //   equal runs over heads' ends   the mean, and the join, and the sums that warps park
  // (16 sequences of 1000 tokens, 32/8 heads of 128, by equal runs 21.1 us, by heads 16.7; of 4096 tokens 51.2 and 46.7; of
  // 32768 tokens 328 and 338.)  tiles, used, most: of all sequences, for one head: tiles, sequences that have some, tiles of the
  // longest.
  auto choose = [&](int tiles, int used, int most) {
    const int heads = used * hc_count;
    whole_run = 0;
    // Equal runs of whole heads, where a head is less than the join, but long enough to be cut often, and a run has few sequences
    // (its ends are found one by one).  200 sequences of 300 tokens, 64/8 heads of 64: 34.2 -> 30.5 us; of 64 tokens 9.1 -> 9.6.
    snap = most >= 4 && most <= S::JOIN_COST && used <= 8 * grid;
    if (heads > grid) return;
    const float mean = tiles * hc_count * a.inv_grid, run_cost = mean + S::RUN_COST;
    const float whole_cost = fmaxf(most * S::ALONE, 1.04f * mean);
    if (whole_cost <= run_cost) whole_run = most;
    if (whole_cost <= kWarps + S::JOIN_COST && whole_run) return;
    int each = static_cast<int>(__fdividef(static_cast<float>(grid), static_cast<float>(heads)));   // (heads * each <= grid)
    each = heads * each > grid ? each - 1 : each;
    each = each < 1 ? 1 : each;
    const int per = static_cast<int>(__fdividef(static_cast<float>(most), static_cast<float>(each))) + 1;
    const int part = per > kWarps ? per : kWarps;
    const float part_cost = part + S::JOIN_COST;
    if (part_cost < whole_cost && part_cost <= run_cost && each * part >= most) whole_run = part;   // (so a head has `each` CTAs at most)
  };
  // places: of the list
  auto partition = [&](int total) {
    run = whole_run ? whole_run : (total + grid - 1) / grid;   // places per CTA
    if (static_cast<long long>(cta) * run >= total) return false;
    x0 = cta * run;
    x1 = total - x0 < run ? total : x0 + run;
    return true;
  };
  auto share_out = [&](int from) {   // the run's places from `from` on, to the warps
    const int each = (x1 - from) / kWarps, more = (x1 - from) % kWarps;   // (the first `more` warps have one place more)
    wx0 = from + warp * each + (warp < more ? warp : more);
    wx1 = wx0 + each + (warp < more);
  };
  Walk cur;
  int chunk_base = 0;   // s_len holds the lengths of the 2 kThreads sequences from here on
  auto open_at = [&](int seq, int n, int place, int seq_place) {   // cur: `place` in the sequence that begins at seq_place
    cur.seq = seq;
    cur.x = place;
    cur.n = n;
    cur.begin = first_token(a, n);
    cur.nt = tile_count<TT>(a, n);
    cur.lead = lead_places(cur.nt, whole_run);
    cur.hc = (place - seq_place) / (cur.nt + cur.lead);
    cur.at = place - seq_place - cur.hc * (cur.nt + cur.lead);
  };
  if (a.n_seqs <= 32) {   // every warp by itself: a lane per sequence, no barrier
    const int n = lane < a.n_seqs ? clamp_len(a, __ldcg(a.len + lane)) : 0;
    s_len[lane] = n;   // (every warp writes the same)
    __syncwarp();
#pragma unroll 1
    for (unsigned empty = __ballot_sync(~0u, lane < a.n_seqs && n == 0 && lane % grid == cta); empty; empty &= empty - 1) zeros(__ffs(empty) - 1);
    const int nt = tile_count<TT>(a, n);
    const int tiles = __reduce_add_sync(~0u, nt), most = __reduce_max_sync(~0u, nt), used = __popc(__ballot_sync(~0u, nt > 0));
    if (tiles == 0) return;
    choose(tiles, used, most);
    const int places = nt ? (nt + lead_places(nt, whole_run)) * hc_count : 0;
    if (!partition(__reduce_add_sync(~0u, places))) return;
    int end = places;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(~0u, end, o);
      if (lane >= o) end += up;
    }
    if (whole_run || snap) {
      const int seq = __ffs(__ballot_sync(~0u, x0 < end)) - 1, begin = __shfl_sync(~0u, end - places, seq);
      open_at(seq, __shfl_sync(~0u, n, seq), x0, begin);
      if (whole_run) {   // one head: its empty places are nobody's
        if (cur.at < cur.lead) {
          cur.x += cur.lead - cur.at;
          cur.at = cur.lead;
        }
        share_out(cur.x);
        cur.at += wx0 - cur.x;
        cur.x = wx0;
      }
    } else {
      share_out(x0);
      const int seq = __ffs(__ballot_sync(~0u, wx0 < end)) - 1;   // (wx0 < x1 unless the part is empty: then -1 or any)
      const int n_seq = __shfl_sync(~0u, n, seq & 31), begin = __shfl_sync(~0u, end - places, seq & 31);
      if (wx0 < wx1 && seq >= 0) open_at(seq, n_seq, wx0, begin);
      else wx1 = wx0;
    }
  } else {
    if (tid == 0) s_empty = 0;
    __syncthreads();
    int tiles = 0, used = 0, most = 0;
#pragma unroll 1
    for (int base = 0; base < a.n_seqs; base += kThreads) {
      const int s = base + tid;
      const int n = s < a.n_seqs ? clamp_len(a, __ldcg(a.len + s)) : 0;
      if (base == 0) s_len[kThreads + tid] = 0;
      if (base <= kThreads) s_len[base + tid] = n;
      if (s < a.n_seqs && n == 0 && s % grid == cta) s_empty = 1;
      const int nt = tile_count<TT>(a, n);
      tiles += nt;
      used += nt > 0;
      most = nt > most ? nt : most;
    }
    tiles = __reduce_add_sync(~0u, tiles);
    used = __reduce_add_sync(~0u, used);
    most = __reduce_max_sync(~0u, most);
    if (lane == 0) {
      s_scan[warp] = tiles;
      s_sums[0][warp] = used;
      s_sums[1][warp] = most;
    }
    __syncthreads();
    if (s_empty) {
#pragma unroll 1
      for (int s = cta; s < a.n_seqs; s += grid)
        if (__ldcg(a.len + s) <= 0) zeros(s);
    }
    tiles = used = most = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      tiles += s_scan[w];
      used += s_sums[0][w];
      most = s_sums[1][w] > most ? s_sums[1][w] : most;
    }
    if (tiles == 0) return;
    choose(tiles, used, most);
    int total = (tiles + used * kToll) * hc_count;
    if (whole_run) {
      total = 0;
#pragma unroll 1
      for (int s = tid; s < a.n_seqs; s += kThreads) {
        const int nt = tile_count<TT>(a, clamp_len(a, __ldcg(a.len + s)));
        total += nt ? (nt + lead_places(nt, whole_run)) * hc_count : 0;
      }
      total = __reduce_add_sync(~0u, total);
      __syncthreads();
      if (lane == 0) s_scan[warp] = total;
      __syncthreads();
      total = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) total += s_scan[w];
    }
    if (!partition(total)) return;
    // sequence that x0 lies in
#pragma unroll 1
    for (int at = 0;; chunk_base += kThreads) {
      if (chunk_base) {
        __syncthreads();
        s_len[tid] = s_len[kThreads + tid];
        const int s = chunk_base + kThreads + tid;
        s_len[kThreads + tid] = s < a.n_seqs ? clamp_len(a, __ldcg(a.len + s)) : 0;
      }
      const int nt = tile_count<TT>(a, s_len[tid]);
      const int places = nt ? (nt + lead_places(nt, whole_run)) * hc_count : 0;
      int end = places;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(~0u, end, o);
        if (lane >= o) end += up;
      }
      __syncthreads();
      if (lane == 31) s_scan[warp] = end;
      __syncthreads();
      int chunk = 0;
      end += at;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        if (w < warp) end += s_scan[w];
        chunk += s_scan[w];
      }
      if (x0 >= end - places && x0 < end) {
        s_last = tid;
        s_scan[kWarps] = end - places;
      }
      __syncthreads();
      if (x0 < at + chunk) {
        open_at(chunk_base + s_last, s_len[s_last], x0, s_scan[kWarps]);
        share_out(whole_run && cur.at < cur.lead ? x0 - cur.at + cur.lead : x0);   // (one head: its empty places are nobody's)
        break;
      }
      at += chunk;
      if (chunk_base + kThreads >= a.n_seqs) return;   // lengths that change under the call: no run to take
    }
  }
  auto next_sequence = [&](Walk& w) {
#pragma unroll 1
    do {
      if (++w.seq >= a.n_seqs) return false;   // (as above)
      const int i = w.seq - chunk_base;
      w.n = i < 2 * kThreads ? s_len[i] : clamp_len(a, __ldcg(a.len + w.seq));
    } while (w.n == 0);
    w.begin = first_token(a, w.n);
    w.nt = tile_count<TT>(a, w.n);
    w.lead = lead_places(w.nt, whole_run);
    w.hc = w.at = 0;
    return true;
  };
  if (snap && !whole_run) {   // the heads that begin in the run, whole
    if (cur.at > 0) {
      cur.x += cur.nt + cur.lead - cur.at;
      cur.at = 0;
      if (++cur.hc == hc_count && !next_sequence(cur)) return;
    }
    Walk last = cur;
    int start = cur.x - cur.hc * (cur.nt + cur.lead);   // of the sequence
#pragma unroll 1
    while (x1 > start + hc_count * (last.nt + last.lead)) {
      start += hc_count * (last.nt + last.lead);
      if (!next_sequence(last)) return;
    }
    const int each = last.nt + last.lead;
    if (x1 > start) x1 = start + (x1 - start + each - 1) / each * each;
    if (cur.x >= x1) return;
    share_out(cur.x);
  }
  // the next piece with tiles behind w's; w.x == wx1: there is none
  auto advance = [&](Walk& w) {
#pragma unroll 1
    do {
      w.x += w.places(wx1);
      w.at = 0;
      if (w.x >= wx1 || (++w.hc == hc_count && !next_sequence(w))) {
        w.x = wx1;
        return;
      }
    } while (w.count(wx1) == 0);
  };
  if (wx0 < wx1) {
#pragma unroll 1
    while (cur.x != wx0) {   // to the sequence that the part begins in
      const int each = cur.nt + cur.lead;
      const int end = cur.x - cur.at + (hc_count - cur.hc) * each;
      if (wx0 < end) {
        const int off = wx0 - (cur.x - cur.at), more = off / each;
        cur.hc += more;
        cur.at = off - more * each;
        cur.x = wx0;
        break;
      }
      cur.x = end;
      if (!next_sequence(cur)) {
        cur.x = wx1;
        break;
      }
    }
    if (cur.x < wx1 && cur.count(wx1) == 0) advance(cur);
  } else {
    cur.x = wx1;
  }

  // ---- this warp's copies ----
  // A window is up to WIN of them in one piece, their pages a run of 8 tokens to a lane; the next window's pages are on their
  // way while this one's tiles are requested.
  struct Window {
    int pages, head, n, begin, tok, left;
  };
  Walk ahead = cur;
  int ahead_j = 0;   // next tile of `ahead`'s piece
  auto next_window = [&](Window& w) {
    w.left = 0;
    if (ahead.x >= wx1) return;
    const int count = ahead.count(wx1);   // (not 0)
    w.left = count - ahead_j < WIN ? count - ahead_j : WIN;
    w.head = ahead.hc / a.chunks;
    w.n = ahead.n;
    w.begin = ahead.begin;
    w.tok = (ahead.begin / TT + ahead.first() + ahead_j) * TT;
    const int tok = w.tok + lane * 8;
    w.pages = lane < w.left * HALVES && tok < w.n
                  ? __ldcg(a.table + static_cast<long long>(ahead.seq) * a.table_stride + (tok >> a.page_shift)) : -1;
    ahead_j += w.left;
    if (ahead_j == count) {
      advance(ahead);
      ahead_j = 0;
    }
  };
  Window win, win_next;
  win.left = 0;
  next_window(win_next);
  int from = 0;   // lane that holds the first page of the next tile
  const uint32_t ring = smem_u32(smem) + warp * NS * S::STAGE;
  const uint32_t scale_ring = smem_u32(smem) + S::RINGS + warp * NS * S::SCALES;
  // What this lane requests of a tile: a run of 2^run_shift tokens (a page's or the tile's) of one column block of the keys
  // (kind 0) or values (1).  Scales come by 16-byte copies of their own: requests of a few bytes are as dear to the copy engine
  // as boxes.
  const int runs = TT >> a.run_shift;
  const int my_row = (lane & (runs - 1)) << a.run_shift, which = lane / runs;
  const int my_kind = which < 2 * S::NCB ? which / S::NCB : 2;
  const int my_block = which % S::NCB;
  const uint32_t my_dst = my_kind * S::KV + my_block * (TT * S::CBB) + my_row * S::CBB;
  int put = 0, get = 0;
  uint32_t phase = 0;
  int tries = kWaitTries;
  auto issue = [&]() {
    if (win.left == 0) {
      win = win_next;
      from = 0;
      if (win.left) next_window(win_next);
    }
    if (win.left) {
      const uint32_t bar = bars + 8 * put;
      const unsigned bad = __ballot_sync(~0u, static_cast<unsigned>(win.pages) >= static_cast<unsigned>(a.n_pages));
      const int page = __shfl_sync(~0u, win.pages, from + (my_row >> 3));
      const bool on = my_kind < 2 && static_cast<unsigned>(page) < static_cast<unsigned>(a.n_pages);
      const unsigned boxes = __ballot_sync(~0u, on);
      if (lane == 0) {
        s_bad[warp][put] = (bad >> from) & ((1u << HALVES) - 1);
        mbar_arrive_expect_tx(bar, (__popc(boxes) * S::CBB) << a.run_shift);
      }
      __syncwarp();
      if (on) {
        const long long row = ((static_cast<long long>(page) * a.heads + win.head) << a.page_shift) + ((win.tok + my_row) & ((1 << a.page_shift) - 1));
        tma_box_2d(ring + put * S::STAGE + my_dst, my_kind ? &v_map : &k_map, my_block * (S::CBB / (I8 ? 1 : 2)), static_cast<int>(row), bar);
      }
      if constexpr (I8) {   // four tokens to a piece
        constexpr int PIECES = TT / 4;
        const int j = lane % PIECES, tok = win.tok + 4 * j;
        const int its_page = __shfl_sync(~0u, win.pages, from + (j >> 1));
        if (lane < 2 * PIECES && static_cast<unsigned>(its_page) < static_cast<unsigned>(a.n_pages)) {
          const long long row = ((static_cast<long long>(its_page) * a.heads + win.head) << a.page_shift) + (tok & ((1 << a.page_shift) - 1));
          cp_async16(scale_ring + put * S::SCALES + lane * 16, (lane < PIECES ? a.ks : a.vs) + row);
        }
        cp_async_arrive(bar);   // when the lane's copy, if any, has come
      }
      win.tok += TT;
      --win.left;
      from += HALVES;
      put = put + 1 == NS ? 0 : put + 1;
    }
  };

  // Queries as the B operand: lane (g, t4) holds head g, dimensions 2 t4, +1, +8, +9 of a step; 8-bit keys come four
  // dimensions to a register, so there a step's slots hold dimensions 4 t4 .. 4 t4 + 3 in order.
  auto load_queries = [&](const Walk& w, uint32_t (&q)[NH][KSTEPS][2]) {
    const int head = w.hc / a.chunks, q0 = (w.hc - head * a.chunks) * HEADS;
    const __half* base = a.q + w.seq * a.q_stride + static_cast<long long>(head * a.group + q0) * D;
#pragma unroll
    for (int nh = 0; nh < NH; ++nh) {
      const bool on = q0 + nh * 8 + g < a.group;
      const __half* p = base + (nh * 8 + g) * D;
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) {
        q[nh][ks][0] = q[nh][ks][1] = 0;
        if (on) {
          if (I8) {
            const uint2 v = __ldcg(reinterpret_cast<const uint2*>(p + ks * 16 + 4 * t4));
            q[nh][ks][0] = v.x;
            q[nh][ks][1] = v.y;
          } else {
            q[nh][ks][0] = __ldcg(reinterpret_cast<const unsigned int*>(p + ks * 16 + 2 * t4));
            q[nh][ks][1] = __ldcg(reinterpret_cast<const unsigned int*>(p + ks * 16 + 8 + 2 * t4));
          }
        }
      }
    }
  };

#pragma unroll 1
  for (int i = 0; i < NS - 1; ++i) issue();
  uint32_t q[NH][KSTEPS][2];
  if (cur.x < wx1) load_queries(cur, q);

  if (lane < 2) s_part[2 * warp + lane].hc = -1;
#pragma unroll 1
  while (cur.x < wx1) {
    // ---- one piece ----
    const int count = cur.count(wx1), tile0 = cur.first();
    const int head = cur.hc / a.chunks, q0 = (cur.hc - head * a.chunks) * HEADS;
    const int rows = a.group - q0 < HEADS ? a.group - q0 : HEADS;
    Walk next = cur;
    advance(next);
    uint32_t qn[S::AHEAD ? NH : 1][S::AHEAD ? KSTEPS : 1][2];
    if constexpr (S::AHEAD) {
      if (next.x < wx1) load_queries(next, qn);
    }

    float o[MT][NH][4];           // [16 dimensions][8 heads]
    float m[NH][2], l[NH][2];     // heads 2 t4, 2 t4 + 1
#pragma unroll
    for (int nh = 0; nh < NH; ++nh) {
      m[nh][0] = m[nh][1] = -INFINITY;
      l[nh][0] = l[nh][1] = 0.0f;
#pragma unroll
      for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][nh][e] = 0.0f;
    }

#pragma unroll 1
    for (int j = 0; j < count; ++j) {
      __syncwarp();   // every lane is done with the tile before this one: its stage is free
      issue();
      if (!mbar_wait(bars + 8 * get, phase, tries)) {   // (a copy that never completes: wrong output, but the kernel ends)
        if (tries && lane == 0) atomicAdd(a.error_flag, 1);
        tries = 0;
      }
      const uint32_t stage = ring + get * S::STAGE, stage_scales = scale_ring + get * S::SCALES;
      const int tok0 = (cur.begin / TT + tile0 + j) * TT;
      const int bad = s_bad[warp][get];
      if (++get == NS) {
        get = 0;
        phase ^= 1;
      }

      // scores: sc[r][nh] = 16 tokens x 8 heads; two sums a step apart, so that fewer products wait for one another
      float sc[R][NH][4];
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int nh = 0; nh < NH; ++nh)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[r][nh][e] = 0.0f;
      if constexpr (I8) {
        // four matrices at a time: a piece of 32 tokens, or two pieces of 16
        constexpr int KJ = R == 1 ? 2 : 1;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ks += KJ)
#pragma unroll
          for (int rr = 0; rr < R; rr += 2) {
            uint32_t b[4];
            ldmatrix4(b, R == 1 ? piece_at<S>(stage, lane & 15, ks + (lane >> 4)) : piece_at<S>(stage, rr * 16 + lane, ks));
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] ^= 0x80808080u;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const uint32_t a0 = bytes_to_half2<0x4140>(b[2 * r]), a1 = bytes_to_half2<0x4140>(b[2 * r + 1]);
              const uint32_t a2 = bytes_to_half2<0x4342>(b[2 * r]), a3 = bytes_to_half2<0x4342>(b[2 * r + 1]);
              const int k = R == 1 ? ks + r : ks;
#pragma unroll
              for (int nh = 0; nh < NH; ++nh) mma16816(sc[R == 1 ? 0 : rr + r][nh], a0, a1, a2, a3, q[nh][k][0], q[nh][k][1]);
            }
          }
      } else {
        float odd[R][NH][4];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int nh = 0; nh < NH; ++nh)
#pragma unroll
            for (int e = 0; e < 4; ++e) odd[r][nh][e] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
          for (int r = 0; r < R; ++r) {
            uint32_t b[4];
            ldmatrix4(b, piece_at<S>(stage, r * 16 + (lane & 15), 2 * ks + (lane >> 4)));
#pragma unroll
            for (int nh = 0; nh < NH; ++nh) mma16816(ks & 1 ? odd[r][nh] : sc[r][nh], b[0], b[1], b[2], b[3], q[nh][ks][0], q[nh][ks][1]);
          }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int nh = 0; nh < NH; ++nh)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[r][nh][e] += odd[r][nh][e];
      }

      // Scale.  8-bit values are multiplied as integers: the weight of token t carries its value scale, 2^s * scale_v, and the
      // maximum is taken of s + log2 scale_v, so that the largest such weight is 1 whatever the scales are.
      float lv[R][2], sv[R][2];   // log2 scale_v, scale_v of tokens g, g + 8 of a block of 16
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float f = a.scale_log2;
          lv[r][e] = 0.0f;
          sv[r][e] = 1.0f;
          if constexpr (I8) {
            f *= lds_f32(stage_scales + (16 * r + 8 * e + g) * 4);
            sv[r][e] = lds_f32(stage_scales + (TT + 16 * r + 8 * e + g) * 4);
            lv[r][e] = fmaxf(log2_fast(sv[r][e]), -40.0f);   // (a scale of 0 goes with integers of 0)
          }
#pragma unroll
          for (int nh = 0; nh < NH; ++nh) {
            sc[r][nh][2 * e] *= f;
            sc[r][nh][2 * e + 1] *= f;
          }
        }
      if (tok0 < cur.begin || tok0 + TT > cur.n || bad) {   // tokens that do not take part
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int tok = tok0 + 16 * r + 8 * e + g;
            if (tok < cur.begin || tok >= cur.n || ((bad >> (2 * r + e)) & 1)) {
#pragma unroll
              for (int nh = 0; nh < NH; ++nh) sc[r][nh][2 * e] = sc[r][nh][2 * e + 1] = -INFINITY;
              lv[r][e] = sv[r][e] = 0.0f;
            }
          }
        // their values become zeros: a weight of 0 does not silence an infinity or NaN
#pragma unroll 1
        for (int i = lane; i < TT * S::NCB * (S::CBB / 16); i += 32) {
          const int row = i / (S::CBB / 16) % TT, tok = tok0 + row;
          if (tok < cur.begin || tok >= cur.n || ((bad >> (row >> 3)) & 1)) sts128(stage + S::KV + i * 16, make_uint4(0, 0, 0, 0));
        }
        fence_proxy_async();   // (the stage's next copy comes behind these writes)
        __syncwarp();
      }

      // running maximum
      float top[NH][2];
      bool up = false;
#pragma unroll
      for (int nh = 0; nh < NH; ++nh)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          top[nh][h] = -INFINITY;
#pragma unroll
          for (int r = 0; r < R; ++r) top[nh][h] = fmaxf(top[nh][h], fmaxf(sc[r][nh][h] + lv[r][0], sc[r][nh][2 + h] + lv[r][1]));
          up |= top[nh][h] > m[nh][h] + kSlack;
        }
      if (__any_sync(~0u, up)) {
#pragma unroll
        for (int nh = 0; nh < NH; ++nh)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float t = top[nh][h];
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) t = fmaxf(t, __shfl_xor_sync(~0u, t, x));
            t = fmaxf(t, m[nh][h]);
            const float alpha = t == -INFINITY ? 1.0f : exp2_fast(m[nh][h] - t);
            m[nh][h] = t;
            l[nh][h] *= alpha;
#pragma unroll
            for (int j2 = 0; j2 < MT; ++j2) {
              o[j2][nh][h] *= alpha;
              o[j2][nh][2 + h] *= alpha;
            }
          }
      }

      // weights: each the sum of two binary16 numbers, so that 22 significant bits reach the product
      uint32_t ph[R][NH][2], pl[R][NH][2];
#pragma unroll
      for (int nh = 0; nh < NH; ++nh) {
        const float b0 = (m[nh][0] == -INFINITY ? 0.0f : m[nh][0]) - kLift, b1 = (m[nh][1] == -INFINITY ? 0.0f : m[nh][1]) - kLift;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float e0 = sc[r][nh][2 * e] - b0, e1 = sc[r][nh][2 * e + 1] - b1;
            float p0 = exp2_fast(e0), p1 = exp2_fast(e1);
            l[nh][0] += p0;
            l[nh][1] += p1;
            if constexpr (I8) {
              p0 *= sv[r][e];   // (2^55 at most in front of a scale of 2^-40)
              p1 *= sv[r][e];
            }
            const uint32_t hi = pack_half2(p0, p1);
            const float2 back = unpack_half2(hi);
            ph[r][nh][e] = transpose8x8(hi);
            pl[r][nh][e] = transpose8x8(pack_half2(p0 - back.x, p1 - back.y));
          }
      }

      // values
      if constexpr (I8) {
        // A transposed matrix gives a lane two adjacent dimensions of two tokens: rows g of the operand are the even
        // dimensions of a run of 16, rows g + 8 the odd ones.
        constexpr int CJ = R == 1 ? 2 : 1;
#pragma unroll
        for (int c = 0; c < MT; c += CJ)
#pragma unroll
          for (int rr = 0; rr < R; rr += 2) {
            uint32_t b[4];
            ldmatrix4_trans(b, R == 1 ? piece_at<S>(stage + S::KV, lane & 15, c + (lane >> 4)) : piece_at<S>(stage + S::KV, rr * 16 + lane, c));
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] ^= 0x80808080u;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const uint32_t a0 = bytes_to_half2<0x4240>(b[2 * r]), a1 = bytes_to_half2<0x4341>(b[2 * r]);
              const uint32_t a2 = bytes_to_half2<0x4240>(b[2 * r + 1]), a3 = bytes_to_half2<0x4341>(b[2 * r + 1]);
              const int j = R == 1 ? c + r : c, block = R == 1 ? 0 : rr + r;
#pragma unroll
              for (int nh = 0; nh < NH; ++nh) {
                mma16816(o[j][nh], a0, a1, a2, a3, ph[block][nh][0], ph[block][nh][1]);
                mma16816(o[j][nh], a0, a1, a2, a3, pl[block][nh][0], pl[block][nh][1]);
              }
            }
          }
      } else {
#pragma unroll
        for (int c = 0; c < MT; ++c)
#pragma unroll
          for (int r = 0; r < R; ++r) {
            uint32_t b[4];
            ldmatrix4_trans(b, piece_at<S>(stage + S::KV, r * 16 + (lane & 7) + ((lane >> 4) << 3), 2 * c + ((lane >> 3) & 1)));
#pragma unroll
            for (int nh = 0; nh < NH; ++nh) {
              mma16816(o[c][nh], b[0], b[1], b[2], b[3], ph[r][nh][0], ph[r][nh][1]);
              mma16816(o[c][nh], b[0], b[1], b[2], b[3], pl[r][nh][0], pl[r][nh][1]);
            }
          }
      }
    }

#pragma unroll
    for (int nh = 0; nh < NH; ++nh)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[nh][h] += __shfl_xor_sync(~0u, l[nh][h], x);
    if (count == cur.nt) {
      // ---- all of the head: out = o / l, eight heads by sixteen dimensions turned round at a time ----
      __half* out = a.out + cur.seq * a.out_stride + static_cast<long long>(head * a.group + q0) * D;
      const long long out_row = static_cast<long long>(cur.seq) * a.n_q_heads + head * a.group + q0;
#pragma unroll
      for (int nh = 0; nh < NH; ++nh) {
        float inv[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          inv[h] = inverse(l[nh][h]);
          const int row = nh * 8 + 2 * t4 + h;
          if (a.lse && g == 0 && row < rows) a.lse[out_row + row] = log_sum(m[nh][h], l[nh][h]);
        }
        const int row = nh * 8 + g;
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          const uint32_t u = transpose8x8(pack_half2(o[j][nh][0] * inv[0], o[j][nh][1] * inv[1]));
          const uint32_t w = transpose8x8(pack_half2(o[j][nh][2] * inv[0], o[j][nh][3] * inv[1]));
          if (row < rows) {
            __half* d = out + row * D + 16 * j;
            if (I8) {   // even dimensions in u, odd ones in w
              *reinterpret_cast<uint2*>(d + 4 * t4) = make_uint2(prmt(u, w, 0x5410), prmt(u, w, 0x7632));
            } else {
              *reinterpret_cast<uint32_t*>(d + 2 * t4) = u;
              *reinterpret_cast<uint32_t*>(d + 8 + 2 * t4) = w;
            }
          }
        }
      }
    } else {
      // ---- a cut piece: parked, or left in the ring if it is this warp's last ----
      const int slot = 2 * warp + (next.x < wx1 ? 0 : 1);
      float* sums = slot & 1 ? reinterpret_cast<float*>(smem + warp * NS * S::STAGE) : a.partial + static_cast<long long>(2 * kMaxCtas + cta * kMaxWarps + warp) * S::SUMS;
      const int pitch = slot & 1 ? S::JROW : D;
      if (slot & 1) __syncwarp();   // every lane has read the last tile
#pragma unroll
      for (int nh = 0; nh < NH; ++nh)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float* row = sums + (nh * 8 + 2 * t4 + h) * pitch;
#pragma unroll
          for (int j = 0; j < MT; ++j) {
            row[16 * j + (I8 ? 2 * g : g)] = o[j][nh][h];
            row[16 * j + (I8 ? 2 * g + 1 : g + 8)] = o[j][nh][2 + h];
          }
          if (g == 0) {
            s_m[slot][nh * 8 + 2 * t4 + h] = m[nh][h];
            s_l[slot][nh * 8 + 2 * t4 + h] = l[nh][h];
          }
        }
      if (lane == 0) s_part[slot] = {cur.seq, cur.hc, tile0, tile0 + count, cur.nt, cur.x - cur.at + cur.lead};
    }

    cur = next;
    if constexpr (S::AHEAD) {
#pragma unroll
      for (int nh = 0; nh < NH; ++nh)
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
          q[nh][ks][0] = qn[nh][ks][0];
          q[nh][ks][1] = qn[nh][ks][1];
        }
    } else {
      if (cur.x < wx1) load_queries(cur, q);
    }
  }

  // ---- the CTA's cut heads, in the order of the list ----
  __syncwarp();
  if (s_part[2 * warp].hc >= 0) {   // the parked sums come back, behind the last piece's
    const float4* src = reinterpret_cast<const float4*>(a.partial + static_cast<long long>(2 * kMaxCtas + cta * kMaxWarps + warp) * S::SUMS);
    unsigned char* dst = smem + warp * NS * S::STAGE + HEADS * S::JROW * 4;
#pragma unroll 8
    for (int i = lane; i < HEADS * (D / 4); i += 32)
      *reinterpret_cast<float4*>(dst + (i / (D / 4) * S::JROW + i % (D / 4) * 4) * 4) = __ldcg(src + i);
  }
  if (tid < 2) s_join[tid] = 0;
  __syncthreads();
  auto finish = [&](int seq, int hc, int row, int col, float4 acc, float top, float sum) {
    const int head = hc / a.chunks, h = head * a.group + (hc - head * a.chunks) * HEADS + row;
    const float inv = inverse(sum);
    *reinterpret_cast<uint2*>(a.out + seq * a.out_stride + static_cast<long long>(h) * D + col) =
        make_uint2(pack_half2(acc.x * inv, acc.y * inv), pack_half2(acc.z * inv, acc.w * inv));
    if (col == 0 && a.lse) a.lse[static_cast<long long>(seq) * a.n_q_heads + h] = log_sum(top, sum);
  };
  auto rows_of = [&](int hc) {
    const int rest = a.group - hc % a.chunks * HEADS;
    return rest < HEADS ? rest : HEADS;
  };
  // lane p looks at part p: which there are, and where another head begins
  Part mine = s_part[lane < 2 * kWarps ? lane : 0];
  if (lane >= 2 * kWarps) mine.hc = -1;
  const unsigned there = __ballot_sync(~0u, mine.hc >= 0);
  const unsigned below = there & ((1u << lane) - 1);
  const int prev = below ? 31 - __clz(below) : lane;
  const int prev_seq = __shfl_sync(~0u, mine.seq, prev), prev_hc = __shfl_sync(~0u, mine.hc, prev);   // (by all lanes, no && between)
  const bool same = below != 0 && prev_seq == mine.seq && prev_hc == mine.hc;
  const unsigned heads = __ballot_sync(~0u, mine.hc >= 0 && !same);
  if (heads == 0) return;
  // heads that go on in other CTAs, in front of this one's run and behind it: their first part
  const int p_first = __ffs(heads) - 1, p_last = 31 - __clz(heads);
  const int first_t0 = __shfl_sync(~0u, mine.t0, p_first), last_t0 = __shfl_sync(~0u, mine.t0, p_last);
  const int last_t1 = __shfl_sync(~0u, mine.t1, 31 - __clz(there)), last_nt = __shfl_sync(~0u, mine.nt, p_last);
  const int open0 = first_t0 ? p_first : -1, open1 = last_t0 == 0 && last_t1 < last_nt ? p_last : -1;
  constexpr int BLOCKS = HEADS * (D / 4) / 32;   // a warp's share of a head's sums at a time
  const int units = __popc(heads) * BLOCKS;
#pragma unroll 1
  for (int unit = warp; unit < units; unit += kWarps) {
    unsigned from_here = heads;
    for (int k = unit / BLOCKS; k; --k) from_here &= from_here - 1;
    const int p0 = __ffs(from_here) - 1;
    const unsigned rest = from_here & (from_here - 1);
    const unsigned parts = there & ~((1u << p0) - 1) & (rest ? (rest & -rest) - 1 : ~0u);
    const int seq = __shfl_sync(~0u, mine.seq, p0), hc = __shfl_sync(~0u, mine.hc, p0), nt = __shfl_sync(~0u, mine.nt, p0);
    const int t0 = __shfl_sync(~0u, mine.t0, p0), t1 = __shfl_sync(~0u, mine.t1, 31 - __clz(parts));
    const int i = unit % BLOCKS * 32 + lane, row = i / (D / 4), col = (i % (D / 4)) * 4;
    if (row >= rows_of(hc)) continue;
    // the parts are the last pieces of some warps, and at most one parked one; all are fetched before any is used
    float pm[kWarps + 1], pl[kWarps + 1];
    float4 v[kWarps + 1];
    const unsigned parked = parts & 0x55555555u;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w <= kWarps; ++w) {
      const bool there_is = w < kWarps ? (parts >> (2 * w + 1)) & 1 : parked != 0;
      const int p = w < kWarps ? 2 * w + 1 : parked ? __ffs(parked) - 1 : 0;
      pm[w] = -INFINITY;
      pl[w] = 0.0f;
      v[w] = make_float4(0, 0, 0, 0);
      if (there_is) {
        pm[w] = s_m[p][row];
        pl[w] = s_l[p][row];
        v[w] = *reinterpret_cast<const float4*>(smem + (p >> 1) * NS * S::STAGE + ((p & 1 ? row : HEADS + row) * S::JROW + col) * 4);
      }
      top = fmaxf(top, pm[w]);
    }
    const float base = top == -INFINITY ? 0.0f : top;
    float4 acc = make_float4(0, 0, 0, 0);
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w <= kWarps; ++w) {
      const float f = exp2_fast(pm[w] - base);
      acc.x += f * v[w].x;
      acc.y += f * v[w].y;
      acc.z += f * v[w].z;
      acc.w += f * v[w].w;
      sum += f * pl[w];
    }
    if (t0 == 0 && t1 == nt) {
      finish(seq, hc, row, col, acc, top, sum);
    } else {
      float* slot = a.partial + static_cast<long long>(2 * cta + (t0 == 0)) * S::SUMS;
      __stcg(reinterpret_cast<float4*>(slot + row * D + col), acc);
      if (col == 0) {
        __stcg(slot + HEADS * D + row, top);
        __stcg(slot + HEADS * D + HEADS + row, sum);
      }
    }
  }
  if (open0 < 0 && open1 < 0) return;   // (the same for every thread)

  // ---- heads that are cut between CTAs c0 .. c1: the last to arrive joins them ----
  __syncthreads();
  if (tid < 2 && (tid ? open1 : open0) >= 0) {
    const Part& p = s_part[tid ? open1 : open0];
    const int c0 = p.begin / run, c1 = (p.begin + p.nt - 1) / run;
    if (arrive(a.counters + c0) == c1 - c0) {
      s_join[tid] = 1;
      s_cta[tid][0] = c0;
      s_cta[tid][1] = c1;
      a.counters[c0] = 0;   // as it was found
    }
  }
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    if (!s_join[k]) continue;
    const Part p = s_part[k ? open1 : open0];
    const int c0 = s_cta[k][0], c1 = s_cta[k][1];
    const int rows = rows_of(p.hc);
    const int n = c1 - c0 + 1;
    float* f_m = reinterpret_cast<float*>(smem);          // [n][rows]: maxima, sums
    float* f_l = f_m + n * rows;
    auto sums_of = [&](int c) { return a.partial + static_cast<long long>(2 * (c0 + c) + (c == 0)) * S::SUMS; };
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < n * rows; i += kThreads) {
      const float* src = sums_of(i / rows) + HEADS * D + i % rows;
      f_m[i] = __ldcg(src);
      f_l[i] = __ldcg(src + HEADS);
    }
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < rows * (D / 4); i += kThreads) {
      const int row = i / (D / 4), col = (i % (D / 4)) * 4;
      constexpr int U = 16;   // partial sums in flight
      float4 acc = make_float4(0, 0, 0, 0);
      float top = -INFINITY, sum = 0.0f;
#pragma unroll 1
      for (int u0 = 0; u0 < n; u0 += U) {
        float4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u0 + u < n) v[u] = __ldcg(reinterpret_cast<const float4*>(sums_of(u0 + u) + row * D + col));
        if (u0 == 0)
#pragma unroll 1
          for (int u = 0; u < n; ++u) top = fmaxf(top, f_m[u * rows + row]);
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (u0 + u < n) {
            const float f = exp2_fast(f_m[(u0 + u) * rows + row] - base);
            acc.x += f * v[u].x;
            acc.y += f * v[u].y;
            acc.z += f * v[u].z;
            acc.w += f * v[u].w;
            sum += f * f_l[(u0 + u) * rows + row];
          }
      }
      finish(p.seq, p.hc, row, col, acc, top, sum);
    }
  }
}

template <int D, bool I8, int NH>
vq_status launch(AttnArgs a, const KvGeometry& g, const KvPool& pool, cudaStream_t s) {
  using S = Shape<D, I8, NH>;
  // What a launch can number: rows of the pool and places of its list in 31 bits.  A list of runs that may cut heads has each head's
  // tiles and kToll; one that gives CTAs of their own to heads (at most kMaxCtas of them then) has a run for each CTA, of up to
  // the longest head's tiles and one, or kWarps if that is more.
  const uint64_t dims[2] = {static_cast<uint64_t>(D), static_cast<uint64_t>(g.n_pages) * g.heads << g.page_shift};
  a.chunks = (a.group + S::HEADS - 1) / S::HEADS;
  const int span = a.window > 0 && a.window < a.max_len ? a.window + S::TT : a.max_len;
  const long long each = (static_cast<long long>(span) + S::TT - 1) / S::TT;   // tiles of a head, as many as there can be
  const long long per_seq = (each + kToll) * a.heads * a.chunks;
  constexpr int kMostTiles = 1 << 21;
  static_assert(static_cast<long long>(kMaxCtas) * (kMostTiles + S::WARPS) <= 0x3fffffff, "runs of a CTA each");
  if (dims[1] > 0x7fffffffu || each > kMostTiles || per_seq > 0x3fffffff) return VQ_ERR_UNSUPPORTED;

  int sms = 0;
  vq_status st = device_sms(&sms);
  if (st != VQ_OK) return st;
  st = device_error_counter(&a.error_flag);
  if (st != VQ_OK) return st;
  static int ready[kMaxDevices] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return VQ_ERR_CUDA;
  auto kernel = attention_kernel<D, I8, NH>;
  if (!__atomic_load_n(&ready[dev], __ATOMIC_ACQUIRE)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(S::SMEM)) != cudaSuccess) return VQ_ERR_CUDA;
    __atomic_store_n(&ready[dev], 1, __ATOMIC_RELEASE);
  }
  // the pools as matrices of tokens; a box is a column block of the tokens that a page and a tile have in common
  while ((1 << a.run_shift) < S::TT && a.run_shift < a.page_shift) ++a.run_shift;
  CUtensorMap maps[2];
  const uint64_t strides[1] = {static_cast<uint64_t>(S::ROW)};
  const uint32_t box[2] = {static_cast<uint32_t>(S::CBB / (I8 ? 1 : 2)), 1u << a.run_shift};
  for (int i = 0; i < 2; ++i) {
    st = encode_tensor_map(&maps[i], i ? pool.v : pool.k, I8 ? 1 : 2, 2, dims, strides, box, S::CBB == 128 ? 2 : 1);
    if (st != VQ_OK) return st;
  }
  // As many sequences at a time as have places below 2^30, by what their table rows (or the window) have room for: with eight heads
  // and tiles of 16 tokens, half a million rows of 4096 tokens (more than a call has), 63 of 2^25.
  const long long seqs = 0x3fffffff / per_seq;
  for (long long from = 0, all = a.n_seqs; from < all; from += seqs) {
    a.n_seqs = static_cast<int>(all - from < seqs ? all - from : seqs);
    const long long most = (each + S::WARPS - 1) / S::WARPS * a.heads * a.chunks * a.n_seqs;   // runs of kWarps tiles
    long long ctas = sms < kMaxCtas ? sms : kMaxCtas;
    if (ctas > most) ctas = most;
    a.inv_grid = 1.0f / static_cast<float>(ctas);
    st = launch_dependent(kernel, dim3(static_cast<unsigned>(ctas)), dim3(S::THREADS), S::SMEM, s, a, maps[0], maps[1]);
    if (st != VQ_OK) return st;
    a.len += a.n_seqs;
    a.table += static_cast<long long>(a.n_seqs) * a.table_stride;
    a.q += a.n_seqs * a.q_stride;
    a.out += a.n_seqs * a.out_stride;
    if (a.lse) a.lse += static_cast<long long>(a.n_seqs) * a.n_q_heads;
  }
  return VQ_OK;
}

template <int D>
vq_status launch_dim(const AttnArgs& a, const KvGeometry& g, const KvPool& pool, cudaStream_t s) {
  if (a.group <= 8) return g.int8 ? launch<D, true, 1>(a, g, pool, s) : launch<D, false, 1>(a, g, pool, s);
  return g.int8 ? launch<D, true, 2>(a, g, pool, s) : launch<D, false, 2>(a, g, pool, s);
}

}  // namespace

bool kv_attention_covers(const KvGeometry& g) {
  return g.dim == 64 || g.dim == 80 || g.dim == 96 || g.dim == 128 || g.dim == 192 || g.dim == 256;
}

// Counters (one per CTA, at the start), two slots of partial sums per CTA, a parking slot per warp.
size_t kv_attention_workspace_bytes(int head_dim) {
  return kMaxCtas * sizeof(int) + static_cast<size_t>(kMaxCtas) * (2 + kMaxWarps) * kMaxHeads * (head_dim + 2) * sizeof(float);
}

vq_status launch_kv_attention(const KvGeometry& g, const KvPool& pool, const KvBooks& books, int n_q_heads, const __half* q,
                              long long q_stride, __half* out, long long out_stride, float* lse, float scale, int window, void* ws,
                              cudaStream_t s) {
  AttnArgs a = {};
  a.run_shift = 3;
  a.ks = pool.ks;
  a.vs = pool.vs;
  a.table = books.table;
  a.len = books.len;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.counters = static_cast<int*>(ws);
  a.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + kMaxCtas * sizeof(int));
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.n_seqs = books.n_seqs;
  a.table_stride = books.table_stride;
  a.max_len = books.max_len;
  a.n_pages = g.n_pages;
  a.page_shift = g.page_shift;
  a.heads = g.heads;
  a.group = n_q_heads / g.heads;
  a.n_q_heads = n_q_heads;
  a.window = window;
  a.scale_log2 = scale * 1.44269504088896341f;
  switch (g.dim) {
    case 64: return launch_dim<64>(a, g, pool, s);
    case 80: return launch_dim<80>(a, g, pool, s);
    case 96: return launch_dim<96>(a, g, pool, s);
    case 128: return launch_dim<128>(a, g, pool, s);
    case 192: return launch_dim<192>(a, g, pool, s);
    case 256: return launch_dim<256>(a, g, pool, s);
  }
  return VQ_ERR_UNSUPPORTED;
}

}  // namespace vq
