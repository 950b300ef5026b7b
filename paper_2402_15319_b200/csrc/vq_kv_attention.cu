// Attention of one new token per sequence over a paged cache (vq_kv_attention).
//
//   out[h] = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale * q_h . k_t - m),  m the running maximum,
// one pass over keys and values (the softmax's maximum and sum run along, accumulators are rescaled when the maximum grows).
//
// Bound by memory: every key and value is read once, 4 * group multiply-adds per pair of stored values, far below what the
// tensor cores need (8 query heads per key/value head at 6.5 TB/s are 0.1 PFLOP/s with the 16-row tile padded).  So the
// products run as mma.sync on 16 x 16 x 8 tiles, the query heads of one key/value head as the rows: no operand passes
// through tensor memory, and the scores stay in the registers that the second product reads.
//
// Split: the tokens of all sequences and key/value heads form one list of tiles (sequence, head, tile); each CTA takes an
// equal run of it, wherever sequences end, so lengths need not be known on the host and ragged batches stay balanced.
// Inside a CTA the warps take tiles in turn, each with its own ring of asynchronous copies: no barrier inside a run.
// A head whose run of tiles is cut between CTAs leaves partial sums (accumulators, maximum, sum) in the workspace; the CTA
// that arrives last joins them in the order of the CTAs, so results do not depend on which one that is.
#include <math.h>

#include "vq_device.cuh"
#include "vq_kv.cuh"

namespace vq {
namespace {

using namespace dev;

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxCtas = 512;           // CTAs of a launch (partial sums and counters are sized for them)
constexpr int kChunkRows = 16;          // query heads that a CTA takes together
// p is held as 2^kLift * exp(...): binary16 pieces of small weights stay normal down to 2^-28 of the largest weight.
constexpr float kLift = 14.0f;

struct AttnArgs {
  const uint8_t* k;
  const uint8_t* v;
  const float* ks;
  const float* vs;
  const int* table;
  const int* len;
  const __half* q;
  __half* out;
  float* lse;
  float* partial;
  int* counters;
  long long q_stride, out_stride;
  int n_seqs, table_stride, max_len, n_pages, page_shift, heads, group, chunks, n_q_heads, window;
  float scale_log2;
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float log2_fast(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool on) {
  const int bytes = on ? 16 : 0;   // 0: zeros, nothing is read
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
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

// Shapes of one instantiation.
template <int D, bool I8>
struct Shape {
  static constexpr int ROW = D * (I8 ? 1 : 2);          // bytes of one token
  static constexpr int CH = ROW / 16;                   // 16-byte pieces of one token
  static constexpr int PITCH = (CH | 1) * 16;           // odd in pieces: eight rows of a matrix lie in different banks
  // tokens per tile: a stage of a warp holds about 8 KB of keys and values
  static constexpr int R = I8 ? (ROW <= 64 ? 4 : 2) : (ROW <= 128 ? 2 : 1);
  static constexpr int TT = 16 * R;
  static constexpr int HALVES = TT / 8;                 // runs of 8 tokens: never across a page
  static constexpr int KV = TT * PITCH;
  static constexpr int STAGE = 2 * KV + (I8 ? 2 * TT * 4 : 0);
  static constexpr int CTAS = 3 * kWarps * STAGE + 2048 <= 113 * 1024 ? 2 : 1;   // resident per SM
  static constexpr int FIT = ((CTAS == 2 ? 113 : 226) * 1024 - 2048) / (kWarps * STAGE);
  static constexpr int NS = FIT > 6 ? 6 : FIT;          // stages of a warp's ring
  static constexpr size_t JOIN = static_cast<size_t>(kWarps) * kChunkRows * (D + 2) * 4;   // (reuses the rings)
  static constexpr size_t SMEM = static_cast<size_t>(kWarps) * NS * STAGE > JOIN ? static_cast<size_t>(kWarps) * NS * STAGE : JOIN;
  static_assert(NS >= 2, "a ring needs two stages");
};

// Tiles of sequence of length n: those that hold a token of the window.
__device__ __forceinline__ int first_token(const AttnArgs& a, int n) { return a.window > 0 && n > a.window ? n - a.window : 0; }
template <int TT>
__device__ __forceinline__ int tile_count(const AttnArgs& a, int n) {
  return n <= 0 ? 0 : (n - 1) / TT - first_token(a, n) / TT + 1;
}
__device__ __forceinline__ int clamp_len(const AttnArgs& a, int n) { return n < 0 ? 0 : n > a.max_len ? a.max_len : n; }

template <int D, bool I8, int ROWS>
__global__ void __launch_bounds__(kThreads, Shape<D, I8>::CTAS) attention_kernel(AttnArgs a) {
  using S = Shape<D, I8>;
  constexpr int TT = S::TT, R = S::R, NT = 2 * R, HALVES = S::HALVES, NS = S::NS;
  constexpr int KSTEPS = D / 16;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ int s_len[kThreads];
  __shared__ long long s_scan[kWarps + 1];
  __shared__ int s_bad[kWarps][NS];
  __shared__ int s_last;
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  const int hc_count = a.heads * a.chunks;

  // ---- the list of tiles: total, then this CTA's run ----
  long long total = 0;
  for (int base = 0; base < a.n_seqs; base += kThreads) {
    const int s = base + tid;
    const int n = s < a.n_seqs ? clamp_len(a, __ldcg(a.len + s)) : 0;
    if (s < a.n_seqs && n == 0 && s % static_cast<int>(gridDim.x) == static_cast<int>(blockIdx.x)) {   // nothing to attend to
      for (int i = 0; i < a.n_q_heads * D / 8; ++i) *reinterpret_cast<uint4*>(a.out + s * a.out_stride + i * 8) = make_uint4(0, 0, 0, 0);
      if (a.lse)
        for (int h = 0; h < a.n_q_heads; ++h) a.lse[static_cast<long long>(s) * a.n_q_heads + h] = -INFINITY;
    }
    total += static_cast<long long>(tile_count<TT>(a, n)) * hc_count;
  }
  for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(~0u, total, o);
  if (lane == 0) s_scan[warp] = total;
  __syncthreads();
  total = 0;
  for (int w = 0; w < kWarps; ++w) total += s_scan[w];
  if (total == 0) return;
  // a CTA per kWarps tiles at most: below that the join costs more than the split saves
  const long long want = (total + kWarps - 1) / kWarps;
  const int ctas = static_cast<int>(want < gridDim.x ? want : gridDim.x);
  const int cta = blockIdx.x;
  if (cta >= ctas) return;
  const long long x0 = cta * total / ctas, x1 = (cta + 1) * total / ctas;

  // sequence that x0 lies in
  int seq = 0, chunk_base = 0;
  long long at = 0;   // tiles in front of `seq`
  for (;; chunk_base += kThreads) {
    const int s = chunk_base + tid;
    const int n = s < a.n_seqs ? clamp_len(a, __ldcg(a.len + s)) : 0;
    __syncthreads();
    s_len[tid] = n;
    const long long mine = static_cast<long long>(tile_count<TT>(a, n)) * hc_count;
    long long incl = mine;
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(~0u, incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    long long before = at, chunk = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) before += s_scan[w];
      chunk += s_scan[w];
    }
    const bool here = x0 >= before + incl - mine && x0 < before + incl;
    __syncthreads();
    if (here) {
      s_last = tid;
      s_scan[kWarps] = before + incl - mine;
    }
    __syncthreads();
    if (x0 < at + chunk) {
      seq = chunk_base + s_last;
      at = s_scan[kWarps];
      break;
    }
    at += chunk;
    if (chunk_base + kThreads >= a.n_seqs) return;   // lengths that change under the call: no run to take
  }

  const uint32_t ring = smem_u32(smem) + warp * NS * S::STAGE;
  long long x = x0;
  while (x < x1) {
    // ---- one piece: tiles [tile0, tile0 + count) of (seq, hc) ----
    const int n = s_len[seq - chunk_base];
    const int begin = first_token(a, n);
    const int nt = tile_count<TT>(a, n);
    const long long idx = x - at;
    const int hc = static_cast<int>(idx / nt), tile0 = static_cast<int>(idx % nt);
    const int count = static_cast<int>(x1 - x < nt - tile0 ? x1 - x : nt - tile0);
    const int head = hc / a.chunks, q0 = (hc % a.chunks) * kChunkRows;
    const int rows = a.group - q0 < kChunkRows ? a.group - q0 : kChunkRows;
    const int qh = head * a.group + q0;
    const int base_tok = (begin / TT + tile0) * TT;
    const int mine = count > warp ? (count - warp + kWarps - 1) / kWarps : 0;   // this warp's tiles: warp, warp + kWarps, ...
    const int* table = a.table + static_cast<long long>(seq) * a.table_stride;

    // pages of the next 32 runs of 8 tokens, one per lane
    int pages = 0, pages_from = 0;
    auto load_pages = [&](int from) {
      const int i = from + lane / HALVES;
      const int tok = base_tok + (warp + i * kWarps) * TT + (lane % HALVES) * 8;
      pages = i < mine && tok < n ? __ldcg(table + (tok >> a.page_shift)) : -1;
      pages_from = from;
    };
    auto issue = [&](int i) {
      if (i < mine) {
        if (i - pages_from >= 32 / HALVES) load_pages(i);
        const int slot = i % NS;
        const uint32_t stage = ring + slot * S::STAGE;
        const int tok0 = base_tok + (warp + i * kWarps) * TT;
        const int from = (i - pages_from) * HALVES;
        const unsigned bad = __ballot_sync(~0u, static_cast<unsigned>(pages) >= static_cast<unsigned>(a.n_pages));
        if (lane == 0) s_bad[warp][slot] = (bad >> from) & ((1u << HALVES) - 1);
        const int mask = (1 << a.page_shift) - 1;
#pragma unroll
        for (int c0 = 0; c0 < TT * S::CH; c0 += 32) {
          const int c = c0 + lane, row = c / S::CH, col = c % S::CH, tok = tok0 + row;
          const int page = __shfl_sync(~0u, pages, from + (row >> 3));
          if (TT * S::CH % 32 == 0 || c < TT * S::CH) {
            const bool on = tok >= begin && tok < n && static_cast<unsigned>(page) < static_cast<unsigned>(a.n_pages);
            const long long off = on ? (((static_cast<long long>(page) * a.heads + head) << a.page_shift) + (tok & mask)) * S::ROW + col * 16 : 0;
            cp_async16(stage + row * S::PITCH + col * 16, a.k + off, on);
            cp_async16(stage + S::KV + row * S::PITCH + col * 16, a.v + off, on);
          }
        }
        if (I8) {   // scales, four tokens to a piece
          const int j = lane % (TT / 4), tok = tok0 + 4 * j;
          const int page = __shfl_sync(~0u, pages, from + (j >> 1));
          const bool on = static_cast<unsigned>(page) < static_cast<unsigned>(a.n_pages);
          const long long off = on ? ((static_cast<long long>(page) * a.heads + head) << a.page_shift) + (tok & mask) : 0;
          if (lane < 2 * (TT / 4)) cp_async16(stage + 2 * S::KV + lane * 16, (lane < TT / 4 ? a.ks : a.vs) + off, on);
        }
      }
      cp_async_commit();
    };

    load_pages(0);
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) issue(i);

    // queries: rows g and g + 8 of the A operand.  8-bit keys come four dimensions to a register, so the reduction slots of
    // a step are filled in that order: slots 2t, 2t+1, 2t+8, 2t+9 hold dimensions 4t .. 4t+3.
    uint32_t qa[KSTEPS][ROWS == 16 ? 4 : 2];
    {
      const __half* qrow = a.q + seq * a.q_stride + static_cast<long long>(qh) * D;
#pragma unroll
      for (int r = 0; r < ROWS / 8; ++r) {
        const bool on = g + 8 * r < rows;
        const __half* p = qrow + (g + 8 * r) * D;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) {
          uint32_t lo = 0, hi = 0;
          if (on) {
            if (I8) {
              const uint2 w = __ldcg(reinterpret_cast<const uint2*>(p + ks * 16 + 4 * t4));
              lo = w.x;
              hi = w.y;
            } else {
              lo = __ldcg(reinterpret_cast<const unsigned int*>(p + ks * 16 + 2 * t4));
              hi = __ldcg(reinterpret_cast<const unsigned int*>(p + ks * 16 + 8 + 2 * t4));
            }
          }
          qa[ks][r] = lo;
          qa[ks][ROWS / 8 + r] = hi;
        }
      }
    }

    float o[D / 8][4];
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < D / 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[j][e] = 0.0f;

    for (int i = 0; i < mine; ++i) {
      cp_async_wait<NS - 2>();
      __syncwarp();   // the tile is there, and every lane is done with the tile before it: its stage is free
      issue(i + NS - 1);
      const int slot = i % NS;
      const uint32_t stage = ring + slot * S::STAGE;
      const int tok0 = base_tok + (warp + i * kWarps) * TT;
      const int bad = s_bad[warp][slot];

      // scores
      float sc[NT][4];
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[j][e] = 0.0f;
      if (I8) {
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
          for (int r = 0; r < R / 2; ++r) {
            uint32_t b[4];
            ldmatrix4(b, stage + (r * 32 + lane) * S::PITCH + ks * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t u = b[e] ^ 0x80808080u;
              mma16816(sc[4 * r + e], qa[ks][0], ROWS == 16 ? qa[ks][1] : 0u, qa[ks][ROWS / 8], ROWS == 16 ? qa[ks][ROWS / 8 + 1] : 0u,
                       bytes_to_half2<0x4140>(u), bytes_to_half2<0x4342>(u));
            }
          }
      } else {
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
          for (int r = 0; r < R; ++r) {
            uint32_t b[4];
            ldmatrix4(b, stage + (r * 16 + (lane & 7) + ((lane >> 4) << 3)) * S::PITCH + (2 * ks + ((lane >> 3) & 1)) * 16);
            mma16816(sc[2 * r], qa[ks][0], ROWS == 16 ? qa[ks][1] : 0u, qa[ks][ROWS / 8], ROWS == 16 ? qa[ks][ROWS / 8 + 1] : 0u, b[0], b[1]);
            mma16816(sc[2 * r + 1], qa[ks][0], ROWS == 16 ? qa[ks][1] : 0u, qa[ks][ROWS / 8], ROWS == 16 ? qa[ks][ROWS / 8 + 1] : 0u, b[2], b[3]);
          }
      }

      // Scale.  8-bit values are multiplied as integers: the weight of token t carries its value scale, 2^(s + log2 scale_v),
      // and the maximum is taken of that exponent, so that the largest weight is 1 whatever the scales are.
      float lv[NT][2];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        float k0 = a.scale_log2, k1 = a.scale_log2;
        if (I8) {
          const float2 kk = *reinterpret_cast<const float2*>(smem + (stage - smem_u32(smem)) + 2 * S::KV + (8 * j + 2 * t4) * 4);
          const float2 vv = *reinterpret_cast<const float2*>(smem + (stage - smem_u32(smem)) + 2 * S::KV + TT * 4 + (8 * j + 2 * t4) * 4);
          k0 *= kk.x;
          k1 *= kk.y;
          lv[j][0] = fmaxf(log2_fast(vv.x), -40.0f);   // (a scale of 0 goes with integers of 0)
          lv[j][1] = fmaxf(log2_fast(vv.y), -40.0f);
          if (vv.x != vv.x) lv[j][0] = vv.x;           // (fmaxf drops a NaN)
          if (vv.y != vv.y) lv[j][1] = vv.y;
        } else {
          lv[j][0] = lv[j][1] = 0.0f;
        }
        sc[j][0] *= k0;
        sc[j][1] *= k1;
        sc[j][2] *= k0;
        sc[j][3] *= k1;
      }
      if (tok0 < begin || tok0 + TT > n || bad) {   // tokens that do not take part
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int tok = tok0 + 8 * j + 2 * t4 + e;
            if (tok < begin || tok >= n || ((bad >> j) & 1)) {
              sc[j][e] = sc[j][2 + e] = -INFINITY;
              lv[j][e] = 0.0f;
            }
          }
      }

      // running maximum, weights
      uint32_t ph[NT][ROWS / 8], pl[NT][ROWS / 8];
      float alpha[2] = {1.0f, 1.0f};
#pragma unroll
      for (int r = 0; r < ROWS / 8; ++r) {
        float top = m[r];
#pragma unroll
        for (int j = 0; j < NT; ++j) top = fmaxf(top, fmaxf(sc[j][2 * r] + lv[j][0], sc[j][2 * r + 1] + lv[j][1]));
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
        top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
        const float base = (top == -INFINITY ? 0.0f : top) - kLift;
        alpha[r] = exp2_fast(m[r] - kLift - base);
        m[r] = top;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const float e0 = sc[j][2 * r] - base, e1 = sc[j][2 * r + 1] - base;
          float p0 = exp2_fast(e0), p1 = exp2_fast(e1);
          sum += p0 + p1;
          if (I8) {
            p0 = exp2_fast(e0 + lv[j][0]);
            p1 = exp2_fast(e1 + lv[j][1]);
          }
          // a weight is the sum of two binary16 numbers: 22 significant bits reach the product
          ph[j][r] = pack_half2(p0, p1);
          const float2 back = unpack_half2(ph[j][r]);
          pl[j][r] = pack_half2(p0 - back.x, p1 - back.y);
        }
        l[r] = l[r] * alpha[r] + sum;
      }
      if (__any_sync(~0u, alpha[0] != 1.0f || alpha[1] != 1.0f)) {
#pragma unroll
        for (int j = 0; j < D / 8; ++j) {
          o[j][0] *= alpha[0];
          o[j][1] *= alpha[0];
          if (ROWS == 16) {
            o[j][2] *= alpha[1];
            o[j][3] *= alpha[1];
          }
        }
      }

      // values
      auto weigh = [&](float (&acc)[4], int r, uint32_t b0, uint32_t b1) {
        mma16816(acc, ph[2 * r][0], ROWS == 16 ? ph[2 * r][ROWS / 8 - 1] : 0u, ph[2 * r + 1][0], ROWS == 16 ? ph[2 * r + 1][ROWS / 8 - 1] : 0u, b0, b1);
        mma16816(acc, pl[2 * r][0], ROWS == 16 ? pl[2 * r][ROWS / 8 - 1] : 0u, pl[2 * r + 1][0], ROWS == 16 ? pl[2 * r + 1][ROWS / 8 - 1] : 0u, b0, b1);
      };
      if (I8) {
        // a transposed matrix gives a lane two adjacent dimensions of two tokens: even and odd dimensions are tiles of their own
#pragma unroll
        for (int c = 0; c < S::CH; ++c)
#pragma unroll
          for (int r = 0; r < R / 2; ++r) {
            uint32_t b[4];
            ldmatrix4_trans(b, stage + S::KV + (r * 32 + lane) * S::PITCH + c * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] ^= 0x80808080u;
            weigh(o[2 * c], 2 * r, bytes_to_half2<0x4240>(b[0]), bytes_to_half2<0x4240>(b[1]));
            weigh(o[2 * c + 1], 2 * r, bytes_to_half2<0x4341>(b[0]), bytes_to_half2<0x4341>(b[1]));
            weigh(o[2 * c], 2 * r + 1, bytes_to_half2<0x4240>(b[2]), bytes_to_half2<0x4240>(b[3]));
            weigh(o[2 * c + 1], 2 * r + 1, bytes_to_half2<0x4341>(b[2]), bytes_to_half2<0x4341>(b[3]));
          }
      } else {
#pragma unroll
        for (int c = 0; c < D / 8; c += 2)
#pragma unroll
          for (int r = 0; r < R; ++r) {
            uint32_t b[4];
            ldmatrix4_trans(b, stage + S::KV + (r * 16 + (lane & 15)) * S::PITCH + (c + (lane >> 4)) * 16);
            weigh(o[c], r, b[0], b[1]);
            weigh(o[c + 1], r, b[2], b[3]);
          }
      }
    }
    cp_async_wait<0>();

    // ---- the warps' sums, joined in shared memory ----
#pragma unroll
    for (int r = 0; r < ROWS / 8; ++r) {
      l[r] += __shfl_xor_sync(~0u, l[r], 1);
      l[r] += __shfl_xor_sync(~0u, l[r], 2);
    }
    __syncthreads();
    float* join = reinterpret_cast<float*>(smem);                        // [warp][row][D]
    float* jm = join + kWarps * kChunkRows * D;                          // [warp][row]: maximum, then sum
    float* jl = jm + kWarps * kChunkRows;
#pragma unroll
    for (int r = 0; r < ROWS / 8; ++r) {
      float* row = join + (warp * kChunkRows + g + 8 * r) * D;
      if (I8) {
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
          *reinterpret_cast<float4*>(row + 16 * c + 4 * t4) = make_float4(o[2 * c][2 * r], o[2 * c + 1][2 * r], o[2 * c][2 * r + 1], o[2 * c + 1][2 * r + 1]);
      } else {
#pragma unroll
        for (int j = 0; j < D / 8; ++j) *reinterpret_cast<float2*>(row + 8 * j + 2 * t4) = make_float2(o[j][2 * r], o[j][2 * r + 1]);
      }
      if (t4 == 0) {
        jm[warp * kChunkRows + g + 8 * r] = m[r];
        jl[warp * kChunkRows + g + 8 * r] = l[r];
      }
    }
    __syncthreads();

    const bool whole = count == nt;
    const long long seg0 = x - tile0, seg1 = seg0 + nt;   // the head's run in the list
    constexpr int SLOT = kChunkRows * (D + 2);
    float* slot = a.partial + static_cast<long long>(2 * cta + (tile0 == 0 ? 1 : 0)) * SLOT;
    for (int i = tid; i < rows * (D / 4); i += kThreads) {
      const int row = i / (D / 4), col = (i % (D / 4)) * 4;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, jm[w * kChunkRows + row]);
      const float base = top == -INFINITY ? 0.0f : top;
      float4 acc = make_float4(0, 0, 0, 0);
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2_fast(jm[w * kChunkRows + row] - base);
        const float4 v = *reinterpret_cast<const float4*>(join + (w * kChunkRows + row) * D + col);
        acc.x += f * v.x;
        acc.y += f * v.y;
        acc.z += f * v.z;
        acc.w += f * v.w;
        sum += f * jl[w * kChunkRows + row];
      }
      if (whole) {
        const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
        uint2 h = make_uint2(pack_half2(acc.x * inv, acc.y * inv), pack_half2(acc.z * inv, acc.w * inv));
        *reinterpret_cast<uint2*>(a.out + seq * a.out_stride + static_cast<long long>(qh + row) * D + col) = h;
        if (col == 0 && a.lse) a.lse[static_cast<long long>(seq) * a.n_q_heads + qh + row] = (base - kLift + log2f(sum)) * 0.693147180559945309f;
      } else {
        *reinterpret_cast<float4*>(slot + row * D + col) = acc;
        if (col == 0) {
          slot[kChunkRows * D + row] = top;
          slot[kChunkRows * D + kChunkRows + row] = sum;
        }
      }
    }
    if (!whole) {
      const int c0 = static_cast<int>(((seg0 + 1) * ctas - 1) / total), c1 = static_cast<int>((seg1 * ctas - 1) / total);
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        const int arrived = atomicAdd(a.counters + c0, 1);
        s_last = arrived == c1 - c0;
        if (s_last) a.counters[c0] = 0;   // as it was found
      }
      __syncthreads();
      if (s_last) {
        __threadfence();
        for (int i = tid; i < rows * (D / 4); i += kThreads) {
          const int row = i / (D / 4), col = (i % (D / 4)) * 4;
          float top = -INFINITY;
          for (int c = c0; c <= c1; ++c)
            top = fmaxf(top, __ldcg(a.partial + static_cast<long long>(2 * c + (c == c0)) * SLOT + kChunkRows * D + row));
          const float base = top == -INFINITY ? 0.0f : top;
          float4 acc = make_float4(0, 0, 0, 0);
          float sum = 0.0f;
          for (int c = c0; c <= c1; ++c) {
            const float* p = a.partial + static_cast<long long>(2 * c + (c == c0)) * SLOT;
            const float f = exp2_fast(__ldcg(p + kChunkRows * D + row) - base);
            const float4 v = __ldcg(reinterpret_cast<const float4*>(p + row * D + col));
            acc.x += f * v.x;
            acc.y += f * v.y;
            acc.z += f * v.z;
            acc.w += f * v.w;
            sum += f * __ldcg(p + kChunkRows * D + kChunkRows + row);
          }
          const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
          uint2 h = make_uint2(pack_half2(acc.x * inv, acc.y * inv), pack_half2(acc.z * inv, acc.w * inv));
          *reinterpret_cast<uint2*>(a.out + seq * a.out_stride + static_cast<long long>(qh + row) * D + col) = h;
          if (col == 0 && a.lse) a.lse[static_cast<long long>(seq) * a.n_q_heads + qh + row] = (base - kLift + log2f(sum)) * 0.693147180559945309f;
        }
      }
    }
    __syncthreads();   // the join's memory is the rings' again, s_last is free

    // ---- next piece ----
    x += count;
    if (x < x1 && x == at + static_cast<long long>(nt) * hc_count) {
      at = x;
      do {
        if (++seq >= a.n_seqs) return;   // (as above)
        if (seq - chunk_base >= kThreads) {
          chunk_base += kThreads;
          __syncthreads();
          s_len[tid] = chunk_base + tid < a.n_seqs ? clamp_len(a, __ldcg(a.len + chunk_base + tid)) : 0;
          __syncthreads();
        }
      } while (s_len[seq - chunk_base] == 0);
    }
  }
}

template <int D, bool I8, int ROWS>
vq_status launch(const AttnArgs& a, int sms, long long tiles, cudaStream_t s) {
  using S = Shape<D, I8>;
  static int ready[kMaxDevices] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return VQ_ERR_CUDA;
  auto kernel = attention_kernel<D, I8, ROWS>;
  if (!__atomic_load_n(&ready[dev], __ATOMIC_ACQUIRE)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(S::SMEM)) != cudaSuccess) return VQ_ERR_CUDA;
    __atomic_store_n(&ready[dev], 1, __ATOMIC_RELEASE);
  }
  long long ctas = static_cast<long long>(sms) * S::CTAS;
  if (ctas > kMaxCtas) ctas = kMaxCtas;
  const long long most = (tiles + kWarps - 1) / kWarps;   // tiles: as many as there can be
  if (ctas > most) ctas = most;
  return launch_dependent(kernel, dim3(static_cast<unsigned>(ctas)), dim3(kThreads), S::SMEM, s, a);
}

template <int D>
vq_status launch_dim(const AttnArgs& a, bool int8, int sms, cudaStream_t s) {
  const int tt = int8 ? Shape<D, true>::TT : Shape<D, false>::TT;
  const int span = a.window > 0 && a.window < a.max_len ? a.window + tt : a.max_len;
  const long long tiles = (static_cast<long long>(span) + tt - 1) / tt * a.heads * a.chunks * a.n_seqs;
  if (a.group <= 8) return int8 ? launch<D, true, 8>(a, sms, tiles, s) : launch<D, false, 8>(a, sms, tiles, s);
  return int8 ? launch<D, true, 16>(a, sms, tiles, s) : launch<D, false, 16>(a, sms, tiles, s);
}

}  // namespace

bool kv_attention_covers(const KvGeometry& g) {
  return g.dim == 64 || g.dim == 80 || g.dim == 96 || g.dim == 128 || g.dim == 192 || g.dim == 256;
}

// Counters (one per CTA, at the start), then two slots of partial sums per CTA.
size_t kv_attention_workspace_bytes(int head_dim) {
  return kMaxCtas * sizeof(int) + static_cast<size_t>(kMaxCtas) * 2 * kChunkRows * (head_dim + 2) * sizeof(float);
}

vq_status launch_kv_attention(const KvGeometry& g, const KvPool& pool, const KvBooks& books, int n_q_heads, const __half* q,
                              long long q_stride, __half* out, long long out_stride, float* lse, float scale, int window, void* ws,
                              cudaStream_t s) {
  int sms = 0;
  const vq_status st = device_sms(&sms);
  if (st != VQ_OK) return st;
  AttnArgs a = {};
  a.k = pool.k;
  a.v = pool.v;
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
  a.chunks = (a.group + kChunkRows - 1) / kChunkRows;
  a.n_q_heads = n_q_heads;
  a.window = window;
  a.scale_log2 = scale * 1.44269504088896341f;
  switch (g.dim) {
    case 64: return launch_dim<64>(a, g.int8, sms, s);
    case 80: return launch_dim<80>(a, g.int8, sms, s);
    case 96: return launch_dim<96>(a, g.int8, sms, s);
    case 128: return launch_dim<128>(a, g.int8, sms, s);
    case 192: return launch_dim<192>(a, g.int8, sms, s);
    case 256: return launch_dim<256>(a, g.int8, sms, s);
  }
  return VQ_ERR_UNSUPPORTED;
}

}  // namespace vq
