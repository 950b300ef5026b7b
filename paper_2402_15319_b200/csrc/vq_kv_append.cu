// New tokens into the paged cache (vq_kv_append): queries and keys rotated, keys and values written to their pages.
//
//   (a, b) -> (a cos - b sin, b cos + a sin),   8-bit rows: scale = max|x| / 127, integer = rint(127 x / max|x|).
//
// Bound by memory: every row is read once and written once.  A CTA serves one token, or (few tokens) a share of one's heads,
// so the token's cosines and sines are fetched once per thread and used for all of them.  A group of LG lanes holds a head's row:
// a lane two 16-byte pieces, the two halves of the pairs that it turns, so that nothing crosses lanes but the 8-bit
// row's maximum.
// 8192 tokens, 64/8 heads of 128: 57.5 us into 8-bit pages, 58 into binary16 ones = 5.8 TB/s; a token each of 16 sequences: 2.0 us.
#include "vq_device.cuh"
#include "vq_kv.cuh"

namespace vq {
namespace {

using namespace dev;

constexpr int kAppendThreads = 128;   // of a CTA at most

struct AppendArgs {
  KvGeometry g;
  KvPool pool;
  KvBooks books;
  KvRotary rot;
  const int* starts;
  const __half* k;
  const __half* v;
  long long k_stride, v_stride;
};

// Sequence of token row `token`: the first s with starts[s + 1] > token, or n_seqs.  32 places a step, by a whole warp.
__device__ __forceinline__ int sequence_of(const int* starts, int n_seqs, int token, int lane) {
  int lo = 0, hi = n_seqs;   // the answer lies in lo .. hi
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32;
    const int at = lo + lane * step;
    const unsigned above = __ballot_sync(~0u, at >= hi || __ldcg(starts + at + 1) > token);
    const int first = above ? __ffs(above) - 1 : 32;   // places lo .. lo + (first - 1) * step are not above
    const int next_hi = first < 32 && lo + first * step < hi ? lo + first * step : hi;
    if (first > 0) lo = lo + (first - 1) * step + 1;
    hi = next_hi;
  }
  return lo;
}

__device__ __forceinline__ void unpack8(uint4 w, float (&x)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ void store8(__half* p, const float (&x)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
    u[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}

template <bool I8, int LG>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(AppendArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, token = blockIdx.x;
  // this lane's two pieces of eight dimensions
  const int p = threadIdx.x % LG, pairs = a.g.dim / 16, turned = a.rot.cs ? a.rot.rot_dim / 16 : 0;
  const bool act = p < pairs, turn = p < turned;
  int d0 = 16 * p, d1 = 16 * p + 8;
  if (turn && !a.rot.interleaved) {
    d0 = 8 * p;
    d1 = 8 * (p + turned);
  }
  const int heads = a.rot.n_q_heads + 2 * a.g.heads;
  const int STEP = blockDim.x / LG;
  const int rounds = (heads + STEP - 1) / STEP;   // (every lane takes part in every round's shuffles)
  // a round's rows, requested a round ahead: the first ones before it is known where they go
  uint4 raw[2];
  auto request = [&](int round) {
    const int h = round * STEP + threadIdx.x / LG;
    raw[0] = raw[1] = make_uint4(0, 0, 0, 0);
    if (h >= heads || !act) return;
    const int kv = h - a.rot.n_q_heads;
    const __half* src = kv < 0 ? a.rot.q + token * a.rot.q_stride + static_cast<long long>(h) * a.g.dim
                      : kv < a.g.heads ? a.k + token * a.k_stride + static_cast<long long>(kv) * a.g.dim
                                       : a.v + token * a.v_stride + static_cast<long long>(kv - a.g.heads) * a.g.dim;
    raw[0] = __ldcg(reinterpret_cast<const uint4*>(src + d0));
    raw[1] = __ldcg(reinterpret_cast<const uint4*>(src + d1));
  };
  request(blockIdx.y);
  int seq = token, start = token, end = token + 1;
  if (a.starts) {
    seq = sequence_of(a.starts, a.books.n_seqs, token, lane);
    if (seq >= a.books.n_seqs) return;   // behind the last sequence
    start = __ldcg(a.starts + seq);
    end = __ldcg(a.starts + seq + 1);
  }
  int len = __ldcg(a.books.len + seq);
  len = len < 0 ? 0 : len > a.books.max_len ? a.books.max_len : len;
  const long long pos64 = static_cast<long long>(len) - end + token;   // the last of the new tokens is the sequence's last
  if (token < start || pos64 < 0 || pos64 >= len) return;
  const int pos = static_cast<int>(pos64);
  const int page = __ldcg(a.books.table + static_cast<long long>(seq) * a.books.table_stride + (pos >> a.g.page_shift));
  const bool on_page = static_cast<unsigned>(page) < static_cast<unsigned>(a.g.n_pages);
  const long long slot = ((static_cast<long long>(page) * a.g.heads) << a.g.page_shift) + (pos & (a.g.page_tokens - 1));

  // what turns this lane's pieces
  float cs[8], sn[8];
  if (turn) {
    const float4* row = reinterpret_cast<const float4*>(a.rot.cs + static_cast<long long>(pos) * (a.rot.rot_dim / 2) + 8 * p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 f = __ldcg(row + i);
      cs[2 * i] = f.x;
      sn[2 * i] = f.y;
      cs[2 * i + 1] = f.z;
      sn[2 * i + 1] = f.w;
    }
  }
  auto rotate = [&](float (&x)[8], float (&y)[8]) {
    if (!a.rot.interleaved) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = x[i], w = y[i];
        x[i] = u * cs[i] - w * sn[i];
        y[i] = w * cs[i] + u * sn[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float u = x[2 * i], w = x[2 * i + 1], u2 = y[2 * i], w2 = y[2 * i + 1];
        x[2 * i] = u * cs[i] - w * sn[i];
        x[2 * i + 1] = w * cs[i] + u * sn[i];
        y[2 * i] = u2 * cs[4 + i] - w2 * sn[4 + i];
        y[2 * i + 1] = w2 * cs[4 + i] + u2 * sn[4 + i];
      }
    }
  };

  for (int round = blockIdx.y; round < rounds; round += gridDim.y) {
    const int h = round * STEP + threadIdx.x / LG;
    const bool mine = h < heads && act;
    const int kv = h - a.rot.n_q_heads;             // < 0: a query head
    const bool value = kv >= a.g.heads;
    const int head = value ? kv - a.g.heads : kv;
    float x[8], y[8];
    unpack8(raw[0], x);
    unpack8(raw[1], y);
    if (round + static_cast<int>(gridDim.y) < rounds) request(round + gridDim.y);
    if (turn && !value) rotate(x, y);
    if (kv < 0) {
      if (mine) {
        __half* dst = a.rot.q_out + token * a.rot.q_out_stride + static_cast<long long>(h) * a.g.dim;
        store8(dst + d0, x);
        store8(dst + d1, y);
      }
    }
    const long long at = slot + (static_cast<long long>(head) << a.g.page_shift);   // row of the pool
    if (I8) {
      // largest magnitude as an unsigned integer: infinities and NaN come out on top
      unsigned top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
        top = max(top, __float_as_uint(y[i]) & 0x7fffffffu);
      }
#pragma unroll
      for (int o = LG / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
      if (mine && kv >= 0 && on_page) {
        const float most = __uint_as_float(top), scale = __fdiv_rn(most, 127.0f);
        uint32_t w[4] = {0, 0, 0, 0};
        if (most >= 0x1p-118f) {   // (below that, which no binary16 row is but by a table of such cosines, the reciprocal ends: zeros)
          // 127 / 128 x of a binary16 value is exact in binary32, and the quotient is rounded once (a rounded reciprocal, then one
          // step with the exact remainder: Markstein's theorem), so a row that is not rotated gets the nearest integers always,
          // ties (one value in 2000) to even.  x / scale by the rounded reciprocal alone was one off in 1.1e-4 of them.
          const float whole = most * 0.0078125f, inv = __frcp_rn(whole);
          auto nearest = [&](float v) {   // low byte: between -127 and 127, as |v| <= most; 1.5 * 2^23 leaves no place behind the point
            const float part = v * 0.9921875f, q = part * inv;
            return __float_as_uint(fmaf(fmaf(-q, whole, part), inv, q) + 12582912.0f);
          };
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            w[i] = prmt(prmt(nearest(x[4 * i]), nearest(x[4 * i + 1]), 0x0040), prmt(nearest(x[4 * i + 2]), nearest(x[4 * i + 3]), 0x0040), 0x5410);
            w[2 + i] = prmt(prmt(nearest(y[4 * i]), nearest(y[4 * i + 1]), 0x0040), prmt(nearest(y[4 * i + 2]), nearest(y[4 * i + 3]), 0x0040), 0x5410);
          }
        }
        uint8_t* dst = (value ? a.pool.v : a.pool.k) + at * a.g.dim;
        *reinterpret_cast<uint2*>(dst + d0) = make_uint2(w[0], w[1]);
        *reinterpret_cast<uint2*>(dst + d1) = make_uint2(w[2], w[3]);
        if (p == 0) (value ? a.pool.vs : a.pool.ks)[at] = top >= 0x7f800000u ? __uint_as_float(0x7fffffffu) : scale;
      }
    } else if (mine && kv >= 0 && on_page) {
      __half* dst = reinterpret_cast<__half*>(value ? a.pool.v : a.pool.k) + at * a.g.dim;
      store8(dst + d0, x);
      store8(dst + d1, y);
    }
  }
}

template <bool I8>
vq_status launch(const AppendArgs& a, int n_tokens, int sms, cudaStream_t s) {
  const int lg = a.g.dim <= 64 ? 4 : a.g.dim <= 128 ? 8 : 16, lanes = (a.rot.n_q_heads + 2 * a.g.heads) * lg;
  // A token's rows wait for a chain of reads (its sequence, length, page), so many tokens want small CTAs, more of them on an SM
  // (8192 tokens of 80 heads of 128 into 8-bit pages with 128 / 64 / 32 threads: 62 / 58 / 57 us, of 16 heads 26 / 18 / 16);
  // of 1000 tokens every lane is needed (10.6 / 12.2 / 18.3), and with few a token's heads are spread over CTAs until
  // there are two per SM.
  const int threads = n_tokens > 24 * sms ? 32 : n_tokens > 8 * sms ? 64 : 128;
  const int rounds = (lanes + threads - 1) / threads;
  int split = 2 * sms / n_tokens;
  split = split < 1 ? 1 : split > rounds ? rounds : split;
  const dim3 grid(static_cast<unsigned>(n_tokens), static_cast<unsigned>(split)), block(static_cast<unsigned>(threads));
  if (lg == 4) return launch_dependent(append_kernel<I8, 4>, grid, block, 0, s, a);
  if (lg == 8) return launch_dependent(append_kernel<I8, 8>, grid, block, 0, s, a);
  return launch_dependent(append_kernel<I8, 16>, grid, block, 0, s, a);
}

}  // namespace

vq_status launch_kv_append(const KvGeometry& g, const KvPool& pool, const KvBooks& books, const int* starts, int n_tokens,
                           const __half* k, long long k_stride, const __half* v, long long v_stride, const KvRotary& rot, cudaStream_t s) {
  int sms = 0;
  const vq_status st = device_sms(&sms);
  if (st != VQ_OK) return st;
  AppendArgs a = {g, pool, books, rot, starts, k, v, k_stride, v_stride};
  return g.int8 ? launch<true>(a, n_tokens, sms, s) : launch<false>(a, n_tokens, sms, s);
}

}  // namespace vq
