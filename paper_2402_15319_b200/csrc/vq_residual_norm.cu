// The residual stream between two blocks (vq_residual_norm): x' = x + scale * gate * post(y), h = pre(x').
//
// Bound by memory: every row of x, y (and the gate, where it has rows) is read once, x' and h are written once.  A row
// stays in registers between its reductions (pieces of eight columns, PER of them a thread), the mean and the centred
// squares are summed one after the other, in binary32, in a fixed order.
// 8192 x 8192, both norms, gate per channel, binary32 residual: 143 us = 5.6 TB/s (with rows straight into registers and weights
// past L1 207); one row of 4096: 1.9 us.
#include "vq_device.cuh"
#include "vq_kv.cuh"
#include "vq_residual_norm.cuh"

namespace vq {
namespace {

using namespace dev;

constexpr int kWaitTries = 1 << 18;   // mbarrier polls before a thread gives up and flags an error

struct Float8 {
  float v[8];
};

// A thread's piece i of a row: eight columns.  VEC: adjacent ones, whole and 16-byte aligned.  Else `gap` = all threads of the
// row apart, so that a warp's loads of one column each are adjacent; columns from `cols` on are zeros.
template <bool VEC>
__device__ __forceinline__ int piece(int first, int step, int i) { return VEC ? (first + i * step) * 8 : first + i * 8 * step; }
__device__ __forceinline__ Float8 unpack8(uint4 w) {
  Float8 f;
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
    f.v[2 * i] = p.x;
    f.v[2 * i + 1] = p.y;
  }
  return f;
}
template <class T, bool CACHED>
__device__ __forceinline__ T fetch_global(const T* p) {
  if constexpr (CACHED) return __ldg(p);
  else return __ldcg(p);
}
template <bool VEC, bool CACHED = false>
__device__ __forceinline__ Float8 load8h(const __half* row, int c, int cols, int gap) {
  Float8 f;
  if (VEC) {
    f = unpack8(fetch_global<uint4, CACHED>(reinterpret_cast<const uint4*>(row + c)));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      f.v[i] = c + i * gap < cols ? __half2float(__ushort_as_half(fetch_global<unsigned short, CACHED>(reinterpret_cast<const unsigned short*>(row) + c + i * gap))) : 0.0f;
  }
  return f;
}
template <bool VEC>
__device__ __forceinline__ Float8 load8f(const float* row, int c, int cols, int gap) {
  Float8 f;
  if (VEC) {
    const float4 a = __ldcg(reinterpret_cast<const float4*>(row + c)), b = __ldcg(reinterpret_cast<const float4*>(row + c + 4));
    f = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = c + i * gap < cols ? __ldcg(row + c + i * gap) : 0.0f;
  }
  return f;
}
template <bool VEC>
__device__ __forceinline__ void store8h(__half* row, int c, int cols, int gap, const Float8& f) {
  if (VEC) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(f.v[2 * i], f.v[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(row + c) = make_uint4(u[0], u[1], u[2], u[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i * gap < cols) row[c + i * gap] = __float2half_rn(f.v[i]);
  }
}
template <bool VEC>
__device__ __forceinline__ void store8f(float* row, int c, int cols, int gap, const Float8& f) {
  if (VEC) {
    *reinterpret_cast<float4*>(row + c) = make_float4(f.v[0], f.v[1], f.v[2], f.v[3]);
    *reinterpret_cast<float4*>(row + c + 4) = make_float4(f.v[4], f.v[5], f.v[6], f.v[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i * gap < cols) row[c + i * gap] = f.v[i];
  }
}

// Sums over the threads of a row: a warp, or the whole CTA (a word per warp in shared memory, two sets by turns: a barrier per
// sum is enough).  Every thread gets the sum, added up in the same order.
struct RowSums {
  float* s;    // [2][32]
  int turn;
};
template <bool WARP_ROW>
__device__ __forceinline__ float row_sum(float v, RowSums& r) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  if (WARP_ROW || blockDim.x == 32) return v;
  float* s = r.s + 32 * r.turn;
  r.turn ^= 1;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  if (lane == 0) s[warp] = v;
  __syncthreads();
  v = lane < warps ? s[lane] : 0.0f;
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}

// The norm of the row in `u`: mean taken away (layer), divided by the root of the mean square; weights and biases follow.
// CACHED: they may come through L1.  EARLY 1: weights asked for before the sums, 2: biases too, where registers hold them (8192
// rows of 4096, rings: 77 -> 70 us, with LayerNorm's 94 -> 97; 16384 of 1000, a warp each: 47 -> 43; one of 4096: 2.02 -> 1.95;
// with rings of 8192 columns, 512 threads: 142 -> 144, so not there, nor with 1024 threads: 200 rows of 8192 6.9 -> 8.4).
template <bool VEC, bool WARP_ROW, int PER, bool CACHED, int EARLY>
__device__ __forceinline__ void norm(Float8 (&u)[PER], const __half* weight, const __half* bias, const ResidualNorm& a, int first, int step,
                                     RowSums& s) {
  const float inv_n = 1.0f / static_cast<float>(a.cols);
  uint4 w8[PER], b8[PER];
  if (VEC && EARLY) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = piece<VEC>(first, step, i);
      w8[i] = b8[i] = make_uint4(0, 0, 0, 0);
      if (c < a.cols) w8[i] = fetch_global<uint4, CACHED>(reinterpret_cast<const uint4*>(weight + c));
      if (EARLY == 2 && c < a.cols && bias) b8[i] = fetch_global<uint4, CACHED>(reinterpret_cast<const uint4*>(bias + c));
    }
  }
  if (a.layer) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += u[i].v[e];
    const float mean = row_sum<WARP_ROW>(sum, s) * inv_n;
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) u[i].v[e] = piece<VEC>(first, step, i) + e * (VEC ? 1 : step) < a.cols ? u[i].v[e] - mean : 0.0f;
  }
  float sq = 0.0f;
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sq += u[i].v[e] * u[i].v[e];
  const float r = rsqrtf(row_sum<WARP_ROW>(sq, s) * inv_n + a.eps);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int c = piece<VEC>(first, step, i);
    if (c >= a.cols) continue;
    const Float8 w = VEC && EARLY ? unpack8(w8[i]) : load8h<VEC, CACHED>(weight, c, a.cols, step);
    Float8 b = {};
    if (VEC && EARLY == 2) b = unpack8(b8[i]);
    else if (bias) b = load8h<VEC, CACHED>(bias, c, a.cols, step);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[i].v[e] = u[i].v[e] * r * w.v[e] + b.v[e];
  }
}

// CACHED: a plain launch, weights through L1 (see residual_norm_rows_kernel).
template <bool VEC, bool WIDE, bool WARP_ROW, int PER, int MAX_THREADS, bool CACHED>
__global__ void __launch_bounds__(MAX_THREADS) residual_norm_kernel(ResidualNorm a) {
  __shared__ float s_sums[64];
  RowSums s = {s_sums, 0};
  constexpr int kEarly = WARP_ROW || (PER == 1 && MAX_THREADS <= 512) ? 2 : 0;
  if (!CACHED) {
    pdl_launch_dependents();
    pdl_wait();
  }
  const long long row = WARP_ROW ? static_cast<long long>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  if (WARP_ROW && row >= a.rows) return;
  const int first = WARP_ROW ? threadIdx.x & 31 : threadIdx.x, step = WARP_ROW ? 32 : blockDim.x;

  Float8 x[PER];
  const float* xf = static_cast<const float*>(a.x) + row * a.x_stride;
  const __half* xh = static_cast<const __half*>(a.x) + row * a.x_stride;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int c = piece<VEC>(first, step, i);
    x[i] = {};
    if (c < a.cols) x[i] = WIDE ? load8f<VEC>(xf, c, a.cols, step) : load8h<VEC>(xh, c, a.cols, step);
  }
  if (a.y) {
    Float8 y[PER];
    const __half* yr = a.y + row * a.y_stride;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = piece<VEC>(first, step, i);
      y[i] = {};
      if (c < a.cols) y[i] = load8h<VEC>(yr, c, a.cols, step);
    }
    if (a.post_w) norm<VEC, WARP_ROW, PER, CACHED, kEarly>(y, a.post_w, a.post_b, a, first, step, s);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = piece<VEC>(first, step, i);
      if (c >= a.cols) continue;
      if (a.gate) {
        const Float8 gt = load8h<VEC>(a.gate + row * a.gate_stride, c, a.cols, step);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[i].v[e] *= gt.v[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i].v[e] += a.scale * y[i].v[e];
    }
  }
  if (a.x_out) {
    float* of = static_cast<float*>(a.x_out) + row * a.x_out_stride;
    __half* oh = static_cast<__half*>(a.x_out) + row * a.x_out_stride;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = piece<VEC>(first, step, i);
      if (c >= a.cols) continue;
      if (WIDE) store8f<VEC>(of, c, a.cols, step, x[i]);
      else store8h<VEC>(oh, c, a.cols, step, x[i]);
    }
  }
  if (a.h) {
    norm<VEC, WARP_ROW, PER, CACHED, kEarly>(x, a.pre_w, a.pre_b, a, first, step, s);
    __half* hr = a.h + row * a.h_stride;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = piece<VEC>(first, step, i);
      if (c < a.cols) store8h<VEC>(hr, c, a.cols, step, x[i]);
    }
  }
}

// Many long rows: CTAs that stay, each with a ring of rows in shared memory that one thread fills by bulk copies, so that the
// next rows are on their way while this one is reduced and stored.  Launched plainly (its start hides nothing beside its
// length), so weights may come through L1, which holds them from row to row.
template <bool WIDE, int PER, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) residual_norm_rows_kernel(ResidualNorm a, int stages, int* error_flag) {
  extern __shared__ __align__(128) unsigned char ring[];
  __shared__ float s_sums[64];
  RowSums s = {s_sums, 0};
  __shared__ __align__(8) unsigned long long s_bar[8];
  const int tid = threadIdx.x;
  const int x_bytes = a.cols * (WIDE ? 4 : 2), h_bytes = a.cols * 2;
  const bool gate_rows = a.gate && a.gate_stride;
  const int stage_bytes = x_bytes + (a.y ? h_bytes : 0) + (gate_rows ? h_bytes : 0);
  const uint32_t bars = smem_u32(s_bar), ring_at = smem_u32(ring);
  if (tid < 8) mbar_init(bars + 8 * tid, 1);
  mbar_init_fence();
  __syncthreads();
  auto fetch = [&](int stage, long long row) {
    const uint32_t bar = bars + 8 * stage, dst = ring_at + stage * stage_bytes;
    mbar_arrive_expect_tx(bar, stage_bytes);
    bulk_g2s(dst, static_cast<const unsigned char*>(a.x) + row * a.x_stride * (WIDE ? 4 : 2), x_bytes, bar);
    if (a.y) bulk_g2s(dst + x_bytes, a.y + row * a.y_stride, h_bytes, bar);
    if (gate_rows) bulk_g2s(dst + x_bytes + h_bytes, a.gate + row * a.gate_stride, h_bytes, bar);
  };
  if (tid == 0)
    for (int i = 0; i < stages; ++i) {
      const long long row = blockIdx.x + static_cast<long long>(i) * gridDim.x;
      if (row < a.rows) fetch(i, row);
    }
  int stage = 0, tries = kWaitTries;
  uint32_t phase = 0;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    if (!mbar_wait(bars + 8 * stage, phase, tries)) {   // (a copy that never completes: wrong output, but the kernel ends)
      if (tries && tid == 0) atomicAdd(error_flag, 1);
      tries = 0;
    }
    const uint32_t at = ring_at + stage * stage_bytes;
    Float8 x[PER], y[PER];
    uint4 g[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = (tid + i * THREADS) * 8;
      x[i] = {};
      y[i] = {};
      g[i] = make_uint4(0, 0, 0, 0);
      if (c >= a.cols) continue;
      if (WIDE) {
        const uint4 u = lds128(at + c * 4), w = lds128(at + c * 4 + 16);
        x[i] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w),
                __uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w)};
      } else {
        x[i] = unpack8(lds128(at + c * 2));
      }
      if (a.y) y[i] = unpack8(lds128(at + x_bytes + c * 2));
      if (gate_rows) g[i] = lds128(at + x_bytes + h_bytes + c * 2);
      else if (a.gate) g[i] = __ldg(reinterpret_cast<const uint4*>(a.gate + c));
    }
    __syncthreads();   // the stage has been read
    const long long ahead = row + static_cast<long long>(stages) * gridDim.x;
    if (tid == 0 && ahead < a.rows) fetch(stage, ahead);
    if (++stage == stages) {
      stage = 0;
      phase ^= 1;
    }
    if (a.y) {
      if (a.post_w) norm<true, false, PER, true, (THREADS <= 256)>(y, a.post_w, a.post_b, a, tid, THREADS, s);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if (a.gate) {
          const Float8 gt = unpack8(g[i]);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[i].v[e] *= gt.v[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i].v[e] += a.scale * y[i].v[e];
      }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = (tid + i * THREADS) * 8;
      if (a.x_out && c < a.cols) {
        if (WIDE) store8f<true>(static_cast<float*>(a.x_out) + row * a.x_out_stride, c, a.cols, 1, x[i]);
        else store8h<true>(static_cast<__half*>(a.x_out) + row * a.x_out_stride, c, a.cols, 1, x[i]);
      }
    }
    if (a.h) {
      norm<true, false, PER, true, (THREADS <= 256)>(x, a.pre_w, a.pre_b, a, tid, THREADS, s);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int c = (tid + i * THREADS) * 8;
        if (c < a.cols) store8h<true>(a.h + row * a.h_stride, c, a.cols, 1, x[i]);
      }
    }
  }
}

template <bool WIDE, int PER, int THREADS>
vq_status launch_rows(const ResidualNorm& a, int sms, cudaStream_t s) {
  static int ready[kMaxDevices] = {};
  int dev = 0, *error_flag = nullptr;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return VQ_ERR_CUDA;
  vq_status st = device_error_counter(&error_flag);
  if (st != VQ_OK) return st;
  auto kernel = residual_norm_rows_kernel<WIDE, PER, THREADS>;
  constexpr int kBytes = 222 * 1024, kMost = 1024 / THREADS;   // rings of an SM; CTAs that its registers hold
  if (!__atomic_load_n(&ready[dev], __ATOMIC_ACQUIRE)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes) != cudaSuccess) return VQ_ERR_CUDA;
    __atomic_store_n(&ready[dev], 1, __ATOMIC_RELEASE);
  }
  const int stage_bytes = a.cols * ((WIDE ? 4 : 2) + (a.y ? 2 : 0) + (a.gate && a.gate_stride ? 2 : 0));
  int per_sm = kMost;
  while (per_sm > 1 && (kBytes / per_sm - 1024) / stage_bytes < 2) --per_sm;   // (1024 bytes of a CTA are not the ring's)
  int stages = (kBytes / per_sm - 1024) / stage_bytes;
  if (stages < 2) return VQ_ERR_UNSUPPORTED;
  if (stages > 8) stages = 8;
  const int ctas = a.rows < sms * per_sm ? a.rows : sms * per_sm;
  kernel<<<ctas, THREADS, static_cast<size_t>(stages) * stage_bytes, s>>>(a, stages, error_flag);
  return check_launch();
}

template <bool VEC, bool WIDE, bool WARP_ROW, int PER, int MAX_THREADS>
vq_status launch_one(const ResidualNorm& a, int threads, bool many, cudaStream_t s) {
  const dim3 grid(static_cast<unsigned>(WARP_ROW ? (a.rows - 1) / (threads / 32) + 1 : a.rows)), block(static_cast<unsigned>(threads));
  if (!many) return launch_dependent(residual_norm_kernel<VEC, WIDE, WARP_ROW, PER, MAX_THREADS, false>, grid, block, 0, s, a);
  residual_norm_kernel<VEC, WIDE, WARP_ROW, PER, MAX_THREADS, true><<<grid, block, 0, s>>>(a);
  return check_launch();
}

template <bool VEC, bool WIDE>
vq_status launch(const ResidualNorm& a, int sms, cudaStream_t s) {
  const int pieces = (a.cols + 7) / 8;
  const bool many = a.rows > 2 * sms;
  if (pieces <= 32) return launch_one<VEC, WIDE, true, 1, 128>(a, 128, many, s);   // short rows: a warp each
  if (pieces <= 128 && many) {
    if (pieces <= 64) return launch_one<VEC, WIDE, true, 2, 128>(a, 128, many, s);
    if (pieces <= 96) return launch_one<VEC, WIDE, true, 3, 128>(a, 128, many, s);
    return launch_one<VEC, WIDE, true, 4, 128>(a, 128, many, s);
  }
  if (VEC && many) {
    const vq_status st = pieces <= 256 ? launch_rows<WIDE, 2, 128>(a, sms, s)
                       : pieces <= 512 ? launch_rows<WIDE, 2, 256>(a, sms, s)
                       : pieces <= 1024 ? launch_rows<WIDE, 2, 512>(a, sms, s)
                       : pieces <= 2048 ? launch_rows<WIDE, 2, 1024>(a, sms, s) : VQ_ERR_UNSUPPORTED;
    if (st != VQ_ERR_UNSUPPORTED) return st;
  }
  // A row per CTA, as many threads as it has pieces while they suffice: the shortest way through the row.
  auto threads = [&](int per) { return ((pieces + per - 1) / per + 31) / 32 * 32; };
  if (pieces <= 512 && !many) return launch_one<VEC, WIDE, false, 1, 512>(a, threads(1), many, s);
  if (pieces <= 1024 && !many) return launch_one<VEC, WIDE, false, 1, 1024>(a, threads(1), many, s);
  if (pieces <= 1024) return launch_one<VEC, WIDE, false, 2, 512>(a, threads(2), many, s);
  return launch_one<VEC, WIDE, false, 4, 1024>(a, threads(4), many, s);
}

}  // namespace

vq_status launch_residual_norm(const ResidualNorm& a, cudaStream_t s) {
  int sms = 0;
  const vq_status st = device_sms(&sms);
  if (st != VQ_OK) return st;
  // whole 16-byte pieces in every row?
  const bool vec = a.cols % 8 == 0 && (a.x_stride | a.y_stride | a.gate_stride | a.x_out_stride | a.h_stride) % 8 == 0;
  if (vec) return a.wide ? launch<true, true>(a, sms, s) : launch<true, false>(a, sms, s);
  return a.wide ? launch<false, true>(a, sms, s) : launch<false, false>(a, sms, s);
}

}  // namespace vq
