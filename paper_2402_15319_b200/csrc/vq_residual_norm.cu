// The residual stream between two blocks (vq_residual_norm): x' = x + scale * gate * post(y), h = pre(x').
//
// Bound by memory: every row of x, y (and the gate, where it has rows) is read once, x' and h are written once.  A row
// stays in registers between its reductions (pieces of eight columns, PER of them a thread), the mean and the centred
// squares are summed one after the other, in binary32, in a fixed order.
#include "vq_device.cuh"
#include "vq_kv.cuh"
#include "vq_residual_norm.cuh"

namespace vq {
namespace {

using namespace dev;

struct Float8 {
  float v[8];
};

// Eight columns from `c` on; columns from `cols` on are zeros.  VEC: the piece is whole and 16-byte aligned.
template <bool VEC>
__device__ __forceinline__ Float8 load8h(const __half* row, int c, int cols) {
  Float8 f;
  if (VEC) {
    const uint4 w = __ldcg(reinterpret_cast<const uint4*>(row + c));
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
      f.v[2 * i] = p.x;
      f.v[2 * i + 1] = p.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      f.v[i] = c + i < cols ? __half2float(__ushort_as_half(__ldcg(reinterpret_cast<const unsigned short*>(row) + c + i))) : 0.0f;
  }
  return f;
}
template <bool VEC>
__device__ __forceinline__ Float8 load8f(const float* row, int c, int cols) {
  Float8 f;
  if (VEC) {
    const float4 a = __ldcg(reinterpret_cast<const float4*>(row + c)), b = __ldcg(reinterpret_cast<const float4*>(row + c + 4));
    f = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = c + i < cols ? __ldcg(row + c + i) : 0.0f;
  }
  return f;
}
template <bool VEC>
__device__ __forceinline__ void store8h(__half* row, int c, int cols, const Float8& f) {
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
      if (c + i < cols) row[c + i] = __float2half_rn(f.v[i]);
  }
}
template <bool VEC>
__device__ __forceinline__ void store8f(float* row, int c, int cols, const Float8& f) {
  if (VEC) {
    *reinterpret_cast<float4*>(row + c) = make_float4(f.v[0], f.v[1], f.v[2], f.v[3]);
    *reinterpret_cast<float4*>(row + c + 4) = make_float4(f.v[4], f.v[5], f.v[6], f.v[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) row[c + i] = f.v[i];
  }
}

// Sum over the threads of a row: a warp, or the whole CTA (then `s` holds a word per warp; every thread gets the sum).
template <bool WARP_ROW>
__device__ __forceinline__ float row_sum(float v, float* s) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  if (WARP_ROW || blockDim.x == 32) return v;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  __syncthreads();   // (the last sum has been read)
  if (lane == 0) s[warp] = v;
  __syncthreads();
  v = lane < warps ? s[lane] : 0.0f;
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}

// The norm of the row in `u`: mean taken away (layer), divided by the root of the mean square; weights and biases follow.
template <bool VEC, bool WARP_ROW, int PER>
__device__ __forceinline__ void norm(Float8 (&u)[PER], const __half* weight, const __half* bias, const ResidualNorm& a, int first, int step,
                                     float* s) {
  const float inv_n = 1.0f / static_cast<float>(a.cols);
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
      for (int e = 0; e < 8; ++e) u[i].v[e] = (first + i * step) * 8 + e < a.cols ? u[i].v[e] - mean : 0.0f;
  }
  float sq = 0.0f;
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sq += u[i].v[e] * u[i].v[e];
  const float r = rsqrtf(row_sum<WARP_ROW>(sq, s) * inv_n + a.eps);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int c = (first + i * step) * 8;
    if (c >= a.cols) continue;
    const Float8 w = load8h<VEC>(weight, c, a.cols);
    Float8 b = {};
    if (bias) b = load8h<VEC>(bias, c, a.cols);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[i].v[e] = u[i].v[e] * r * w.v[e] + b.v[e];
  }
}

template <bool VEC, bool WIDE, bool WARP_ROW, int PER, int MAX_THREADS>
__global__ void __launch_bounds__(MAX_THREADS) residual_norm_kernel(ResidualNorm a) {
  __shared__ float s[32];
  pdl_launch_dependents();
  pdl_wait();
  const long long row = WARP_ROW ? static_cast<long long>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  if (WARP_ROW && row >= a.rows) return;
  const int first = WARP_ROW ? threadIdx.x & 31 : threadIdx.x, step = WARP_ROW ? 32 : blockDim.x;

  Float8 x[PER];
  const float* xf = static_cast<const float*>(a.x) + row * a.x_stride;
  const __half* xh = static_cast<const __half*>(a.x) + row * a.x_stride;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int c = (first + i * step) * 8;
    x[i] = {};
    if (c < a.cols) x[i] = WIDE ? load8f<VEC>(xf, c, a.cols) : load8h<VEC>(xh, c, a.cols);
  }
  if (a.y) {
    Float8 y[PER];
    const __half* yr = a.y + row * a.y_stride;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = (first + i * step) * 8;
      y[i] = {};
      if (c < a.cols) y[i] = load8h<VEC>(yr, c, a.cols);
    }
    if (a.post_w) norm<VEC, WARP_ROW, PER>(y, a.post_w, a.post_b, a, first, step, s);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = (first + i * step) * 8;
      if (c >= a.cols) continue;
      if (a.gate) {
        const Float8 gt = load8h<VEC>(a.gate + row * a.gate_stride, c, a.cols);
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
      const int c = (first + i * step) * 8;
      if (c >= a.cols) continue;
      if (WIDE) store8f<VEC>(of, c, a.cols, x[i]);
      else store8h<VEC>(oh, c, a.cols, x[i]);
    }
  }
  if (a.h) {
    norm<VEC, WARP_ROW, PER>(x, a.pre_w, a.pre_b, a, first, step, s);
    __half* hr = a.h + row * a.h_stride;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = (first + i * step) * 8;
      if (c < a.cols) store8h<VEC>(hr, c, a.cols, x[i]);
    }
  }
}

template <bool VEC, bool WIDE>
vq_status launch(const ResidualNorm& a, int sms, cudaStream_t s) {
  const int pieces = (a.cols + 7) / 8;
  if (pieces <= 32) {   // short rows: a warp each, four to a CTA
    return launch_dependent(residual_norm_kernel<VEC, WIDE, true, 1, 128>, dim3(static_cast<unsigned>((a.rows + 3) / 4)), dim3(128), 0, s, a);
  }
  // A row per CTA.  Few rows: a thread per piece, the shortest way through the row.  Many: four pieces a thread, so that
  // several CTAs share an SM and one row's loads run under another's reductions.
  const int per = a.rows <= sms && pieces <= 1024 ? 1 : 4;
  const int threads = ((pieces + per - 1) / per + 31) / 32 * 32;
  const dim3 grid(static_cast<unsigned>(a.rows)), block(static_cast<unsigned>(threads));
  if (per == 1) return launch_dependent(residual_norm_kernel<VEC, WIDE, false, 1, 1024>, grid, block, 0, s, a);
  if (threads <= 512) return launch_dependent(residual_norm_kernel<VEC, WIDE, false, 4, 512>, grid, block, 0, s, a);
  return launch_dependent(residual_norm_kernel<VEC, WIDE, false, 4, 1024>, grid, block, 0, s, a);   // (rows of over 16384)
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
