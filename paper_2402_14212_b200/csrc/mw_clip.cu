// Clipping by the norm of all gradients together (mw_clip_gradients):
//   norm = sqrt(sum g^2),   out = g min(1, max_norm / norm)
// HBM bounds it: every element is read for the norm, read again and written for the product.  Tensors are cut into
// chunks that the blocks take in turn, so one launch serves many tensors of any sizes; squares are summed in 64 bits.
#include <math.h>

#include "mw_common.cuh"

namespace mw {
namespace {

constexpr int kGroup = 256;             // tensors of one launch
constexpr int kChunk = 8192;            // elements
constexpr int kClipThreads = 512;
constexpr int kClipBlocks = 296;

struct ClipGroup {
  const void* in[kGroup];
  void* out[kGroup];
  int64_t size[kGroup];
  int64_t first[kGroup + 1];            // chunks of the tensors before
  uint8_t bf16[kGroup];
  int count;
};

__device__ __forceinline__ int tensor_of(const ClipGroup& g, int64_t chunk) {
  int lo = 0, hi = g.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (g.first[mid] <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double block_sum(double v, double* warp_sum) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
  for (int w = 0; w < kClipThreads / 32; ++w) t += warp_sum[w];
  return t;
}

__global__ void __launch_bounds__(kClipThreads) squares_kernel(const __grid_constant__ ClipGroup g, double* partial) {
  __shared__ double warp_sum[kClipThreads / 32];
  double sum = 0.0;
  for (int64_t c = blockIdx.x; c < g.first[g.count]; c += gridDim.x) {
    const int t = tensor_of(g, c);
    const int64_t i0 = (c - g.first[t]) * kChunk;
    const int n = (int)(g.size[t] - i0 < kChunk ? g.size[t] - i0 : kChunk);
    for (int i = threadIdx.x; i < n; i += kClipThreads) {
      const double v = g.bf16[t] ? (double)__bfloat162float(static_cast<const __nv_bfloat16*>(g.in[t])[i0 + i])
                                 : (double)static_cast<const float*>(g.in[t])[i0 + i];
      sum = fma(v, v, sum);
    }
  }
  sum = block_sum(sum, warp_sum);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ void __launch_bounds__(kClipThreads)
scale_kernel(const __grid_constant__ ClipGroup g, const double* __restrict__ partial, int partials, double max_norm, float* norm_out) {
  __shared__ double warp_sum[kClipThreads / 32];
  double sum = 0.0;
  for (int i = threadIdx.x; i < partials; i += kClipThreads) sum += partial[i];
  const double norm = sqrt(block_sum(sum, warp_sum));
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const float k = norm > max_norm && isfinite(norm) ? (float)(max_norm / norm) : 1.f;
  for (int64_t c = blockIdx.x; c < g.first[g.count]; c += gridDim.x) {
    const int t = tensor_of(g, c);
    if (!g.out[t] || (k == 1.f && g.in[t] == g.out[t])) continue;
    const int64_t i0 = (c - g.first[t]) * kChunk;
    const int n = (int)(g.size[t] - i0 < kChunk ? g.size[t] - i0 : kChunk);
    for (int i = threadIdx.x; i < n; i += kClipThreads) {
      if (g.bf16[t])
        static_cast<__nv_bfloat16*>(g.out[t])[i0 + i] =
            __float2bfloat16_rn(k * __bfloat162float(static_cast<const __nv_bfloat16*>(g.in[t])[i0 + i]));
      else
        static_cast<float*>(g.out[t])[i0 + i] = k * static_cast<const float*>(g.in[t])[i0 + i];
    }
  }
}

}  // namespace
}  // namespace mw

extern "C" mw_status mw_clip_scratch_bytes(int32_t count, size_t* bytes) {
  using namespace mw;
  if (!bytes || count < 0) return MW_ERR_INVALID_ARG;
  *bytes = 256 + sizeof(double) * kClipBlocks * (size_t)(count ? ceil_div(count, kGroup) : 1);
  return MW_OK;
}

extern "C" mw_status mw_clip_gradients(int32_t count, const void* const* in, void* const* out, const int64_t* sizes,
                                       const int32_t* dtypes, double max_norm, float* norm, void* scratch, size_t scratch_bytes,
                                       void* stream) {
  using namespace mw;
  if (count < 0 || !norm || !(max_norm > 0.0) || (count > 0 && (!in || !sizes || !dtypes)) || (count > 0 && !out && !isinf(max_norm)))
    return MW_ERR_INVALID_ARG;
  for (int k = 0; k < count; ++k) {
    if (sizes[k] < 0 || (dtypes[k] != MW_F32 && dtypes[k] != MW_BF16_F32ACC)) return MW_ERR_INVALID_ARG;
    if (sizes[k] > 0 && (!in[k] || (out && !out[k]))) return MW_ERR_INVALID_ARG;
  }
  size_t need = 0;
  MW_TRY(mw_clip_scratch_bytes(count, &need));
  if (!scratch || ((uintptr_t)scratch & 255u) || scratch_bytes < need) return MW_ERR_WORKSPACE;
  cudaStream_t s = (cudaStream_t)stream;
  double* partial = static_cast<double*>(scratch);
  const int groups = count ? ceil_div(count, kGroup) : 1;
  static thread_local ClipGroup g;
  auto fill = [&](int group) {
    const int k0 = group * kGroup;
    g.count = count - k0 < kGroup ? count - k0 : kGroup;
    int64_t chunks = 0;
    for (int k = 0; k < g.count; ++k) {
      g.in[k] = in[k0 + k];
      g.out[k] = out ? out[k0 + k] : nullptr;
      g.size[k] = sizes[k0 + k];
      g.bf16[k] = dtypes[k0 + k] == MW_BF16_F32ACC;
      g.first[k] = chunks;
      chunks += (sizes[k0 + k] + kChunk - 1) / kChunk;
    }
    g.first[g.count] = chunks;
  };
  for (int i = 0; i < groups; ++i) {
    fill(i);
    squares_kernel<<<kClipBlocks, kClipThreads, 0, s>>>(g, partial + (size_t)i * kClipBlocks);
    MW_TRY(launch_ok());
  }
  for (int i = 0; i < groups; ++i) {
    fill(i);
    scale_kernel<<<kClipBlocks, kClipThreads, 0, s>>>(g, partial, groups * kClipBlocks, max_norm, i ? nullptr : norm);
    MW_TRY(launch_ok());
  }
  return MW_OK;
}
