// Clipping by the norm of all gradients together (mw_clip_gradients):
//   norm = sqrt(sum g^2),   out = g min(1, max_norm / norm)
// HBM bounds it: every element is read for the norm, read again and written for the product. Tensors are cut into
// chunks that the blocks take in turn, so one launch serves many tensors of any sizes; squares are summed in 64 bits,
// which costs nothing (64 of 1024x1024 fp32, 268 MB: squares 46 to 55 us with sums in 64 bits and in 32). Measured, the
// same case: 136 us for both launches, 5.9 TB/s of the 805 MB that pass; of the second read L2 holds what the first
// ended with, which is where it begins.
#include <math.h>

#include <algorithm>
#include <memory>
#include <new>

#include "mw_launch.cuh"

namespace mw {
namespace {

constexpr int kGroup = 256;             // tensors of one launch
constexpr int kChunkBytes = 65536;      // of a tensor, a block at a time
constexpr int kClipThreads = 1024;
constexpr int kClipBlocks = 296;        // two a multiprocessor
constexpr int kAccesses = kChunkBytes / 16 / kClipThreads;      // of 16 bytes, a thread, all under way at once

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

struct Share { int64_t first; int count; bool wide, bf16; const char* in; char* out; };
__device__ __forceinline__ Share share_of(const ClipGroup& g, int64_t chunk) {
  const int t = tensor_of(g, chunk);
  Share c;
  c.bf16 = g.bf16[t];
  const int e = c.bf16 ? 2 : 4, per = kChunkBytes / e;
  c.first = (chunk - g.first[t]) * per;
  const int64_t left = g.size[t] - c.first;
  c.count = (int)(left < per ? left : per);
  c.in = static_cast<const char*>(g.in[t]) + c.first * e;
  c.out = g.out[t] ? static_cast<char*>(g.out[t]) + c.first * e : nullptr;
  c.wide = (((uintptr_t)c.in | (uintptr_t)c.out) & 15) == 0;
  return c;
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ float element(const Share& c, int i) {
  return c.bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(c.in)[i]) : reinterpret_cast<const float*>(c.in)[i];
}
__device__ __forceinline__ void add_square(double& sum, float v) { sum = fma((double)v, (double)v, sum); }

__global__ void __launch_bounds__(kClipThreads) squares_kernel(const __grid_constant__ ClipGroup g, double* partial) {
  after_previous();
  __shared__ double warp_sum[kClipThreads / 32];
  double sum = 0.0;
  for (int64_t chunk = blockIdx.x; chunk < g.first[g.count]; chunk += gridDim.x) {
    const Share c = share_of(g, chunk);
    int done = 0;
    if (c.wide) {
      const int vecs = c.count * (c.bf16 ? 2 : 4) / 16;
      uint4 x[kAccesses];
#pragma unroll
      for (int k = 0; k < kAccesses; ++k) {
        const int i = k * kClipThreads + threadIdx.x;
        x[k] = i < vecs ? reinterpret_cast<const uint4*>(c.in)[i] : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int k = 0; k < kAccesses; ++k) {
        const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (c.bf16) {
            add_square(sum, low(w[q]));
            add_square(sum, high(w[q]));
          } else {
            add_square(sum, __uint_as_float(w[q]));
          }
        }
      }
      done = vecs * (c.bf16 ? 8 : 4);
    }
#pragma unroll 8
    for (int i = done + threadIdx.x; i < c.count; i += kClipThreads) add_square(sum, element(c, i));
  }
  sum = block_sum(sum, warp_sum);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

// Chunks are taken from the last to the first: what the squares have just read is still in L2.
__global__ void __launch_bounds__(kClipThreads)
scale_kernel(const __grid_constant__ ClipGroup g, const double* __restrict__ partial, int partials, double max_norm, float* norm_out) {
  after_previous();
  __shared__ double warp_sum[kClipThreads / 32];
  double sum = 0.0;
  for (int i = threadIdx.x; i < partials; i += kClipThreads) sum += partial[i];
  const double norm = sqrt(block_sum(sum, warp_sum));
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const float k = norm > max_norm && isfinite(norm) ? (float)(max_norm / norm) : 1.f;
  for (int64_t chunk = g.first[g.count] - 1 - blockIdx.x; chunk >= 0; chunk -= gridDim.x) {
    const Share c = share_of(g, chunk);
    if (!c.out || (k == 1.f && c.in == c.out)) continue;
    int done = 0;
    if (c.wide) {
      const int vecs = c.count * (c.bf16 ? 2 : 4) / 16;
      uint4 x[kAccesses];
#pragma unroll
      for (int j = 0; j < kAccesses; ++j) {
        const int i = j * kClipThreads + threadIdx.x;
        if (i < vecs) x[j] = reinterpret_cast<const uint4*>(c.in)[i];
      }
#pragma unroll
      for (int j = 0; j < kAccesses; ++j) {
        const int i = j * kClipThreads + threadIdx.x;
        uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (c.bf16) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(k * low(w[q]), k * high(w[q]));
            w[q] = *reinterpret_cast<const uint32_t*>(&h);
          } else {
            w[q] = __float_as_uint(k * __uint_as_float(w[q]));
          }
        }
        if (i < vecs) reinterpret_cast<uint4*>(c.out)[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
      done = vecs * (c.bf16 ? 8 : 4);
    }
#pragma unroll 8
    for (int i = done + threadIdx.x; i < c.count; i += kClipThreads) {
      const float v = k * element(c, i);
      if (c.bf16) reinterpret_cast<__nv_bfloat16*>(c.out)[i] = __float2bfloat16_rn(v);
      else reinterpret_cast<float*>(c.out)[i] = v;
    }
  }
}

// Whether what a call writes is apart from what its other blocks read and write: a tensor that stands in the list twice
// would be scaled twice, or half of it.
struct Span { uintptr_t from, to; };
bool overlaps(const Span& a, const Span& b) { return a.from < b.to && b.from < a.to; }
mw_status check_apart(int count, const void* const* in, void* const* out, const int64_t* sizes, const int32_t* dtypes, bool norm_alone) {
  std::unique_ptr<Span[]> written(new (std::nothrow) Span[count]);
  if (!written) return MW_ERR_WORKSPACE;
  int n = 0;
  auto span = [&](const void* p, int k) { return Span{(uintptr_t)p, (uintptr_t)p + (uintptr_t)sizes[k] * (dtypes[k] == MW_BF16_F32ACC ? 2 : 4)}; };
  for (int k = 0; k < count; ++k)
    if (sizes[k] > 0 && !(norm_alone && in[k] == out[k])) written[n++] = span(out[k], k);
  auto before = [](const Span& a, const Span& b) { return a.from < b.from; };
  if (!std::is_sorted(&written[0], &written[0] + n, before)) std::sort(&written[0], &written[0] + n, before);
  for (int i = 1; i < n; ++i)
    if (overlaps(written[i - 1], written[i])) return MW_ERR_INVALID_ARG;
  for (int k = 0; k < count && n; ++k) {
    if (sizes[k] == 0 || in[k] == out[k]) continue;
    const Span x = span(in[k], k);
    const Span* next = std::lower_bound(&written[0], &written[0] + n, x, before);          // the first that starts there or later
    if ((next < &written[0] + n && overlaps(*next, x)) || (next > &written[0] && overlaps(next[-1], x))) return MW_ERR_INVALID_ARG;
  }
  return MW_OK;
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
  if (out && count > 0) MW_TRY(check_apart(count, in, out, sizes, dtypes, isinf(max_norm)));
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
      const int64_t per = kChunkBytes / (g.bf16[k] ? 2 : 4);
      chunks += (sizes[k0 + k] + per - 1) / per;
    }
    g.first[g.count] = chunks;
  };
  for (int i = 0; i < groups; ++i) {
    fill(i);
    MW_TRY(launch_after(squares_kernel, kClipBlocks, kClipThreads, 0, s, g, partial + (size_t)i * kClipBlocks));
  }
  for (int i = 0; i < groups; ++i) {
    fill(i);
    MW_TRY(launch_after(scale_kernel, kClipBlocks, kClipThreads, 0, s, g, partial, groups * kClipBlocks, max_norm, i ? nullptr : norm));
  }
  return MW_OK;
}
