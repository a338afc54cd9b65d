// Softmax cross entropy over a vocabulary, and its gradient (mw_token_loss_*):
//   z = s h W^T,  loss_i = log sum_j exp z_ij - z_{i,t_i},  dz_ij = g_i (p_ij - [j = t_i]),  dh = s dz W,  dW = s dz^T h
// Rows that have a target are put together first, so that the others cost nothing and nothing of them is read.
#include <math.h>

#include "mw_common.cuh"

namespace mw {
namespace {

constexpr int kIndexRows = 1024;          // rows of one block that looks for targets
constexpr int64_t kPieceBytes = (int64_t)1 << 30;

// what the kernels of one call share, behind the status block
struct LossInfo {
  DeviceStatus st;
  unsigned pad[59];
  int live;                 // rows that are not left out
  unsigned pad2[63];
};

struct LossArgs {
  int64_t rows;
  int vocab, dim;
  int64_t ld_h, ld_w, ld_dh, ld_dw;
  float scale;
};

template <typename I>
__device__ __forceinline__ int target_of(const I* targets, const float* weight, int64_t i, int vocab) {
  const I t = targets[i];
  const bool in = t >= 0 && t < (I)vocab && (weight == nullptr || weight[i] != 0.f);
  return in ? (int)t : -1;
}

template <typename I>
__global__ void __launch_bounds__(kIndexRows) count_live_kernel(const I* targets, const float* weight, int64_t rows, int vocab, int* counts) {
  const int64_t i = (int64_t)blockIdx.x * kIndexRows + threadIdx.x;
  const int n = __syncthreads_count(i < rows && target_of(targets, weight, i, vocab) >= 0);
  if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

// rows with a target to the front of `row`, in order, the others to its end, and their losses are zero
template <typename I>
__global__ void __launch_bounds__(kIndexRows)
index_live_kernel(const I* targets, const float* weight, int64_t rows, int vocab, const int* counts, int blocks, int* row, int* target,
                  float* g, float* loss, LossInfo* info) {
  __shared__ int warp_sum[32];
  __shared__ int sums[2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x < 2) sums[threadIdx.x] = 0;
  __syncthreads();
  int mine[2] = {0, 0};
  for (int b = threadIdx.x; b < blocks; b += kIndexRows) {
    mine[0] += counts[b];
    if (b < (int)blockIdx.x) mine[1] += counts[b];
  }
  if (mine[0]) atomicAdd(&sums[0], mine[0]);
  if (mine[1]) atomicAdd(&sums[1], mine[1]);
  const int64_t i = (int64_t)blockIdx.x * kIndexRows + threadIdx.x;
  const int t = i < rows ? target_of(targets, weight, i, vocab) : -1;
  const unsigned on = __ballot_sync(0xffffffffu, t >= 0);
  if (lane == 0) warp_sum[warp] = __popc(on);
  __syncthreads();
  const int live = sums[0];
  int at = sums[1] + __popc(on & ((1u << lane) - 1u));
  for (int w = 0; w < warp; ++w) at += warp_sum[w];
  if (blockIdx.x == 0 && threadIdx.x == 0) info->live = live;
  if (i >= rows) return;
  if (t >= 0) {
    row[at] = (int)i;
    target[at] = t;
    g[at] = weight ? weight[i] : 1.f / (float)live;
  } else {
    row[rows - 1 - (i - at)] = (int)i;
    loss[i] = 0.f;
  }
}

template <typename T>
__global__ void __launch_bounds__(256)
stage_rows_kernel(LossArgs a, const T* h, const int* row, const LossInfo* info, float* staged, T* dh) {
  const int live = info->live;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* from = h + (int64_t)row[r] * a.ld_h;
    for (int c = threadIdx.x; c < a.dim; c += 256) {
      staged[r * a.dim + c] = r < live ? to_f32(from[c]) : 0.f;
      if (r >= live && dh) dh[(int64_t)row[r] * a.ld_dh + c] = from_f64<T>(0.0);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) stage_weight_kernel(LossArgs a, const T* w, float* staged) {
  for (int64_t v = blockIdx.x; v < a.vocab; v += gridDim.x)
    for (int c = threadIdx.x; c < a.dim; c += 256) staged[v * a.dim + c] = to_f32(w[v * a.ld_w + c]);
}

__device__ __forceinline__ float block_reduce(float v, bool max, float* warp_v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const float o = __shfl_xor_sync(0xffffffffu, v, d);
    v = max ? fmaxf(v, o) : v + o;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) warp_v[threadIdx.x >> 5] = v;
  __syncthreads();
  v = warp_v[0];
  for (int w = 1; w < 8; ++w) v = max ? fmaxf(v, warp_v[w]) : v + warp_v[w];
  return v;
}

__global__ void __launch_bounds__(256)
softmax_kernel(LossArgs a, float* z, int first, const int* row, const int* target, const float* g, const LossInfo* info, float* loss,
               double* part, bool gradient) {
  __shared__ float warp_v[8];
  const int r = blockIdx.x, i = first + r;
  float* at = z + (size_t)r * a.vocab;
  const bool on = i < info->live;
  if (!on) {
    if (gradient)
      for (int j = threadIdx.x; j < a.vocab; j += 256) at[j] = 0.f;
    if (threadIdx.x == 0) part[i] = 0.0;
    return;
  }
  float m = -INFINITY;
  for (int j = threadIdx.x; j < a.vocab; j += 256) m = fmaxf(m, at[j]);
  m = block_reduce(m, true, warp_v);
  float sum = 0.f;
  for (int j = threadIdx.x; j < a.vocab; j += 256) sum += expf(at[j] - m);
  sum = block_reduce(sum, false, warp_v);
  const int t = target[i];
  const float l = logf(sum) - (at[t] - m);
  __syncthreads();
  if (threadIdx.x == 0) {
    loss[row[i]] = l;
    part[i] = (double)g[i] * l;
  }
  if (gradient)
    for (int j = threadIdx.x; j < a.vocab; j += 256) {
      const float p = expf(at[j] - m) / sum;
      at[j] = g[i] * (j == t ? expm1f(-l) : p);
    }
}

__global__ void __launch_bounds__(256) total_kernel(const double* part, int64_t rows, float* total) {
  __shared__ double sums[256];
  double t = 0.0;
  for (int64_t i = threadIdx.x; i < rows; i += 256) t += part[i];
  sums[threadIdx.x] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    t = 0.0;
    for (int i = 0; i < 256; ++i) t += sums[i];
    *total = (float)t;
  }
}

__device__ __forceinline__ void put(float* at, float v) { *at = v; }
__device__ __forceinline__ void put(__nv_bfloat16* at, float v) { *at = __float2bfloat16_rn(v); }

template <typename T>
__global__ void __launch_bounds__(256)
store_rows_kernel(LossArgs a, const float* from, int first, int rows, const int* row, const LossInfo* info, T* dh) {
  const int live = info->live;
  for (int r = blockIdx.x; r < rows && first + r < live; r += gridDim.x)
    for (int c = threadIdx.x; c < a.dim; c += 256) put(dh + (int64_t)row[first + r] * a.ld_dh + c, from[(size_t)r * a.dim + c]);
}
template <typename G>
__global__ void __launch_bounds__(256) store_weight_kernel(LossArgs a, const float* from, G* dw) {
  for (int64_t v = blockIdx.x; v < a.vocab; v += gridDim.x)
    for (int c = threadIdx.x; c < a.dim; c += 256) put(dw + v * a.ld_dw + c, from[v * a.dim + c]);
}

struct LossWs {
  LossInfo* info;
  int *counts, *row, *target;
  float* g;
  double* part;
  float *h, *w, *z, *dh, *dw;
  int blocks, piece;
};
size_t loss_layout(const mw_token_loss_desc* d, bool gradient, char* base, LossWs* l) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* p = base + at;
    at += align_up(bytes, 256);
    return p;
  };
  const size_t n = (size_t)d->rows, v = (size_t)d->vocab, dim = (size_t)d->dim;
  l->blocks = ceil_div(d->rows, kIndexRows);
  int64_t piece = d->piece_rows;
  if (!piece) {
    piece = kPieceBytes / (4 * (int64_t)v);
    if (piece < 1024) piece = 1024;
  }
  l->piece = (int)(piece < d->rows ? piece : (d->rows ? d->rows : 1));
  l->info = (LossInfo*)take(sizeof(LossInfo));
  l->counts = (int*)take((size_t)l->blocks * 4);
  l->row = (int*)take(n * 4);
  l->target = (int*)take(n * 4);
  l->g = (float*)take(n * 4);
  l->part = (double*)take(n * 8);
  l->h = (float*)take(n * dim * 4);
  l->w = (float*)take(v * dim * 4);
  l->z = (float*)take((size_t)l->piece * v * 4);
  l->dh = (float*)take(gradient ? (size_t)l->piece * dim * 4 : 0);
  l->dw = (float*)take(gradient ? v * dim * 4 : 0);
  return at + 256;
}

mw_status check_loss(const mw_token_loss_desc* d) {
  if (!d || d->rows < 0 || d->vocab < 1 || d->dim < 1 || d->piece_rows < 0 || !isfinite(d->scale)) return MW_ERR_INVALID_ARG;
  if (d->index_bytes != 4 && d->index_bytes != 8) return MW_ERR_INVALID_ARG;
  if (d->rows > (1 << 24) || d->vocab > (1 << 24) || d->dim > (1 << 16) || d->dtype == MW_F64) return MW_ERR_UNSUPPORTED;
  if (d->dtype != MW_F32 && d->dtype != MW_BF16_F32ACC) return MW_ERR_INVALID_ARG;
  if (d->grad_dtype != 0 && d->grad_dtype != MW_F32 && d->grad_dtype != MW_BF16_F32ACC) return MW_ERR_INVALID_ARG;
  for (int64_t ld : {d->ld_h, d->ld_weight, d->ld_dh, d->ld_dweight})
    if (ld != 0 && ld < d->dim) return MW_ERR_INVALID_ARG;
  return MW_OK;
}

template <typename T, typename I>
mw_status loss_run(const mw_token_loss_desc* d, const T* h, const T* w, const I* targets, const float* weight, float* loss, float* total,
                   T* dh, void* dw, bool gradient, char* ws, cudaStream_t s) {
  LossArgs a;
  a.rows = d->rows; a.vocab = d->vocab; a.dim = d->dim;
  a.ld_h = d->ld_h ? d->ld_h : d->dim;
  a.ld_w = d->ld_weight ? d->ld_weight : d->dim;
  a.ld_dh = d->ld_dh ? d->ld_dh : d->dim;
  a.ld_dw = d->ld_dweight ? d->ld_dweight : d->dim;
  a.scale = (float)d->scale;
  LossWs l;
  loss_layout(d, gradient, ws, &l);
  MW_CUDA_OK(cudaMemsetAsync(ws, 0, sizeof(LossInfo), s));
  const unsigned wide = 148 * 8;
  if (a.rows > 0) {
    count_live_kernel<I><<<l.blocks, kIndexRows, 0, s>>>(targets, weight, a.rows, a.vocab, l.counts);
    index_live_kernel<I><<<l.blocks, kIndexRows, 0, s>>>(targets, weight, a.rows, a.vocab, l.counts, l.blocks, l.row, l.target, l.g, loss, l.info);
    stage_rows_kernel<T><<<wide, 256, 0, s>>>(a, h, l.row, l.info, l.h, dh);
    stage_weight_kernel<T><<<wide, 256, 0, s>>>(a, w, l.w);
    MW_TRY(launch_ok(4));
  }
  if (dw && a.rows == 0) MW_CUDA_OK(cudaMemsetAsync(l.dw, 0, (size_t)a.vocab * a.dim * 4, s));
  for (int64_t first = 0; first < a.rows; first += l.piece) {
    const int rows = (int)(a.rows - first < l.piece ? a.rows - first : l.piece);
    MW_TRY(gemm_simt<float>(0, 1, rows, a.vocab, a.dim, a.scale, l.h + first * a.dim, a.dim, l.w, a.dim, 0.0, l.z, a.vocab, s));
    softmax_kernel<<<rows, 256, 0, s>>>(a, l.z, (int)first, l.row, l.target, l.g, l.info, loss, l.part, gradient);
    MW_TRY(launch_ok());
    if (dh) {
      MW_TRY(gemm_simt<float>(0, 0, rows, a.dim, a.vocab, a.scale, l.z, a.vocab, l.w, a.dim, 0.0, l.dh, a.dim, s));
      store_rows_kernel<T><<<wide, 256, 0, s>>>(a, l.dh, (int)first, rows, l.row, l.info, dh);
      MW_TRY(launch_ok());
    }
    if (dw) MW_TRY(gemm_simt<float>(1, 0, a.vocab, a.dim, rows, a.scale, l.z, a.vocab, l.h + first * a.dim, a.dim, first ? 1.0 : 0.0, l.dw, a.dim, s));
  }
  if (dw) {
    const int32_t g = d->grad_dtype ? d->grad_dtype : d->dtype;
    if (g == MW_F32) store_weight_kernel<float><<<wide, 256, 0, s>>>(a, l.dw, (float*)dw);
    else store_weight_kernel<__nv_bfloat16><<<wide, 256, 0, s>>>(a, l.dw, (__nv_bfloat16*)dw);
    MW_TRY(launch_ok());
  }
  if (total) {
    total_kernel<<<1, 256, 0, s>>>(l.part, a.rows, total);
    MW_TRY(launch_ok());
  }
  return MW_OK;
}

mw_status loss_call(const mw_token_loss_desc* d, const void* h, const void* w, const void* targets, const float* weight, float* loss,
                    float* total, void* dh, void* dw, bool gradient, void* ws, size_t bytes, void* stream) {
  MW_TRY(check_loss(d));
  if (!w || (d->rows > 0 && (!h || !targets || !loss))) return MW_ERR_INVALID_ARG;
  const int64_t ld_h = d->ld_h ? d->ld_h : d->dim, ld_dh = d->ld_dh ? d->ld_dh : d->dim;
  if (dh == h && dh && ld_h != ld_dh) return MW_ERR_INVALID_ARG;
  LossWs l;
  if (!ws || ((uintptr_t)ws & 255u) || bytes < loss_layout(d, gradient, nullptr, &l)) return MW_ERR_WORKSPACE;
  cudaStream_t s = (cudaStream_t)stream;
  char* b = static_cast<char*>(ws);
  using bf = __nv_bfloat16;
  if (d->dtype == MW_F32) {
    if (d->index_bytes == 4) return loss_run<float, int32_t>(d, (const float*)h, (const float*)w, (const int32_t*)targets, weight, loss, total, (float*)dh, dw, gradient, b, s);
    return loss_run<float, int64_t>(d, (const float*)h, (const float*)w, (const int64_t*)targets, weight, loss, total, (float*)dh, dw, gradient, b, s);
  }
  if (d->index_bytes == 4) return loss_run<bf, int32_t>(d, (const bf*)h, (const bf*)w, (const int32_t*)targets, weight, loss, total, (bf*)dh, dw, gradient, b, s);
  return loss_run<bf, int64_t>(d, (const bf*)h, (const bf*)w, (const int64_t*)targets, weight, loss, total, (bf*)dh, dw, gradient, b, s);
}

}  // namespace
}  // namespace mw

extern "C" mw_status mw_token_loss_workspace_bytes(const mw_token_loss_desc* desc, int32_t gradient, size_t* bytes) {
  using namespace mw;
  if (!bytes || (gradient != 0 && gradient != 1)) return MW_ERR_INVALID_ARG;
  MW_TRY(check_loss(desc));
  LossWs l;
  *bytes = loss_layout(desc, gradient != 0, nullptr, &l);
  return MW_OK;
}

extern "C" mw_status mw_token_loss_forward(const mw_token_loss_desc* desc, const void* h, const void* weight, const void* targets,
                                           const float* row_weight, float* loss, float* total, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  return mw::loss_call(desc, h, weight, targets, row_weight, loss, total, nullptr, nullptr, false, workspace, workspace_bytes, stream);
}

extern "C" mw_status mw_token_loss_gradient(const mw_token_loss_desc* desc, const void* h, const void* weight, const void* targets,
                                            const float* row_weight, float* loss, float* total, void* dh, void* dweight,
                                            void* workspace, size_t workspace_bytes, void* stream) {
  return mw::loss_call(desc, h, weight, targets, row_weight, loss, total, dh, dweight, true, workspace, workspace_bytes, stream);
}

extern "C" mw_status mw_token_loss_status(const void* workspace, void* stream) {
  using namespace mw;
  if (!workspace) return MW_ERR_INVALID_ARG;
  DeviceStatus host;
  MW_CUDA_OK(cudaMemcpyAsync(&host, workspace, sizeof(host), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
  MW_CUDA_OK(cudaStreamSynchronize((cudaStream_t)stream));
  return (mw_status)host.code;
}
