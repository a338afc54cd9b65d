// Orthogonalised momentum update (mw_orth_*): Newton-Schulz products on the momentum of each weight.
#include <math.h>

#include <new>

#include "mw_common.cuh"

struct mw_orth {
  mw_orth_desc d;
  int m, n;            // shorter and longer side
  bool tall;           // rows > cols: the iterate is the transpose
  int steps;
  double c0, c1, c2;
};

namespace mw {
namespace {

constexpr int kNormBlocks = 64;       // partial sums of ||U||^2 per matrix

template <typename T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// M' = beta M + G, U and its sum of squares (double partials, one per block, fixed order)
template <typename TU>
__global__ void __launch_bounds__(256)
orth_momentum_kernel(const TU* __restrict__ u_in, const float* __restrict__ g, const float* mom, float* mom_out,
                     float* __restrict__ U, int64_t n, float beta, int nesterov, double* __restrict__ partials) {
  __shared__ double buf[8];
  double s = 0.0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float u;
    if (u_in) {
      u = to_f32(u_in[i]);
    } else {
      const float m2 = fmaf(beta, mom[i], g[i]);
      mom_out[i] = m2;
      u = nesterov ? fmaf(beta, m2, g[i]) : m2;
    }
    U[i] = u;
    s += (double)u * (double)u;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < 8; ++w) t += buf[w];
    partials[blockIdx.x] = t;
  }
}

// X_0 = U / ||U||_F, transposed when rows > cols
__global__ void __launch_bounds__(256)
orth_normalise_kernel(const float* __restrict__ U, int rows, int cols, int tall, const double* __restrict__ partials,
                      float* __restrict__ X) {
  double t = 0.0;
  for (int i = 0; i < kNormBlocks; ++i) t += partials[i];
  const double r = t > 0.0 ? 1.0 / sqrt(t) : (t == 0.0 ? 0.0 : t);      // NaN stays NaN
  const int64_t n = (int64_t)rows * cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const float v = (float)((double)U[i] * r);
    X[tall ? (i % cols) * (int64_t)rows + i / cols : i] = v;
  }
}

// W' = keep W - step X (params given), or X itself
template <typename T>
__global__ void __launch_bounds__(256)
orth_apply_kernel(const float* __restrict__ X, int rows, int cols, int tall, const T* params, T* out, float keep,
                  float step) {
  const int64_t n = (int64_t)rows * cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const float v = X[tall ? (i % cols) * (int64_t)rows + i / cols : i];
    out[i] = narrow<T>(params ? fmaf(-step, v, keep * to_f32(params[i])) : v);
  }
}

struct OrthWs {
  double* partials;
  float *U, *X, *Y, *A, *B;
};

size_t orth_layout(const mw_orth* p, char* base, OrthWs* w) {
  size_t off = 256;                       // device status
  auto take = [&](size_t bytes) {
    char* q = base ? base + off : nullptr;
    off += align_up(bytes, 256);
    return q;
  };
  const size_t mn = (size_t)p->m * p->n, mm = (size_t)p->m * p->m;
  OrthWs l;
  l.partials = reinterpret_cast<double*>(take(kNormBlocks * sizeof(double)));
  l.U = reinterpret_cast<float*>(take(mn * 4));
  l.X = reinterpret_cast<float*>(take(mn * 4));
  l.Y = reinterpret_cast<float*>(take(mn * 4));
  l.A = reinterpret_cast<float*>(take(mm * 4));
  l.B = reinterpret_cast<float*>(take(mm * 4));
  if (w) *w = l;
  return off;
}

template <typename T>
mw_status orth_run(mw_orth* p, const void* const* params, const void* const* grads, const void* const* momentum,
                   void* const* out, void* const* momentum_out, const void* const* project_in, double lr, double beta,
                   double wd, double scale, char* ws, cudaStream_t s) {
  OrthWs l;
  orth_layout(p, ws, &l);
  MW_CUDA_OK(cudaMemsetAsync(ws, 0, 256, s));
  const int rows = p->d.rows, cols = p->d.cols, m = p->m, n = p->n;
  const int64_t mn = (int64_t)m * n;
  const int wide = (int)((mn + 255) / 256 < 2048 ? (mn + 255) / 256 : 2048);
  for (int i = 0; i < p->d.count; ++i) {
    orth_momentum_kernel<T><<<kNormBlocks, 256, 0, s>>>(
        project_in ? static_cast<const T*>(project_in[i]) : nullptr, grads ? static_cast<const float*>(grads[i]) : nullptr,
        momentum ? static_cast<const float*>(momentum[i]) : nullptr,
        momentum_out ? static_cast<float*>(momentum_out[i]) : nullptr, l.U, mn, (float)beta, p->d.nesterov, l.partials);
    orth_normalise_kernel<<<wide, 256, 0, s>>>(l.U, rows, cols, p->tall, l.partials, l.X);
    MW_TRY(launch_ok(2));
    float *X = l.X, *Y = l.Y;
    for (int k = 0; k < p->steps; ++k) {
      MW_TRY(gemm_simt<float>(0, 1, m, m, n, 1.0, X, n, X, n, 0.0, l.A, m, s));
      MW_CUDA_OK(cudaMemcpyAsync(l.B, l.A, sizeof(float) * (size_t)m * m, cudaMemcpyDeviceToDevice, s));
      MW_TRY(gemm_simt<float>(0, 0, m, m, m, p->c2, l.A, m, l.A, m, p->c1, l.B, m, s));
      MW_CUDA_OK(cudaMemcpyAsync(Y, X, sizeof(float) * (size_t)mn, cudaMemcpyDeviceToDevice, s));
      MW_TRY(gemm_simt<float>(0, 0, m, n, m, 1.0, l.B, m, X, n, p->c0, Y, n, s));
      float* t = X;
      X = Y;
      Y = t;
    }
    orth_apply_kernel<T><<<wide, 256, 0, s>>>(X, rows, cols, p->tall, params ? static_cast<const T*>(params[i]) : nullptr,
                                              static_cast<T*>(out[i]), (float)(1.0 - lr * wd), (float)(lr * scale));
    MW_TRY(launch_ok());
  }
  return MW_OK;
}

bool all_set(const void* const* p, int n) {
  if (!p) return false;
  for (int i = 0; i < n; ++i)
    if (!p[i]) return false;
  return true;
}

mw_status check_ws(const mw_orth* p, const void* ws, size_t bytes) {
  return (!ws || ((uintptr_t)ws & 255u) || bytes < orth_layout(p, nullptr, nullptr)) ? MW_ERR_WORKSPACE : MW_OK;
}

}  // namespace
}  // namespace mw

extern "C" mw_status mw_orth_create(const mw_orth_desc* desc, mw_orth** out) {
  using namespace mw;
  if (!desc || !out) return MW_ERR_INVALID_ARG;
  *out = nullptr;
  const mw_orth_desc& d = *desc;
  if (d.rows < 1 || d.cols < 1 || d.count < 1 || d.steps < 0 || d.steps > 16 || d.terms < 0 || d.terms > 2 ||
      d.reserved != 0 || (d.nesterov != 0 && d.nesterov != 1))
    return MW_ERR_INVALID_ARG;
  if (d.prec == MW_F64) return MW_ERR_UNSUPPORTED;
  if (d.prec != MW_F32 && d.prec != MW_BF16_F32ACC) return MW_ERR_INVALID_ARG;
  for (double c : d.coef)
    if (!isfinite(c)) return MW_ERR_INVALID_ARG;
  mw_orth* p = new (std::nothrow) mw_orth();
  if (!p) return MW_ERR_CUDA;
  p->d = d;
  p->tall = d.rows > d.cols;
  p->m = p->tall ? d.cols : d.rows;
  p->n = p->tall ? d.rows : d.cols;
  p->steps = d.steps ? d.steps : 5;
  const bool given = d.coef[0] != 0.0 || d.coef[1] != 0.0 || d.coef[2] != 0.0;
  p->c0 = given ? d.coef[0] : 3.4445;
  p->c1 = given ? d.coef[1] : -4.7750;
  p->c2 = given ? d.coef[2] : 2.0315;
  *out = p;
  return MW_OK;
}

extern "C" void mw_orth_destroy(mw_orth* plan) { delete plan; }

extern "C" mw_status mw_orth_workspace_bytes(const mw_orth* plan, size_t* bytes) {
  if (!plan || !bytes) return MW_ERR_INVALID_ARG;
  *bytes = mw::orth_layout(plan, nullptr, nullptr);
  return MW_OK;
}

extern "C" mw_status mw_orth_step(mw_orth* plan, const void* const* params, const void* const* grads,
                                  const void* const* momentum, void* const* params_out, void* const* momentum_out,
                                  double lr, double beta, double weight_decay, double scale, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  using namespace mw;
  if (!plan || !isfinite(lr) || !isfinite(beta) || !isfinite(weight_decay) || !isfinite(scale)) return MW_ERR_INVALID_ARG;
  const int n = plan->d.count;
  if (!all_set(params, n) || !all_set(grads, n) || !all_set(momentum, n) || !all_set(params_out, n) ||
      !all_set(momentum_out, n))
    return MW_ERR_INVALID_ARG;
  MW_TRY(check_ws(plan, workspace, workspace_bytes));
  cudaStream_t s = (cudaStream_t)stream;
  char* ws = static_cast<char*>(workspace);
  return plan->d.prec == MW_F32
             ? orth_run<float>(plan, params, grads, momentum, params_out, momentum_out, nullptr, lr, beta, weight_decay, scale, ws, s)
             : orth_run<__nv_bfloat16>(plan, params, grads, momentum, params_out, momentum_out, nullptr, lr, beta, weight_decay,
                                       scale, ws, s);
}

extern "C" mw_status mw_orth_project(mw_orth* plan, const void* const* in, void* const* out, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  using namespace mw;
  if (!plan || !all_set(in, plan->d.count) || !all_set(out, plan->d.count)) return MW_ERR_INVALID_ARG;
  MW_TRY(check_ws(plan, workspace, workspace_bytes));
  cudaStream_t s = (cudaStream_t)stream;
  char* ws = static_cast<char*>(workspace);
  return plan->d.prec == MW_F32 ? orth_run<float>(plan, nullptr, nullptr, nullptr, out, nullptr, in, 0, 0, 0, 0, ws, s)
                                : orth_run<__nv_bfloat16>(plan, nullptr, nullptr, nullptr, out, nullptr, in, 0, 0, 0, 0, ws, s);
}

extern "C" mw_status mw_orth_status(const mw_orth* plan, const void* workspace, void* stream) {
  using namespace mw;
  if (!plan || !workspace) return MW_ERR_INVALID_ARG;
  DeviceStatus host;
  MW_CUDA_OK(cudaMemcpyAsync(&host, workspace, sizeof(host), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
  MW_CUDA_OK(cudaStreamSynchronize((cudaStream_t)stream));
  return (mw_status)host.code;
}
