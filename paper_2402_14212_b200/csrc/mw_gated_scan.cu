// Gated linear recurrence (mw_gated_scan_*), per channel:
//   a = sigmoid(f),  u = 1 - a or sqrt(1 - a^2),  h_t = r_t a_t h_{t-1} + u_t v_t
// backward, with g_t the whole cotangent of h_t:
//   g_t = dy_t + r_{t+1} a_{t+1} g_{t+1},  dv = u g,  df = a (1 - a) g (r h_{t-1} + u'(a) v)
#include "mw_common.cuh"

namespace mw {
namespace {

constexpr int kEvery = MW_SCAN_STATE_EVERY;

struct ScanArgs {
  int B, T, D;
  int64_t v_b, v_t, f_b, f_t, y_b, y_t, dv_b, dv_t, df_b, df_t;
  const void *v, *f, *dy;
  const uint8_t* reset;
  const int32_t* lengths;
  const float *h0, *dh_last, *states_in;
  void *y, *dv, *df;
  float *h_last, *states, *dh0;
};

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// a = sigmoid(f) and w = 1 - a, each to full relative accuracy at either end (one exponential, one
// reciprocal: 1 - a formed by subtraction would lose the slow channels, where a is close to 1)
__device__ __forceinline__ void gate_of(float f, float& a, float& w) {
  const float e = __expf(-fabsf(f)), big = __fdividef(1.f, 1.f + e), small = e * big;
  a = f >= 0.f ? big : small;
  w = f >= 0.f ? small : big;
  if (isnan(f)) a = w = f;
}
template <int GATE>
__device__ __forceinline__ float input_of(float a, float w) {
  return GATE == MW_SCAN_COMPLEMENT ? w : sqrtf(w * (1.f + a));
}
// a (1 - a) u'(a): -a w, or -a^2 w / u = -a^2 sqrt(w / (1 + a)) (finite where u is zero)
template <int GATE>
__device__ __forceinline__ float input_slope(float a, float w) {
  return GATE == MW_SCAN_COMPLEMENT ? -a * w : -a * a * sqrtf(__fdividef(w, 1.f + a));
}

__device__ __forceinline__ int length_of(const ScanArgs& p, int b) {
  if (p.lengths == nullptr) return p.T;
  const int n = p.lengths[b];
  return n < 0 ? 0 : (n < p.T ? n : p.T);
}

// one thread per channel walks the whole sequence
template <typename T, int GATE>
__global__ void __launch_bounds__(128)
scan_walk_kernel(const ScanArgs p) {
  const int c = blockIdx.x * 128 + threadIdx.x, b = blockIdx.y;
  if (c >= p.D) return;
  const int n = length_of(p, b);
  const T* v = static_cast<const T*>(p.v) + b * p.v_b + c;
  const T* f = static_cast<const T*>(p.f) + b * p.f_b + c;
  T* y = static_cast<T*>(p.y) + b * p.y_b + c;
  const int64_t bc = (int64_t)b * p.D + c;
  float h = p.h0 ? p.h0[bc] : 0.f;
  const int64_t nst = (p.T + kEvery - 1) / kEvery;
  for (int t = 0; t < p.T; ++t) {
    if (p.states && t % kEvery == 0) p.states[(b * nst + t / kEvery) * p.D + c] = h;
    float out = 0.f;
    if (t < n) {
      float a, w;
      gate_of(to_f32(f[t * p.f_t]), a, w);
      const float u = input_of<GATE>(a, w);
      const bool cut = p.reset && p.reset[(int64_t)b * p.T + t];
      h = cut ? u * to_f32(v[t * p.v_t]) : fmaf(a, h, u * to_f32(v[t * p.v_t]));
      out = h;
    }
    y[t * p.y_t] = from_f32<T>(out);
  }
  if (p.h_last) p.h_last[bc] = h;
}

template <typename T, int GATE>
__global__ void __launch_bounds__(128)
scan_walk_back_kernel(const ScanArgs p) {
  const int c = blockIdx.x * 128 + threadIdx.x, b = blockIdx.y;
  if (c >= p.D) return;
  const int n = length_of(p, b);
  const T* v = static_cast<const T*>(p.v) + b * p.v_b + c;
  const T* f = static_cast<const T*>(p.f) + b * p.f_b + c;
  const T* dy = p.dy ? static_cast<const T*>(p.dy) + b * p.y_b + c : nullptr;
  T* dv = static_cast<T*>(p.dv) + b * p.dv_b + c;
  T* df = static_cast<T*>(p.df) + b * p.df_b + c;
  const int64_t bc = (int64_t)b * p.D + c;
  const int64_t nst = (p.T + kEvery - 1) / kEvery;
  float g = p.dh_last ? p.dh_last[bc] : 0.f;       // cotangent of the state after the current step
  for (int i = (int)nst - 1; i >= 0; --i) {
    const int t0 = i * kEvery, len = min(kEvery, p.T - t0);
    float before[kEvery];
    float h = p.states_in[(b * nst + i) * p.D + c];
    for (int j = 0; j < len; ++j) {
      const int t = t0 + j;
      const bool cut = p.reset && p.reset[(int64_t)b * p.T + t];
      before[j] = cut ? 0.f : h;
      if (t < n) {
        float a, w;
        gate_of(to_f32(f[t * p.f_t]), a, w);
        h = fmaf(a, before[j], input_of<GATE>(a, w) * to_f32(v[t * p.v_t]));
      }
    }
    for (int j = len - 1; j >= 0; --j) {
      const int t = t0 + j;
      float ov = 0.f, of = 0.f;
      if (t < n) {
        float a, w;
        gate_of(to_f32(f[t * p.f_t]), a, w);
        if (dy) g += to_f32(dy[t * p.y_t]);
        ov = input_of<GATE>(a, w) * g;
        of = g * fmaf(a * w, before[j], input_slope<GATE>(a, w) * to_f32(v[t * p.v_t]));
        const bool cut = p.reset && p.reset[(int64_t)b * p.T + t];
        g = cut ? 0.f : a * g;
      }
      dv[t * p.dv_t] = from_f32<T>(ov);
      df[t * p.df_t] = from_f32<T>(of);
    }
  }
  if (p.dh0) p.dh0[bc] = g;
}

mw_status check_desc(const mw_gated_scan_desc* d) {
  if (!d || d->batch < 0 || d->length < 0 || d->channels < 1 || d->reserved != 0) return MW_ERR_INVALID_ARG;
  if (d->input_gate != MW_SCAN_COMPLEMENT && d->input_gate != MW_SCAN_ENERGY) return MW_ERR_INVALID_ARG;
  if (d->dtype == 0) return MW_ERR_UNSUPPORTED;
  if (d->dtype != 1 && d->dtype != 2) return MW_ERR_INVALID_ARG;
  if (d->batch > 65535) return MW_ERR_UNSUPPORTED;
  return MW_OK;
}

// a pair of strides, dense when both are zero; steps and sequences must not overlap
bool strides(const mw_gated_scan_desc* d, int64_t b_in, int64_t t_in, int64_t& b, int64_t& t) {
  b = b_in;
  t = t_in;
  if (b == 0 && t == 0) {
    t = d->channels;
    b = t * d->length;
    return true;
  }
  if (d->length > 1 && t < d->channels) return false;
  return d->batch <= 1 || b >= d->channels;
}

mw_status fill_scan(const mw_gated_scan_desc* d, ScanArgs& p) {
  MW_TRY(check_desc(d));
  p = ScanArgs();
  p.B = d->batch; p.T = d->length; p.D = d->channels;
  if (!strides(d, d->v_batch, d->v_time, p.v_b, p.v_t) || !strides(d, d->f_batch, d->f_time, p.f_b, p.f_t) ||
      !strides(d, d->y_batch, d->y_time, p.y_b, p.y_t) || !strides(d, d->dv_batch, d->dv_time, p.dv_b, p.dv_t) ||
      !strides(d, d->df_batch, d->df_time, p.df_b, p.df_t))
    return MW_ERR_INVALID_ARG;
  return MW_OK;
}

template <typename T, int GATE>
mw_status run_scan(const ScanArgs& p, bool backward, cudaStream_t s) {
  const dim3 grid((unsigned)ceil_div(p.D, 128), (unsigned)p.B);
  if (backward) scan_walk_back_kernel<T, GATE><<<grid, 128, 0, s>>>(p);
  else scan_walk_kernel<T, GATE><<<grid, 128, 0, s>>>(p);
  return launch_ok();
}

mw_status dispatch_scan(const mw_gated_scan_desc* d, const ScanArgs& p, bool backward, cudaStream_t s) {
  if (d->dtype == 1)
    return d->input_gate == MW_SCAN_COMPLEMENT ? run_scan<float, MW_SCAN_COMPLEMENT>(p, backward, s)
                                               : run_scan<float, MW_SCAN_ENERGY>(p, backward, s);
  return d->input_gate == MW_SCAN_COMPLEMENT ? run_scan<__nv_bfloat16, MW_SCAN_COMPLEMENT>(p, backward, s)
                                             : run_scan<__nv_bfloat16, MW_SCAN_ENERGY>(p, backward, s);
}

}  // namespace
}  // namespace mw

extern "C" mw_status mw_gated_scan_states_bytes(const mw_gated_scan_desc* desc, size_t* bytes) {
  using namespace mw;
  if (!bytes) return MW_ERR_INVALID_ARG;
  MW_TRY(check_desc(desc));
  *bytes = sizeof(float) * (size_t)desc->batch * (((size_t)desc->length + kEvery - 1) / kEvery) * (size_t)desc->channels;
  return MW_OK;
}

extern "C" mw_status mw_gated_scan_forward(const mw_gated_scan_desc* desc, const void* v, const void* f,
                                           const uint8_t* reset, const int32_t* lengths, const float* h0, void* y,
                                           float* h_last, float* states, void* stream) {
  using namespace mw;
  ScanArgs p;
  MW_TRY(fill_scan(desc, p));
  cudaStream_t s = (cudaStream_t)stream;
  if (p.B == 0) return MW_OK;
  if (p.T == 0) {
    // the state passes through
    if (h_last && h_last != h0) {
      const size_t n = sizeof(float) * (size_t)p.B * (size_t)p.D;
      if (h0) MW_CUDA_OK(cudaMemcpyAsync(h_last, h0, n, cudaMemcpyDeviceToDevice, s));
      else MW_CUDA_OK(cudaMemsetAsync(h_last, 0, n, s));
    }
    return MW_OK;
  }
  if (!v || !f || !y) return MW_ERR_INVALID_ARG;
  p.v = v; p.f = f; p.reset = reset; p.lengths = lengths; p.h0 = h0; p.y = y; p.h_last = h_last; p.states = states;
  return dispatch_scan(desc, p, false, s);
}

extern "C" mw_status mw_gated_scan_backward(const mw_gated_scan_desc* desc, const void* v, const void* f,
                                            const uint8_t* reset, const int32_t* lengths, const float* states,
                                            const void* dy, const float* dh_last, void* dv, void* df, float* dh0,
                                            void* stream) {
  using namespace mw;
  ScanArgs p;
  MW_TRY(fill_scan(desc, p));
  cudaStream_t s = (cudaStream_t)stream;
  if (p.B == 0) return MW_OK;
  if (p.T == 0) {
    if (dh0 && dh0 != dh_last) {
      const size_t n = sizeof(float) * (size_t)p.B * (size_t)p.D;
      if (dh_last) MW_CUDA_OK(cudaMemcpyAsync(dh0, dh_last, n, cudaMemcpyDeviceToDevice, s));
      else MW_CUDA_OK(cudaMemsetAsync(dh0, 0, n, s));
    }
    return MW_OK;
  }
  if (!v || !f || !states || !dv || !df) return MW_ERR_INVALID_ARG;
  p.v = v; p.f = f; p.reset = reset; p.lengths = lengths; p.states_in = states; p.dy = dy; p.dh_last = dh_last;
  p.dv = dv; p.df = df; p.dh0 = dh0;
  return dispatch_scan(desc, p, true, s);
}
