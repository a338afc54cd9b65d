// Residual sum of a block with the norms around it (mw_residual_norm_*):
//   p = w_post b / rms(b),  x' = x + scale silu(z) p,  n = w_pre x' / rms(x')
// One pass over each row in both directions: a group of G threads holds the row in registers, so
// every tensor crosses HBM once (forward 10 bytes an element in bf16, backward 16).
#include "mw_common.cuh"

namespace mw {
namespace {

constexpr int kMaxCols = 32768;
constexpr int kNormThreads = 256;

struct NormArgs {
  int64_t rows;
  int cols;
  float eps;
  int64_t ld_x, ld_b, ld_z;
  const void *x, *b, *z;
  const float *w_post, *scale, *w_pre;
  void *x_out, *n;
  float* inv_rms;
  // backward
  const float* rms_in;
  const void *dx_out, *dn;
  void *dx, *db, *dz;
  float* partials;      // [grid][3][cols]
};

// VEC consecutive elements of a row as floats
template <typename T, int VEC>
struct Pack;
template <>
struct Pack<float, 1> {
  using Raw = float;
  static __device__ __forceinline__ void get(Raw r, float (&v)[1]) { v[0] = r; }
  static __device__ __forceinline__ Raw put(const float (&v)[1]) { return v[0]; }
  static __device__ __forceinline__ Raw zero() { return 0.f; }
};
template <>
struct Pack<float, 4> {
  using Raw = float4;
  static __device__ __forceinline__ void get(Raw r, float (&v)[4]) { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
  static __device__ __forceinline__ Raw put(const float (&v)[4]) { return make_float4(v[0], v[1], v[2], v[3]); }
  static __device__ __forceinline__ Raw zero() { return make_float4(0.f, 0.f, 0.f, 0.f); }
};
template <>
struct Pack<__nv_bfloat16, 1> {
  using Raw = __nv_bfloat16;
  static __device__ __forceinline__ void get(Raw r, float (&v)[1]) { v[0] = __bfloat162float(r); }
  static __device__ __forceinline__ Raw put(const float (&v)[1]) { return __float2bfloat16_rn(v[0]); }
  static __device__ __forceinline__ Raw zero() { return __float2bfloat16_rn(0.f); }
};
template <>
struct Pack<__nv_bfloat16, 8> {
  using Raw = uint4;
  static __device__ __forceinline__ void get(Raw r, float (&v)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ Raw put(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ Raw zero() { return make_uint4(0u, 0u, 0u, 0u); }
};

template <int VEC>
__device__ __forceinline__ void load_weight(const float* w, int col, float (&v)[VEC]) {
  if (w == nullptr) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = 1.f;
  } else if (VEC == 1) {
    v[0] = __ldg(w + col);
  } else {
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i) {
      const float4 t = __ldg(reinterpret_cast<const float4*>(w + col) + i);
      v[4 * i] = t.x; v[4 * i + 1] = t.y; v[4 * i + 2] = t.z; v[4 * i + 3] = t.w;
    }
  }
}

__device__ __forceinline__ float sigmoid_f(float z) {
  const float e = __expf(-fabsf(z)), big = __frcp_rn(1.f + e);
  return z >= 0.f ? big : e * big;
}

// sums over the G threads that share a row (G a power of two, 32..1024, aligned inside the block);
// `buf` double-buffers by call so that one barrier a reduction is enough
template <int G, int N>
__device__ __forceinline__ void row_sum(float (&s)[N], float* buf) {
#pragma unroll
  for (int o = 16; o; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
  if (G > 32) {
    constexpr int W = G / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = warp / W * W;
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) buf[warp * N + i] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] += buf[(first + w) * N + i];
  }
}

template <typename T, int VEC, int G, int K>
__global__ void __launch_bounds__(G > kNormThreads ? G : kNormThreads)
norm_forward_kernel(const NormArgs a) {
  using P = Pack<T, VEC>;
  using Raw = typename P::Raw;
  constexpr int kRows = (G > kNormThreads ? G : kNormThreads) / G;
  __shared__ float buf[2][32];
  const int t = threadIdx.x % G;
  int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
  const bool live = row < a.rows;
  if (!live) row = a.rows - 1;                // takes part in the barriers, stores nothing
  const int D = a.cols;
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  const T* b = static_cast<const T*>(a.b);
  const T* z = static_cast<const T*>(a.z);
  if (b) b += row * a.ld_b;
  if (z) z += row * a.ld_z;
  Raw rx[K], rb[K], rz[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * G + t) * VEC;
    rx[k] = rb[k] = rz[k] = P::zero();
    if (c < D) {
      rx[k] = *reinterpret_cast<const Raw*>(x + c);
      if (b) rb[k] = *reinterpret_cast<const Raw*>(b + c);
      if (z) rz[k] = *reinterpret_cast<const Raw*>(z + c);
    }
  }
  float inv_b = 1.f;
  if (b && a.w_post) {
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float v[VEC];
      P::get(rb[k], v);
#pragma unroll
      for (int i = 0; i < VEC; ++i) s[0] = fmaf(v[i], v[i], s[0]);
    }
    row_sum<G, 1>(s, buf[0]);
    inv_b = rsqrtf(s[0] / (float)D + a.eps);
  }
  float y[K][VEC];
  float s[1] = {0.f};
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * G + t) * VEC;
    P::get(rx[k], y[k]);
    if (b && c < D) {
      float vb[VEC], vz[VEC], wp[VEC], sc[VEC];
      P::get(rb[k], vb);
      load_weight<VEC>(a.w_post, c, wp);
      load_weight<VEC>(a.scale, c, sc);
      P::get(rz[k], vz);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float gate = z ? vz[i] * sigmoid_f(vz[i]) : 1.f;
        y[k][i] = fmaf(sc[i] * gate, vb[i] * inv_b * wp[i], y[k][i]);
      }
    }
    if (live && a.x_out && c < D)
      *reinterpret_cast<Raw*>(static_cast<T*>(a.x_out) + row * D + c) = P::put(y[k]);
#pragma unroll
    for (int i = 0; i < VEC; ++i) s[0] = fmaf(y[k][i], y[k][i], s[0]);
  }
  float inv_x = 1.f;
  if (a.w_pre) {
    row_sum<G, 1>(s, buf[1]);
    inv_x = rsqrtf(s[0] / (float)D + a.eps);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + t) * VEC;
      if (live && c < D) {
        float w[VEC], o[VEC];
        load_weight<VEC>(a.w_pre, c, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) o[i] = y[k][i] * inv_x * w[i];
        *reinterpret_cast<Raw*>(static_cast<T*>(a.n) + row * D + c) = P::put(o);
      }
    }
  }
  if (live && a.inv_rms && t == 0) {
    a.inv_rms[row] = inv_b;
    a.inv_rms[a.rows + row] = inv_x;
  }
}

// Backward of a row, with xh = x' / rms, bh = b / rms, q = dn w_pre, tau = scale silu(z) w_post bh:
//   dx  = dx_out + (q - xh m1) / rms(x'),             m1 = mean(q xh)
//   dp  = dx scale silu(z);  db = (dp w_post - bh m2) / rms(b),  m2 = mean(dp w_post bh) = mean(dx tau)
// m2 needs dx, which needs m1; written out, mean(dx tau) = mean((dx_out + q/rms) tau) - m1 mean(xh tau)/rms,
// so the three sums go through ONE reduction a row.
// The grid is persistent; a thread meets the same columns in every row and keeps its share of the
// weight gradients in registers, partials meet in fixed order in norm_reduce_kernel.
template <typename T, int VEC, int G, int K>
__global__ void __launch_bounds__(G > kNormThreads ? G : kNormThreads)
norm_backward_kernel(const NormArgs a) {
  using P = Pack<T, VEC>;
  using Raw = typename P::Raw;
  constexpr int kThreads = G > kNormThreads ? G : kNormThreads;
  constexpr int kRows = kThreads / G;
  __shared__ float buf[2][96];
  const int t = threadIdx.x % G, sub = threadIdx.x / G;
  const int D = a.cols;
  const bool has_b = a.b != nullptr, has_z = a.z != nullptr;
  float acc_wp[K][VEC], acc_sc[K][VEC], acc_wn[K][VEC];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc_wp[k][i] = acc_sc[k][i] = acc_wn[k][i] = 0.f;
  int flip = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.rows; base += (int64_t)gridDim.x * kRows) {
    int64_t row = base + sub;
    const bool live = row < a.rows;
    if (!live) row = a.rows - 1;
    const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
    const T* b = has_b ? static_cast<const T*>(a.b) + row * a.ld_b : nullptr;
    const T* z = has_z ? static_cast<const T*>(a.z) + row * a.ld_z : nullptr;
    const T* go = a.dx_out ? static_cast<const T*>(a.dx_out) + row * D : nullptr;
    const T* gn = a.dn ? static_cast<const T*>(a.dn) + row * D : nullptr;
    Raw rx[K], rb[K], rz[K], ro[K], rn[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + t) * VEC;
      rx[k] = rb[k] = rz[k] = ro[k] = rn[k] = P::zero();
      if (c < D) {
        rx[k] = *reinterpret_cast<const Raw*>(x + c);
        if (b) rb[k] = *reinterpret_cast<const Raw*>(b + c);
        if (z) rz[k] = *reinterpret_cast<const Raw*>(z + c);
        if (go) ro[k] = *reinterpret_cast<const Raw*>(go + c);
        if (gn) rn[k] = *reinterpret_cast<const Raw*>(gn + c);
      }
    }
    const float inv_b = a.rms_in[row], inv_x = a.rms_in[a.rows + row];
    const float inv_d = 1.f / (float)D;
    float s[3] = {0.f, 0.f, 0.f};
    // one element's quantities, formed again after the reduction (cheaper than keeping them)
    struct El { float xh, bh, gate, dgate, q, go; };
    auto element = [&](float vx, float vb, float vz, float vo, float vn, float wp, float sc, float wn) {
      El e;
      float sig = 1.f;
      e.gate = 1.f;
      e.dgate = 0.f;
      if (has_z) {
        sig = sigmoid_f(vz);
        e.gate = vz * sig;
        e.dgate = sig * fmaf(vz, 1.f - sig, 1.f);
      }
      e.bh = vb * inv_b;
      e.xh = (has_b ? fmaf(sc * e.gate, e.bh * wp, vx) : vx) * inv_x;
      e.q = vn * wn;
      e.go = vo;
      return e;
    };
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + t) * VEC;
      if (c >= D) continue;
      float vx[VEC], vb[VEC], vz[VEC], vo[VEC], vn[VEC], wp[VEC], sc[VEC], wn[VEC];
      P::get(rx[k], vx); P::get(rb[k], vb); P::get(rz[k], vz); P::get(ro[k], vo); P::get(rn[k], vn);
      load_weight<VEC>(a.w_post, c, wp); load_weight<VEC>(a.scale, c, sc); load_weight<VEC>(a.w_pre, c, wn);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const El e = element(vx[i], vb[i], vz[i], vo[i], vn[i], wp[i], sc[i], wn[i]);
        const float tau = sc[i] * e.gate * wp[i] * e.bh;
        s[0] = fmaf(e.q, e.xh, s[0]);
        s[1] = fmaf(fmaf(e.q, inv_x, e.go), tau, s[1]);
        s[2] = fmaf(e.xh, tau, s[2]);
      }
    }
    row_sum<G, 3>(s, buf[flip]);
    flip ^= 1;
    const float m1 = a.w_pre ? s[0] * inv_d : 0.f;
    const float m2 = (s[1] - m1 * inv_x * s[2]) * inv_d;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + t) * VEC;
      if (c >= D || !live) continue;
      float vx[VEC], vb[VEC], vz[VEC], vo[VEC], vn[VEC], wp[VEC], sc[VEC], wn[VEC];
      P::get(rx[k], vx); P::get(rb[k], vb); P::get(rz[k], vz); P::get(ro[k], vo); P::get(rn[k], vn);
      load_weight<VEC>(a.w_post, c, wp); load_weight<VEC>(a.scale, c, sc); load_weight<VEC>(a.w_pre, c, wn);
      float ox[VEC], ob[VEC], oz[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const El e = element(vx[i], vb[i], vz[i], vo[i], vn[i], wp[i], sc[i], wn[i]);
        const float dx = a.w_pre ? fmaf(inv_x, e.q - e.xh * m1, e.go) : e.go;
        ox[i] = dx;
        if (has_b) {
          const float p = e.bh * wp[i], dxg = dx * e.gate, dp = dxg * sc[i];
          ob[i] = a.w_post ? inv_b * (dp * wp[i] - e.bh * m2) : dp;
          oz[i] = dx * sc[i] * p * e.dgate;
          acc_wp[k][i] = fmaf(dp, e.bh, acc_wp[k][i]);
          acc_sc[k][i] = fmaf(dxg, p, acc_sc[k][i]);
        }
        acc_wn[k][i] = fmaf(vn[i], e.xh, acc_wn[k][i]);
      }
      if (a.dx) *reinterpret_cast<Raw*>(static_cast<T*>(a.dx) + row * D + c) = P::put(ox);
      if (a.db) *reinterpret_cast<Raw*>(static_cast<T*>(a.db) + row * D + c) = P::put(ob);
      if (a.dz) *reinterpret_cast<Raw*>(static_cast<T*>(a.dz) + row * D + c) = P::put(oz);
    }
  }
  if (a.partials == nullptr) return;
  // rows that share a block meet here; block partials meet in norm_reduce_kernel
  float* out = a.partials + ((int64_t)blockIdx.x * kRows + sub) * 3 * D;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * G + t) * VEC;
    if (c >= D) continue;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      out[c + i] = acc_wp[k][i];
      out[D + c + i] = acc_sc[k][i];
      out[2 * D + c + i] = acc_wn[k][i];
    }
  }
}

// sums of `parts` rows of [3][D], in fixed order: a block owns 32 columns, its 8 warps the parts w, w+8, ...
__global__ void __launch_bounds__(256)
norm_reduce_kernel(const float* __restrict__ partials, int parts, int D, float* __restrict__ dw_post,
                   float* __restrict__ dscale, float* __restrict__ dw_pre) {
  __shared__ float buf[8][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane, which = blockIdx.y;
  float* out = which == 0 ? dw_post : (which == 1 ? dscale : dw_pre);
  if (out == nullptr) return;
  float s = 0.f;
  if (c < D)
    for (int p = warp; p < parts; p += 8) s += partials[((int64_t)p * 3 + which) * D + c];
  buf[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < D) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += buf[w][lane];
    out[c] = v;
  }
}

// threads that share a row of `cols`: as few as keep 16 values a thread (32 beyond 16384 columns)
int group_of(int cols) {
  int g = 32;
  while (g < 1024 && g * 16 < cols) g <<= 1;
  return g;
}
int rows_per_block(int g) { return g > kNormThreads ? 1 : kNormThreads / g; }

int norm_sms() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
    cudaGetLastError();
    n = 148;
  }
  return n;
}
// blocks of the backward pass: two blocks of 256 threads (or one larger) an SM
int64_t backward_blocks(int64_t rows, int cols) {
  const int g = group_of(cols), r = rows_per_block(g);
  const int64_t need = (rows + r - 1) / r, most = (int64_t)norm_sms() * (g > 512 ? 1 : 2);
  return need < most ? need : most;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

template <typename T, int VEC, int G, int K>
mw_status launch_norm(const NormArgs& a, bool backward, cudaStream_t s) {
  const int threads = G > kNormThreads ? G : kNormThreads, r = threads / G;
  const int64_t need = (a.rows + r - 1) / r;
  if (backward)
    norm_backward_kernel<T, VEC, G, K><<<(unsigned)backward_blocks(a.rows, a.cols), threads, 0, s>>>(a);
  else
    norm_forward_kernel<T, VEC, G, K><<<(unsigned)need, threads, 0, s>>>(a);
  return launch_ok();
}

template <typename T, int VEC>
mw_status dispatch_norm(const NormArgs& a, bool backward, cudaStream_t s) {
  constexpr int K = 16 / VEC;
  switch (group_of(a.cols)) {
    case 32: return launch_norm<T, VEC, 32, K>(a, backward, s);
    case 64: return launch_norm<T, VEC, 64, K>(a, backward, s);
    case 128: return launch_norm<T, VEC, 128, K>(a, backward, s);
    case 256: return launch_norm<T, VEC, 256, K>(a, backward, s);
    case 512: return launch_norm<T, VEC, 512, K>(a, backward, s);
    default:
      return a.cols <= 16384 ? launch_norm<T, VEC, 1024, K>(a, backward, s)
                             : launch_norm<T, VEC, 1024, 2 * K>(a, backward, s);
  }
}

// 16-byte accesses where every row of every tensor starts on such a boundary, else element by element
template <typename T, int VEC>
mw_status run_norm(const NormArgs& a, bool backward, cudaStream_t s) {
  const void* ptrs[] = {a.x, a.b, a.z, a.w_post, a.scale, a.w_pre, a.x_out, a.n, a.dx_out, a.dn, a.dx, a.db, a.dz};
  bool wide = a.cols % VEC == 0 && a.ld_x % VEC == 0 && a.ld_b % VEC == 0 && a.ld_z % VEC == 0;
  for (const void* p : ptrs) wide = wide && aligned16(p);
  return wide ? dispatch_norm<T, VEC>(a, backward, s) : dispatch_norm<T, 1>(a, backward, s);
}

mw_status fill_norm(const mw_residual_norm_desc* d, const void* x, const void* b, const void* z, const float* w_post,
                    const float* scale, const float* w_pre, NormArgs& a) {
  if (!d || d->rows < 0 || d->cols < 1 || !(d->eps > 0.0)) return MW_ERR_INVALID_ARG;
  if (d->dtype != 1 && d->dtype != 2) return d->dtype == 0 ? MW_ERR_UNSUPPORTED : MW_ERR_INVALID_ARG;
  if (d->cols > kMaxCols || d->rows > ((int64_t)1 << 31) - 1) return MW_ERR_UNSUPPORTED;
  a = NormArgs();
  a.rows = d->rows;
  a.cols = d->cols;
  a.eps = (float)d->eps;
  a.ld_x = d->ld_x ? d->ld_x : d->cols;
  a.ld_b = d->ld_b ? d->ld_b : d->cols;
  a.ld_z = d->ld_z ? d->ld_z : d->cols;
  if (a.ld_x < d->cols || a.ld_b < d->cols || a.ld_z < d->cols) return MW_ERR_INVALID_ARG;
  if (d->rows && (!x || (!b && (z || w_post || scale)))) return MW_ERR_INVALID_ARG;
  a.x = x; a.b = b; a.z = z; a.w_post = w_post; a.scale = scale; a.w_pre = w_pre;
  return MW_OK;
}

}  // namespace
}  // namespace mw

extern "C" mw_status mw_residual_norm_forward(const mw_residual_norm_desc* desc, const void* x, const void* b,
                                              const void* z, const float* w_post, const float* scale,
                                              const float* w_pre, void* x_out, void* n, float* inv_rms, void* stream) {
  using namespace mw;
  NormArgs a;
  MW_TRY(fill_norm(desc, x, b, z, w_post, scale, w_pre, a));
  if (a.rows && ((w_pre != nullptr) != (n != nullptr) || (!x_out && !n))) return MW_ERR_INVALID_ARG;
  if (x_out == x && a.ld_x != a.cols) return MW_ERR_INVALID_ARG;
  if (a.rows == 0) return MW_OK;
  a.x_out = x_out; a.n = n; a.inv_rms = inv_rms;
  return desc->dtype == 1 ? run_norm<float, 4>(a, false, (cudaStream_t)stream)
                          : run_norm<__nv_bfloat16, 8>(a, false, (cudaStream_t)stream);
}

extern "C" mw_status mw_residual_norm_scratch_bytes(const mw_residual_norm_desc* desc, size_t* bytes) {
  using namespace mw;
  if (!desc || !bytes || desc->rows < 0 || desc->cols < 1) return MW_ERR_INVALID_ARG;
  if (desc->cols > kMaxCols) return MW_ERR_UNSUPPORTED;
  *bytes = (size_t)backward_blocks(desc->rows, desc->cols) * rows_per_block(group_of(desc->cols)) * 3 *
           (size_t)desc->cols * sizeof(float);
  return MW_OK;
}

extern "C" mw_status mw_residual_norm_backward(const mw_residual_norm_desc* desc, const void* x, const void* b,
                                               const void* z, const float* w_post, const float* scale,
                                               const float* w_pre, const float* inv_rms, const void* dx_out,
                                               const void* dn, void* dx, void* db, void* dz, float* dw_post,
                                               float* dscale, float* dw_pre, void* scratch, size_t scratch_bytes,
                                               void* stream) {
  using namespace mw;
  NormArgs a;
  MW_TRY(fill_norm(desc, x, b, z, w_post, scale, w_pre, a));
  if (a.rows && ((dn && !w_pre) || (db && !b) || (dz && !z) || (dw_post && !w_post) || (dscale && !scale) || (dw_pre && !w_pre)))
    return MW_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  if (a.rows == 0) {
    float* w[] = {dw_post, dscale, dw_pre};
    for (float* p : w)
      if (p) MW_CUDA_OK(cudaMemsetAsync(p, 0, sizeof(float) * (size_t)a.cols, s));
    return MW_OK;
  }
  if (!inv_rms) return MW_ERR_INVALID_ARG;
  a.rms_in = inv_rms;
  a.dx_out = dx_out; a.dn = dn; a.dx = dx; a.db = db; a.dz = dz;
  const bool sums = dw_post || dscale || dw_pre;
  if (sums) {
    size_t need = 0;
    MW_TRY(mw_residual_norm_scratch_bytes(desc, &need));
    if (!scratch || ((uintptr_t)scratch & 255u) || scratch_bytes < need) return MW_ERR_WORKSPACE;
    a.partials = static_cast<float*>(scratch);
  }
  MW_TRY(desc->dtype == 1 ? (run_norm<float, 4>(a, true, s)) : (run_norm<__nv_bfloat16, 8>(a, true, s)));
  if (!sums) return MW_OK;
  const int parts = (int)backward_blocks(a.rows, a.cols) * rows_per_block(group_of(a.cols));
  norm_reduce_kernel<<<dim3((unsigned)((a.cols + 31) / 32), 3), 256, 0, s>>>(a.partials, parts, a.cols, dw_post, dscale,
                                                                             dw_pre);
  return launch_ok();
}
