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
  float* partials;      // [grid * rows a block][2][cols]
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

// (the exponential of a z far below zero is infinite, and the quotient zero)
__device__ __forceinline__ float sigmoid_f(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

// sums over the G threads that share a row (G a power of two, 32..1024, aligned inside the block); the
// caller alternates between two buffers, so that one barrier a reduction is enough
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
      for (int i = 0; i < N; ++i) buf[i * 32 + warp] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = buf[i * 32 + first + (lane & (W - 1))];
#pragma unroll
    for (int o = W / 2; o; o >>= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
  }
}

// per-column constants of a thread: scale times post-norm weight, pre-norm weight
template <int VEC, int G, int K>
__device__ __forceinline__ void column_constants(const NormArgs& a, int t, float (&ks)[K][VEC], float (&wn)[K][VEC]) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * G + t) * VEC;
    if (c < a.cols) {
      float wp[VEC], sc[VEC];
      load_weight<VEC>(a.w_post, c, wp);
      load_weight<VEC>(a.scale, c, sc);
      load_weight<VEC>(a.w_pre, c, wn[k]);
#pragma unroll
      for (int i = 0; i < VEC; ++i) ks[k][i] = wp[i] * sc[i];
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) ks[k][i] = wn[k][i] = 0.f;
    }
  }
}

// The grid is persistent in both directions: a thread meets the same columns in every row, keeps their
// weights in registers, and has the next row's loads under way while it works on the present one.
template <typename T, int VEC, int G, int K>
__global__ void __launch_bounds__(G > kNormThreads ? G : kNormThreads, G > kNormThreads ? 1 : 2)
norm_forward_kernel(const NormArgs a) {
  using P = Pack<T, VEC>;
  using Raw = typename P::Raw;
  constexpr int kRows = (G > kNormThreads ? G : kNormThreads) / G;
  __shared__ float buf[2][32];
  const int t = threadIdx.x % G, sub = threadIdx.x / G;
  const int D = a.cols;
  const float inv_d = 1.f / (float)D;
  const bool has_b = a.b != nullptr, has_z = a.z != nullptr;
  Raw rx[K], rb[K], rz[K];
  auto load = [&](int64_t row) {
    if (row >= a.rows) row = a.rows - 1;        // takes part in the barriers, stores nothing
    const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
    const T* b = static_cast<const T*>(a.b) + row * a.ld_b;
    const T* z = static_cast<const T*>(a.z) + row * a.ld_z;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + t) * VEC;
      rx[k] = rb[k] = rz[k] = P::zero();
      if (c < D) {
        rx[k] = __ldcs(reinterpret_cast<const Raw*>(x + c));
        if (has_b) rb[k] = __ldcs(reinterpret_cast<const Raw*>(b + c));
        if (has_z) rz[k] = __ldcs(reinterpret_cast<const Raw*>(z + c));
      }
    }
  };
  const int64_t stride = (int64_t)gridDim.x * kRows;
  load((int64_t)blockIdx.x * kRows + sub);
  float ks[K][VEC], wn[K][VEC];
  column_constants<VEC, G, K>(a, t, ks, wn);
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.rows; base += stride) {
    const int64_t row = base + sub;
    const bool live = row < a.rows;
    float y[K][VEC], tau[K][VEC];
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float vb[VEC], vz[VEC];
      P::get(rx[k], y[k]);
      P::get(rb[k], vb);
      P::get(rz[k], vz);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        s[0] = fmaf(vb[i], vb[i], s[0]);
        tau[k][i] = ks[k][i] * vb[i] * (has_z ? vz[i] * sigmoid_f(vz[i]) : 1.f);
      }
    }
    if (base + stride < a.rows) load(row + stride);
    float inv_b = 1.f;
    if (a.w_post) {
      row_sum<G, 1>(s, buf[0]);
      inv_b = rsqrtf(fmaf(s[0], inv_d, a.eps));
    }
    s[0] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + t) * VEC;
      if (has_b)
#pragma unroll
        for (int i = 0; i < VEC; ++i) y[k][i] = fmaf(tau[k][i], inv_b, y[k][i]);
      if (live && a.x_out && c < D) __stcs(reinterpret_cast<Raw*>(static_cast<T*>(a.x_out) + row * D + c), P::put(y[k]));
#pragma unroll
      for (int i = 0; i < VEC; ++i) s[0] = fmaf(y[k][i], y[k][i], s[0]);
    }
    float inv_x = 1.f;
    if (a.w_pre) {
      row_sum<G, 1>(s, buf[1]);
      inv_x = rsqrtf(fmaf(s[0], inv_d, a.eps));
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = (k * G + t) * VEC;
        if (live && c < D) {
          float o[VEC];
#pragma unroll
          for (int i = 0; i < VEC; ++i) o[i] = y[k][i] * inv_x * wn[k][i];
          __stcs(reinterpret_cast<Raw*>(static_cast<T*>(a.n) + row * D + c), P::put(o));
        }
      }
    }
    if (live && a.inv_rms && t == 0) {
      a.inv_rms[row] = inv_b;
      a.inv_rms[a.rows + row] = inv_x;
    }
    // (each buffer is written again only after the other's barrier, or this row's, has been passed by all)
    if (G > 32 && !(a.w_post && a.w_pre)) __syncthreads();
  }
}

// rows whose copies (80 bytes for each 16-byte piece of a row) fit beside each other: four up to 40 KB a row, two up
// to 80 KB; longer rows are held in registers
__host__ __device__ constexpr int backward_stages(int pieces) {
  return pieces <= 512 ? 4 : (pieces <= 1024 ? 2 : 0);
}

// Backward of a row, with xh = x' / rms, bh = b / rms, q = dn w_pre, ks = scale w_post, tau = ks silu(z) bh:
//   dx = dx_out + (q - xh m1) / rms(x'),                m1 = mean(q xh)
//   db = (dx ks silu(z) - bh m2) / rms(b),              m2 = mean(dx tau)
//   dz = dx ks bh silu'(z);   dw_pre = sum dn xh;   dw_post = scale S, dscale = w_post S,  S = sum dx silu(z) bh
// m2 needs dx, which needs m1; written out, mean(dx tau) = mean((dx_out + q/rms) tau) - m1 mean(xh tau)/rms,
// so the three sums go through ONE reduction a row.  A thread keeps its columns' two sums over rows in
// registers; the blocks' partials meet in fixed order in norm_reduce_kernel.
template <typename T, int VEC, int G, int K>
__global__ void __launch_bounds__(G > kNormThreads ? G : kNormThreads, G > kNormThreads ? 1 : 2)
norm_backward_kernel(const NormArgs a) {
  using P = Pack<T, VEC>;
  using Raw = typename P::Raw;
  constexpr int kThreads = G > kNormThreads ? G : kNormThreads;
  constexpr int kRows = kThreads / G;
  __shared__ float buf[2][96];
  const int t = threadIdx.x % G, sub = threadIdx.x / G;
  const int D = a.cols;
  const float inv_d = 1.f / (float)D;
  const bool has_b = a.b != nullptr, has_z = a.z != nullptr, normed = a.w_post != nullptr;
  // A thread's 16 bytes of each tensor come by asynchronous copies into shared memory of its own, kStages - 1 rows
  // ahead: at 40 bytes an element in and out, one row ahead leaves HBM idle while a row is reduced.  (Rows
  // that are read element by element, whose copies could not be that small, are held in registers, one
  // row ahead.)
  constexpr bool kStaged = sizeof(Raw) == 16 && backward_stages(kThreads * K) > 0;
  constexpr int kStages = kStaged ? backward_stages(kThreads * K) : 1;
  extern __shared__ __align__(16) unsigned char ring[];
  unsigned char* mine = ring + threadIdx.x * 16;
  constexpr uint32_t kTensor = kThreads * 16, kPart = 5 * kTensor, kStage = K * kPart;
  Raw rx[K], rb[K], rz[K], ro[K], rn[K];
  float next_b = 0.f, next_x = 0.f;
  auto place = [&](int64_t row, const T* (&at)[5]) {
    at[0] = static_cast<const T*>(a.x) + row * a.ld_x;
    at[1] = static_cast<const T*>(a.b) + row * a.ld_b;
    at[2] = static_cast<const T*>(a.z) + row * a.ld_z;
    at[3] = static_cast<const T*>(a.dx_out) + row * D;
    at[4] = static_cast<const T*>(a.dn) + row * D;
  };
  const bool has[5] = {true, has_b, has_z, a.dx_out != nullptr, a.dn != nullptr};
  const int64_t stride = (int64_t)gridDim.x * kRows;
  // start the copies of the row `ahead` iterations from `row` (one group each, empty past the end)
  auto fetch = [&](int64_t row, int stage) {
    if (row < a.rows) {
      const T* at[5];
      place(row, at);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = (k * G + t) * VEC;
#pragma unroll
        for (int j = 0; j < 5; ++j) {
          const bool on = has[j] && c < D;
          const uint32_t to = (uint32_t)__cvta_generic_to_shared(mine + stage * kStage + k * kPart + j * kTensor);
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(on ? (const void*)(at[j] + c) : a.x),
                       "r"(on ? 16 : 0)
                       : "memory");
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // the present row's values; the rows' two factors come one row ahead in registers either way
  auto load = [&](int64_t row) {
    if (row >= a.rows) row = a.rows - 1;        // takes part in the barriers, counts for nothing
    if (!kStaged) {
      const T* at[5];
      place(row, at);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = (k * G + t) * VEC;
        rx[k] = rb[k] = rz[k] = ro[k] = rn[k] = P::zero();
        if (c < D) {
          rx[k] = __ldcs(reinterpret_cast<const Raw*>(at[0] + c));
          if (has[1]) rb[k] = __ldcs(reinterpret_cast<const Raw*>(at[1] + c));
          if (has[2]) rz[k] = __ldcs(reinterpret_cast<const Raw*>(at[2] + c));
          if (has[3]) ro[k] = __ldcs(reinterpret_cast<const Raw*>(at[3] + c));
          if (has[4]) rn[k] = __ldcs(reinterpret_cast<const Raw*>(at[4] + c));
        }
      }
    }
    next_b = a.rms_in[row];
    next_x = a.rms_in[a.rows + row];
  };
  const int64_t row0 = (int64_t)blockIdx.x * kRows + sub;
  if (kStaged)
    for (int i = 0; i < kStages - 1; ++i) fetch(row0 + i * stride, i);
  load(row0);
  float ks[K][VEC], wn[K][VEC], acc_s[K][VEC], acc_n[K][VEC];
  column_constants<VEC, G, K>(a, t, ks, wn);
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc_s[k][i] = acc_n[k][i] = 0.f;
  int flip = 0, stage = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.rows; base += stride) {
    const int64_t row = base + sub;
    const bool live = row < a.rows;
    if (kStaged) {
      fetch(row + (kStages - 1) * stride, (stage + kStages - 1) % kStages);
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      const unsigned char* at = mine + stage * kStage;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        rx[k] = *reinterpret_cast<const Raw*>(at + k * kPart);
        rb[k] = *reinterpret_cast<const Raw*>(at + k * kPart + kTensor);
        rz[k] = *reinterpret_cast<const Raw*>(at + k * kPart + 2 * kTensor);
        ro[k] = *reinterpret_cast<const Raw*>(at + k * kPart + 3 * kTensor);
        rn[k] = *reinterpret_cast<const Raw*>(at + k * kPart + 4 * kTensor);
      }
      stage = stage + 1 == kStages ? 0 : stage + 1;
    }
    const float inv_b = next_b, inv_x = a.w_pre ? next_x : 0.f, xs = next_x;
    // kept over the reduction: dx_out + q / rms(x'), xh, silu(z), silu'(z), b
    float A[K][VEC], xh[K][VEC], gate[K][VEC], slope[K][VEC];
    Raw cb[K];
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float vx[VEC], vb[VEC], vz[VEC], vo[VEC], vn[VEC];
      P::get(rx[k], vx); P::get(rb[k], vb); P::get(rz[k], vz); P::get(ro[k], vo); P::get(rn[k], vn);
      cb[k] = rb[k];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        gate[k][i] = 1.f;
        slope[k][i] = 0.f;
        if (has_z) {
          const float sig = sigmoid_f(vz[i]);
          gate[k][i] = vz[i] * sig;
          slope[k][i] = sig * fmaf(vz[i], 1.f - sig, 1.f);
        }
        const float tau = ks[k][i] * (vb[i] * inv_b) * gate[k][i];
        xh[k][i] = (has_b ? vx[i] + tau : vx[i]) * xs;
        const float q = vn[i] * wn[k][i];
        A[k][i] = fmaf(q, inv_x, vo[i]);
        s[0] = fmaf(q, xh[k][i], s[0]);
        s[1] = fmaf(A[k][i], tau, s[1]);
        s[2] = fmaf(xh[k][i], tau, s[2]);
        if (live) acc_n[k][i] = fmaf(vn[i], xh[k][i], acc_n[k][i]);
      }
    }
    if (base + stride < a.rows) load(row + stride);
    row_sum<G, 3>(s, buf[flip]);
    flip ^= 1;
    const float m1 = s[0] * inv_d * inv_x;
    const float m2 = normed ? fmaf(-m1, s[2], s[1]) * inv_d * inv_b : 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (k * G + t) * VEC;
      if (c >= D || !live) continue;
      float vb[VEC], ox[VEC], ob[VEC], oz[VEC];
      P::get(cb[k], vb);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float dx = fmaf(-xh[k][i], m1, A[k][i]), bh = vb[i] * inv_b, dk = dx * ks[k][i], dg = dx * gate[k][i];
        ox[i] = dx;
        ob[i] = fmaf(dk * gate[k][i], inv_b, -bh * m2);
        oz[i] = dk * bh * slope[k][i];
        acc_s[k][i] = fmaf(dg, bh, acc_s[k][i]);
      }
      if (a.dx) __stcs(reinterpret_cast<Raw*>(static_cast<T*>(a.dx) + row * D + c), P::put(ox));
      if (a.db) __stcs(reinterpret_cast<Raw*>(static_cast<T*>(a.db) + row * D + c), P::put(ob));
      if (a.dz) __stcs(reinterpret_cast<Raw*>(static_cast<T*>(a.dz) + row * D + c), P::put(oz));
    }
  }
  if (a.partials == nullptr) return;
  float* out = a.partials + ((int64_t)blockIdx.x * kRows + sub) * 2 * D;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (k * G + t) * VEC;
    if (c >= D) continue;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      out[c + i] = acc_s[k][i];
      out[D + c + i] = acc_n[k][i];
    }
  }
}

// sums of `parts` rows of [2][D], in fixed order: a block owns 32 columns, its 32 warps the parts w, w + 32, ...
__global__ void __launch_bounds__(1024)
norm_reduce_kernel(const float* __restrict__ partials, int parts, int D, const float* __restrict__ w_post,
                   const float* __restrict__ scale, float* dw_post, float* dscale, float* dw_pre) {
  __shared__ float buf[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane, which = blockIdx.y;
  if (which == 0 ? !dw_post && !dscale : !dw_pre) return;
  float s = 0.f;
  if (c < D)
    for (int p = warp; p < parts; p += 32) s += partials[((int64_t)p * 2 + which) * D + c];
  buf[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < D) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 32; ++w) v += buf[w][lane];
    if (which == 1) {
      dw_pre[c] = v;
    } else {
      if (dw_post) dw_post[c] = v * (scale ? scale[c] : 1.f);
      if (dscale) dscale[c] = v * (w_post ? w_post[c] : 1.f);
    }
  }
}

// Threads that share a row of `cols`: the forward pass keeps 16 values a thread, the backward pass, whose
// threads also carry three sums a column and the next row's five tensors, 8 (more beyond 512 threads' worth).
int group_of(int cols, bool backward) {
  int g = 32;
  while (g < (backward ? 512 : 1024) && g * (backward ? 8 : 16) < cols) g <<= 1;
  return g;
}
int rows_per_block(int g) { return g > kNormThreads ? 1 : kNormThreads / g; }

int norm_sms() {
  static int cached[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) dev = 0;
  if (cached[dev] == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
      cudaGetLastError();
      n = 148;
    }
    cached[dev] = n;
  }
  return cached[dev];
}
// blocks of the backward pass: two of 256 threads (or one of 512) an SM
int64_t backward_blocks(int64_t rows, int cols) {
  const int g = group_of(cols, true), r = rows_per_block(g);
  const int64_t need = (rows + r - 1) / r, most = (int64_t)norm_sms() * (g > 256 ? 1 : 2);
  return need < most ? need : most;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

template <typename T, int VEC, int G, int VALUES>
mw_status launch_forward(const NormArgs& a, cudaStream_t s) {
  constexpr int threads = G > kNormThreads ? G : kNormThreads, r = threads / G;
  const int64_t need = (a.rows + r - 1) / r, most = (int64_t)norm_sms() * (G > kNormThreads ? 1 : 2);
  norm_forward_kernel<T, VEC, G, VALUES / VEC><<<(unsigned)(need < most ? need : most), threads, 0, s>>>(a);
  return launch_ok();
}
template <typename T, int VEC, int G, int VALUES>
mw_status launch_backward(const NormArgs& a, cudaStream_t s) {
  constexpr int threads = G > kNormThreads ? G : kNormThreads, K = VALUES / VEC;
  const size_t ring = VEC * sizeof(T) == 16 ? (size_t)backward_stages(threads * K) * threads * K * 80 : 0;
  auto kernel = norm_backward_kernel<T, VEC, G, K>;
  MW_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ring));
  kernel<<<(unsigned)backward_blocks(a.rows, a.cols), threads, ring, s>>>(a);
  return launch_ok();
}

template <typename T, int VEC>
mw_status dispatch_norm(const NormArgs& a, bool backward, cudaStream_t s) {
  if (backward) {
    switch (group_of(a.cols, true)) {
      case 32: return launch_backward<T, VEC, 32, 8>(a, s);
      case 64: return launch_backward<T, VEC, 64, 8>(a, s);
      case 128: return launch_backward<T, VEC, 128, 8>(a, s);
      case 256: return launch_backward<T, VEC, 256, 8>(a, s);
      default:
        if (a.cols <= 4096) return launch_backward<T, VEC, 512, 8>(a, s);
        if (a.cols <= 8192) return launch_backward<T, VEC, 512, 16>(a, s);
        if (a.cols <= 16384) return launch_backward<T, VEC, 512, 32>(a, s);
        return launch_backward<T, VEC, 512, 64>(a, s);
    }
  }
  switch (group_of(a.cols, false)) {
    case 32: return launch_forward<T, VEC, 32, 16>(a, s);
    case 64: return launch_forward<T, VEC, 64, 16>(a, s);
    case 128: return launch_forward<T, VEC, 128, 16>(a, s);
    case 256: return launch_forward<T, VEC, 256, 16>(a, s);
    case 512: return launch_forward<T, VEC, 512, 16>(a, s);
    default:
      return a.cols <= 16384 ? launch_forward<T, VEC, 1024, 16>(a, s) : launch_forward<T, VEC, 1024, 32>(a, s);
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
  *bytes = (size_t)backward_blocks(desc->rows, desc->cols) * rows_per_block(group_of(desc->cols, true)) * 2 *
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
  const int parts = (int)backward_blocks(a.rows, a.cols) * rows_per_block(group_of(a.cols, true));
  norm_reduce_kernel<<<dim3((unsigned)((a.cols + 31) / 32), 2), 1024, 0, s>>>(a.partials, parts, a.cols, w_post, scale,
                                                                              dw_post, dscale, dw_pre);
  return launch_ok();
}
