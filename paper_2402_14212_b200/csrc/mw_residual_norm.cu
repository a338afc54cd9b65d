// Residual sum of a block with the norms around it (mw_residual_norm_*):
//   p = w_post b / rms(b),  x' = x + scale silu(z) p,  n = w_pre x' / rms(x')
// One pass over each row in both directions: W warps hold the row in registers (or several rows share a warp,
// or a cluster of blocks shares a row), so every tensor crosses HBM once (forward 10 bytes an element in
// bf16, backward 16).
#include "mw_cluster.cuh"
#include "mw_common.cuh"

namespace mw {
namespace {

constexpr int kMaxCols = 32768;
constexpr int kBlockWarps = 8;          // rows are put together up to this many warps a block
constexpr int kRowWarps = 16;           // most warps of one block on one row
constexpr int kForwardValues = 16, kBackwardValues = 8;      // of a row, a thread

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
  float* partials;      // [blocks, or clusters][2][cols]
};

// How rows are laid over threads.  A piece is the VEC elements of one access; a thread takes K of them.
struct NormPlan {
  int lanes;            // 32, or fewer where a row is that short
  int warps;            // of one block on one row, a power of two
  int rows;             // of one block at a time
  int cluster;          // blocks that share a row
  int per;              // pieces of one block
  int threads;
  int64_t blocks;       // grid
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

// (The exponential of a z far below zero is infinite, and the quotient zero.  The fast exponential rounds z log2(e)
// first, |z| 2^-24 of the result: the results of 1003x1111 f32 are 1.6e-7 from 64 bits, 1.4e-7 with the library's.)
__device__ __forceinline__ float sigmoid_f(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

// Where a row's sums meet: its warps' in shared memory, alternating between two buffers, so that one barrier a
// reduction is enough.  Blocks of a cluster send their warps' sums to each other, 16 bytes each, counted on a
// barrier at the receiver; a buffer is sent to again only by a warp that has every sum of the reduction between,
// which no warp sends before it has read this one's.
template <bool CLUSTER>
struct RowMeet {
  float own[CLUSTER ? 1 : 2][CLUSTER ? 1 : 3 * 32];
  float4 box[CLUSTER ? 2 : 1][CLUSTER ? 8 * kRowWarps : 1];
  unsigned long long arrived[2];

  __device__ __forceinline__ void begin(int C) {
    if (C == 1) return;
    if (threadIdx.x == 0) {
      for (int i = 0; i < 2; ++i)
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(shared_address(&arrived[i])) : "memory");
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    cluster_sync();
  }
  // no block leaves while sums are still being sent to it
  __device__ __forceinline__ void end(int C) {
    if (C > 1) cluster_sync();
  }

  // sums of N <= 3 values over the threads of a row: `n` counts the reductions, `ok` turns false (and the sums NaN)
  // if sums of other blocks did not come
  template <int LANES, int W, int N>
  __device__ __forceinline__ void sum(float (&s)[N], int n, const NormPlan& p, int rank, bool& ok) {
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
    if (W == 1) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, flip = n & 1;
    if constexpr (!CLUSTER) {
      float* buf = own[flip];
      if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) buf[i * 32 + warp] = s[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) s[i] = buf[i * 32 + warp / W * W + (lane & (W - 1))];
#pragma unroll
      for (int o = W / 2; o; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
      return;
    }
    if constexpr (CLUSTER) {
      const float4 mine = make_float4(s[0], N > 1 ? s[N > 1 ? 1 : 0] : 0.f, N > 2 ? s[N > 2 ? 2 : 0] : 0.f, 0.f);
      const int sums = p.cluster * W;
      const uint32_t bar = shared_address(&arrived[flip]);
      if (threadIdx.x == 0)
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)sums * 16u) : "memory");
      if (lane < p.cluster)
        asm volatile(
            "st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(
                in_rank(shared_address(&box[flip][rank * W + warp]), lane)),
            "f"(mine.x), "f"(mine.y), "f"(mine.z), "f"(mine.w), "r"(in_rank(bar, lane))
            : "memory");
      ok = ok && wait_phase(bar, (uint32_t)(n >> 1) & 1u);
      float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int e = lane; e < sums; e += 32) {
        const float4 v = box[flip][e];
        t.x += v.x; t.y += v.y; t.z += v.z;
      }
      s[0] = ok ? t.x : __int_as_float(0x7fffffff);
      if (N > 1) s[N > 1 ? 1 : 0] = ok ? t.y : __int_as_float(0x7fffffff);
      if (N > 2) s[N > 2 ? 2 : 0] = ok ? t.z : __int_as_float(0x7fffffff);
#pragma unroll
      for (int o = 16; o; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
    }
  }
};

// This thread's place: the row of its block's `rows`, its first piece, the end
struct NormPlace {
  int sub, piece, end, rank;
  // whether the piece `ahead` of the first lies in the row, or in the block's part of it
  template <int VEC, bool CLUSTER>
  __device__ __forceinline__ bool holds(int ahead, int cols) const {
    return CLUSTER ? piece + ahead < end : (piece + ahead) * VEC < cols;
  }
};
template <int VEC, int LANES, int W, bool CLUSTER>
__device__ __forceinline__ NormPlace norm_place(const NormArgs& a, const NormPlan& p) {
  NormPlace w;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  w.rank = CLUSTER ? (int)(blockIdx.x % p.cluster) : 0;
  w.sub = LANES < 32 ? threadIdx.x / LANES : (W >= kBlockWarps ? 0 : warp / W);
  w.piece = LANES < 32 ? threadIdx.x % LANES : (W >= kBlockWarps ? (int)threadIdx.x : warp % W * 32 + lane);
  const int all = (a.cols + VEC - 1) / VEC;
  w.end = all;
  if (CLUSTER) {
    w.piece += w.rank * p.per;
    w.end = all < (w.rank + 1) * p.per ? all : (w.rank + 1) * p.per;
  }
  return w;
}

// per-column constants of a thread: scale times post-norm weight, pre-norm weight
template <int VEC, int STEP, bool CLUSTER, int K>
__device__ __forceinline__ void column_constants(const NormArgs& a, const NormPlace& w, float (&ks)[K][VEC], float (&wn)[K][VEC]) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (w.piece + k * STEP) * VEC;
    if (w.template holds<VEC, CLUSTER>(k * STEP, a.cols)) {
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

// Bound by HBM: 16384x4096 bf16 takes 107 to 113 us for its 671 MB, 90 to 96% of a plain copy's rate.  (The kernels
// that go element by element, and those of fp32 rows of 8 warps and more, store 16 to 136 bytes of registers a thread:
// 8192x4097 bf16 takes 149 us, where its bytes would take 51.)
// The grid is persistent in both directions: a thread meets the same columns in every row, keeps their
// weights in registers, and has the next row's loads under way while it works on the present one.
template <typename T, int VEC, int LANES, int W, bool CLUSTER>
__global__ void __launch_bounds__(32 * kRowWarps, 1)
norm_forward_kernel(const NormArgs a, const NormPlan p) {
  using P = Pack<T, VEC>;
  using Raw = typename P::Raw;
  constexpr int K = kForwardValues / VEC, STEP = LANES < 32 ? LANES : 32 * W;
  __shared__ __align__(16) RowMeet<CLUSTER> meet;
  const NormPlace w = norm_place<VEC, LANES, W, CLUSTER>(a, p);
  const int C = CLUSTER ? p.cluster : 1;
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
      const int c = (w.piece + k * STEP) * VEC;
      rx[k] = rb[k] = rz[k] = P::zero();
      if (w.template holds<VEC, CLUSTER>(k * STEP, D)) {
        rx[k] = __ldcs(reinterpret_cast<const Raw*>(x + c));
        if (has_b) rb[k] = __ldcs(reinterpret_cast<const Raw*>(b + c));
        if (has_z) rz[k] = __ldcs(reinterpret_cast<const Raw*>(z + c));
      }
    }
  };
  const int rows = LANES == 32 && W >= kBlockWarps ? 1 : p.rows;
  const int64_t stride = (int64_t)(gridDim.x / C) * rows, first = (int64_t)(blockIdx.x / C) * rows;
  load(first + w.sub);
  meet.begin(C);
  float ks[K][VEC], wn[K][VEC];
  column_constants<VEC, STEP, CLUSTER, K>(a, w, ks, wn);
  int n = 0;
  bool ok = true;
  for (int64_t base = first; base < a.rows; base += stride) {
    const int64_t row = base + w.sub;
    const bool live = (LANES == 32 && W >= kBlockWarps) || row < a.rows;
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
      meet.template sum<LANES, W, 1>(s, CLUSTER ? n++ : 0, p, w.rank, ok);
      inv_b = rsqrtf(fmaf(s[0], inv_d, a.eps));
    }
    s[0] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (w.piece + k * STEP) * VEC;
      if (has_b)
#pragma unroll
        for (int i = 0; i < VEC; ++i) y[k][i] = fmaf(tau[k][i], inv_b, y[k][i]);
      if (live && a.x_out && w.template holds<VEC, CLUSTER>(k * STEP, D)) __stcs(reinterpret_cast<Raw*>(static_cast<T*>(a.x_out) + row * D + c), P::put(y[k]));
#pragma unroll
      for (int i = 0; i < VEC; ++i) s[0] = fmaf(y[k][i], y[k][i], s[0]);
    }
    float inv_x = 1.f;
    if (a.w_pre) {
      meet.template sum<LANES, W, 1>(s, CLUSTER ? n++ : 1, p, w.rank, ok);
      inv_x = rsqrtf(fmaf(s[0], inv_d, a.eps));
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = (w.piece + k * STEP) * VEC;
        if (live && w.template holds<VEC, CLUSTER>(k * STEP, D)) {
          float o[VEC];
#pragma unroll
          for (int i = 0; i < VEC; ++i) o[i] = y[k][i] * inv_x * wn[k][i];
          __stcs(reinterpret_cast<Raw*>(static_cast<T*>(a.n) + row * D + c), P::put(o));
        }
      }
    }
    if (live && a.inv_rms && w.piece == 0) {
      a.inv_rms[row] = inv_b;
      a.inv_rms[a.rows + row] = inv_x;
    }
    // (either buffer is written again only after all have passed the other's barrier, or this one)
    if (!CLUSTER && W > 1 && !(a.w_post && a.w_pre)) __syncthreads();
  }
  meet.end(C);
}

// most threads of a block whose rows take W warps
__host__ __device__ constexpr int norm_threads(int W) { return 32 * (W > kBlockWarps ? W : kBlockWarps); }
// rows in flight or at work on an SM: with 16 warps there 120 or 160 KB of copies (a fourth row for the smaller
// type gained nothing: 16384x4096 bf16 233 us, 231 with three)
__host__ __device__ constexpr int backward_stages(int K) { return K == 1 ? 3 : 2; }

// Backward of a row, with xh = x' / rms, bh = b / rms, q = dn w_pre, ks = scale w_post, tau = ks silu(z) bh:
//   dx = dx_out + (q - xh m1) / rms(x'),                m1 = mean(q xh)
//   db = (dx ks silu(z) - bh m2) / rms(b),              m2 = mean(dx tau)
//   dz = dx ks bh silu'(z);   dw_pre = sum dn xh;   dw_post = scale S, dscale = w_post S,  S = sum dx silu(z) bh
// m2 needs dx, which needs m1; written out, mean(dx tau) = mean((dx_out + q/rms) tau) - m1 mean(xh tau)/rms,
// so the three sums go through ONE reduction a row (16384x4096 bf16: 230 us for 1074 MB, 71% of a plain copy's
// rate; one block of 16 warps an SM at 128 registers a thread does not cover its reduction's waits; element by element
// the kernels spill as well, 24 to 84 bytes stored: 8192x4097 438 us).  A thread keeps its columns' two sums over
// rows in registers; the blocks' partials meet in fixed order in norm_reduce_kernel.
template <typename T, int VEC, int LANES, int W, bool CLUSTER>
__global__ void __launch_bounds__(32 * kRowWarps, 1)
norm_backward_kernel(const NormArgs a, const NormPlan p) {
  using P = Pack<T, VEC>;
  using Raw = typename P::Raw;
  constexpr int K = kBackwardValues / VEC, STEP = LANES < 32 ? LANES : 32 * W;
  __shared__ __align__(16) RowMeet<CLUSTER> meet;
  const NormPlace w = norm_place<VEC, LANES, W, CLUSTER>(a, p);
  const int C = CLUSTER ? p.cluster : 1;
  const int D = a.cols;
  const float inv_d = 1.f / (float)D;
  // (without a cotangent of n nothing depends on x': what it holds, infinities too, stays out of the sums)
  const bool has_b = a.b != nullptr, has_z = a.z != nullptr, has_n = a.dn != nullptr, normed = a.w_post != nullptr;
  // A thread's 16 bytes of each tensor come by asynchronous copies into shared memory of its own, kStages - 1 rows
  // ahead: at 40 bytes an element in and out, one row ahead leaves HBM idle while a row is reduced.  (Rows
  // that are read element by element, whose copies could not be that small, are held in registers, one
  // row ahead.)
  constexpr bool kStaged = sizeof(Raw) == 16;
  constexpr int kStages = kStaged ? backward_stages(K) : 1;
  extern __shared__ __align__(16) unsigned char ring[];
  unsigned char* mine = ring + threadIdx.x * 16;
  constexpr uint32_t kTensor = norm_threads(W) * 16, kPart = 5 * kTensor, kStage = K * kPart;
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
  const int rows = LANES == 32 && W >= kBlockWarps ? 1 : p.rows;
  const int64_t stride = (int64_t)(gridDim.x / C) * rows, first = (int64_t)(blockIdx.x / C) * rows;
  // start the copies of the row `ahead` iterations from `row` (one group each, empty past the end)
  auto fetch = [&](int64_t row, int stage) {
    if (row < a.rows) {
      const T* at[5];
      place(row, at);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = (w.piece + k * STEP) * VEC;
#pragma unroll
        for (int j = 0; j < 5; ++j) {
          const bool on = has[j] && w.template holds<VEC, CLUSTER>(k * STEP, D);
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
        const int c = (w.piece + k * STEP) * VEC;
        rx[k] = rb[k] = rz[k] = ro[k] = rn[k] = P::zero();
        if (w.template holds<VEC, CLUSTER>(k * STEP, D)) {
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
  const int64_t row0 = first + w.sub;
  if (kStaged)
    for (int i = 0; i < kStages - 1; ++i) fetch(row0 + i * stride, i);
  load(row0);
  meet.begin(C);
  float ks[K][VEC], wn[K][VEC], acc_s[K][VEC], acc_n[K][VEC];
  column_constants<VEC, STEP, CLUSTER, K>(a, w, ks, wn);
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc_s[k][i] = acc_n[k][i] = 0.f;
  int n = 0, stage = 0;
  bool ok = true;
  for (int64_t base = first; base < a.rows; base += stride) {
    const int64_t row = base + w.sub;
    const bool live = (LANES == 32 && W >= kBlockWarps) || row < a.rows;
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
    const float inv_b = next_b, inv_x = has_n ? next_x : 0.f, xs = next_x;
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
        if (live && has_n) acc_n[k][i] = fmaf(vn[i], xh[k][i], acc_n[k][i]);
      }
    }
    if (base + stride < a.rows) load(row + stride);
    meet.template sum<LANES, W, 3>(s, n, p, w.rank, ok);
    n = CLUSTER ? n + 1 : n ^ 1;
    const float m1 = has_n ? s[0] * inv_d * inv_x : 0.f;
    const float m2 = normed ? (has_n ? fmaf(-m1, s[2], s[1]) : s[1]) * inv_d * inv_b : 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (w.piece + k * STEP) * VEC;
      if (!w.template holds<VEC, CLUSTER>(k * STEP, D) || !live) continue;
      float vb[VEC], ox[VEC], ob[VEC], oz[VEC];
      P::get(cb[k], vb);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        float dx = A[k][i];
        if (has_n) dx = fmaf(-xh[k][i], m1, dx);
        const float bh = vb[i] * inv_b, dk = dx * ks[k][i], dg = dx * gate[k][i];
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
  meet.end(C);
  if (a.partials == nullptr) return;
  // the block's rows meet in fixed order, so that a block leaves one partial sum a column: first those of a warp ...
  if (LANES < 32)
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < VEC; ++i)
#pragma unroll
        for (int o = LANES; o < 32; o <<= 1) {
          acc_s[k][i] += __shfl_xor_sync(0xffffffffu, acc_s[k][i], o);
          acc_n[k][i] += __shfl_xor_sync(0xffffffffu, acc_n[k][i], o);
        }
  // ... then, one after the other, those of its warps (of as many columns as leave more than one row to a block)
  // (in the copies' room: past the last row they are empty)
  float* joined = reinterpret_cast<float*>(ring);
  if (rows > 1) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
  }
  const int turns = LANES < 32 ? (int)(blockDim.x >> 5) : rows, turn = LANES < 32 ? (int)(threadIdx.x >> 5) : w.sub;
  float* out = a.partials + (int64_t)(blockIdx.x / C) * 2 * D;
  for (int r = 0; r < turns; ++r) {
    if (r) __syncthreads();
    if (turn != r || (LANES < 32 && (threadIdx.x & 31) >= LANES)) continue;
    const bool last = r == turns - 1;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = (w.piece + k * STEP) * VEC;
      if (!w.template holds<VEC, CLUSTER>(k * STEP, D)) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float vs = r ? joined[c + i] + acc_s[k][i] : acc_s[k][i], vn = r ? joined[D + c + i] + acc_n[k][i] : acc_n[k][i];
        if (last) {
          out[c + i] = vs;
          out[D + c + i] = vn;
        } else {
          joined[c + i] = vs;
          joined[D + c + i] = vn;
        }
      }
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
// clusters of C blocks that the device holds at once, a block an SM
int norm_clusters(int C) {
  static int cached[64][9] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) dev = 0;
  if (cached[dev][C] == 0) {
    auto kernel = norm_backward_kernel<__nv_bfloat16, 8, 32, kRowWarps, true>;
    const int ring = backward_stages(1) * 80 * 32 * kRowWarps;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)C);
    cfg.blockDim = dim3(32 * kRowWarps);
    cfg.dynamicSmemBytes = ring;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)C;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ring) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
      cudaGetLastError();
      n = norm_sms() / C;
    }
    cached[dev][C] = n;
  }
  return cached[dev][C];
}

// A row takes the fewest warps that hold it, a power of two: 16 warps an SM, in blocks of
// up to eight with several rows each, or of up to sixteen with one; wider rows are shared by a cluster.  (One block
// that holds such a row spills its registers: 2048x16384 bf16 backward 625 us so, 169 in clusters of four; 8192x6144
// 282 and 245.  Rows shorter than a warp's share get 8 or 16 lanes: 65536x64 bf16 forward 12 us, backward 20, 40
// and 56 with a warp each.  A power of two of warps: any number, known at run time only, measured a tenth slower.)
NormPlan norm_plan(int64_t rows, int cols, int vec, bool backward) {
  NormPlan p;
  const int values = backward ? kBackwardValues : kForwardValues;
  const int pieces = (cols + vec - 1) / vec, each = values / vec;
  p.cluster = (cols + values * 32 * kRowWarps - 1) / (values * 32 * kRowWarps);
  p.per = (pieces + p.cluster - 1) / p.cluster;
  p.warps = p.cluster > 1 ? kRowWarps : 1;
  while (p.warps * 32 * each < p.per) p.warps *= 2;
  p.lanes = 32;
  while (p.lanes > 8 && p.lanes / 2 * each >= pieces) p.lanes /= 2;
  // few rows: one block an SM before several rows a block
  const int64_t spread = rows > norm_sms() ? (rows + norm_sms() - 1) / norm_sms() : 1;
  if (p.lanes < 32) {
    const int in_warp = 32 / p.lanes;
    int warps = (int)(spread < (int64_t)kBlockWarps * in_warp ? (spread + in_warp - 1) / in_warp : kBlockWarps);
    p.threads = 32 * warps;
    p.rows = warps * in_warp;
  } else {
    const int most = p.warps > kBlockWarps ? 1 : kBlockWarps / p.warps;
    p.rows = (int)(spread < most ? spread : most);
    p.threads = 32 * p.warps * p.rows;
  }
  const int64_t need = (rows + p.rows - 1) / p.rows, at_once = p.cluster > 1 ? norm_clusters(p.cluster) : (int64_t)norm_sms() * (32 * kRowWarps / p.threads);
  p.blocks = (need < at_once ? need : at_once) * p.cluster;
  return p;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// a plan's launch; with clusters, as many as are resident at once
template <typename Kernel>
mw_status launch_norm(Kernel kernel, const NormArgs& a, NormPlan p, size_t ring, cudaStream_t s) {
  if (ring) MW_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ring));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.blocks);
  cfg.blockDim = dim3((unsigned)p.threads);
  cfg.dynamicSmemBytes = ring;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  if (p.cluster > 1) {
    cfg.attrs = attr;
    cfg.numAttrs = 1;
  }
  ++g_launch_count;
  return cudaLaunchKernelEx(&cfg, kernel, a, p) == cudaSuccess ? MW_OK : MW_ERR_CUDA;
}

template <typename T, int VEC, int LANES, int W, bool CLUSTER>
mw_status launch_either(const NormArgs& a, const NormPlan& p, bool backward, cudaStream_t s) {
  constexpr int K = kBackwardValues / VEC;
  // (rows that share a block meet there at the end)
  const size_t join = p.threads > 32 * W ? (size_t)2 * a.cols * sizeof(float) : 0;
  const size_t ring = VEC * sizeof(T) == 16 ? (size_t)backward_stages(K) * K * 80 * norm_threads(W) : join;
  return backward ? launch_norm(norm_backward_kernel<T, VEC, LANES, W, CLUSTER>, a, p, ring, s)
                  : launch_norm(norm_forward_kernel<T, VEC, LANES, W, CLUSTER>, a, p, 0, s);
}

template <typename T, int VEC>
mw_status dispatch_norm(const NormArgs& a, bool backward, cudaStream_t s) {
  const NormPlan p = norm_plan(a.rows, a.cols, VEC, backward);
  if (p.cluster > 1) return launch_either<T, VEC, 32, kRowWarps, true>(a, p, backward, s);
  if (p.lanes == 8) return launch_either<T, VEC, 8, 1, false>(a, p, backward, s);
  if (p.lanes == 16) return launch_either<T, VEC, 16, 1, false>(a, p, backward, s);
  switch (p.warps) {
    case 1: return launch_either<T, VEC, 32, 1, false>(a, p, backward, s);
    case 2: return launch_either<T, VEC, 32, 2, false>(a, p, backward, s);
    case 4: return launch_either<T, VEC, 32, 4, false>(a, p, backward, s);
    case 8: return launch_either<T, VEC, 32, 8, false>(a, p, backward, s);
    default: return launch_either<T, VEC, 32, 16, false>(a, p, backward, s);
  }
}

// 16-byte accesses where every row of every tensor starts on such a boundary, else element by element
template <typename T, int VEC>
bool norm_wide(const NormArgs& a) {
  const void* ptrs[] = {a.x, a.b, a.z, a.w_post, a.scale, a.w_pre, a.x_out, a.n, a.dx_out, a.dn, a.dx, a.db, a.dz};
  bool wide = a.cols % VEC == 0 && a.ld_x % VEC == 0 && a.ld_b % VEC == 0 && a.ld_z % VEC == 0;
  for (const void* p : ptrs) wide = wide && aligned16(p);
  return wide;
}
template <typename T, int VEC>
mw_status run_norm(const NormArgs& a, bool backward, cudaStream_t s) {
  return norm_wide<T, VEC>(a) ? dispatch_norm<T, VEC>(a, backward, s) : dispatch_norm<T, 1>(a, backward, s);
}
// partial sums that the backward pass leaves
int backward_parts(int64_t rows, int cols, int vec) {
  const NormPlan p = norm_plan(rows, cols, vec, true);
  return (int)(p.blocks / p.cluster);
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
  // a partial sum a block: at most one a row, and two blocks an SM
  const int64_t most = 2 * (int64_t)norm_sms();
  *bytes = (size_t)(desc->rows < most ? desc->rows : most) * 2 * (size_t)desc->cols * sizeof(float);
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
  const bool wide = desc->dtype == 1 ? norm_wide<float, 4>(a) : norm_wide<__nv_bfloat16, 8>(a);
  const int parts = backward_parts(a.rows, a.cols, wide ? (desc->dtype == 1 ? 4 : 8) : 1);
  norm_reduce_kernel<<<dim3((unsigned)((a.cols + 31) / 32), 2), 1024, 0, s>>>(a.partials, parts, a.cols, w_post, scale,
                                                                              dw_post, dscale, dw_pre);
  return launch_ok();
}
