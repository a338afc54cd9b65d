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
// reciprocal: 1 - a formed by subtraction would lose the slow channels, where a is close to 1).  The
// exponent is held below 116, where a is 1e-35 and w exactly 1: the exponential stays finite.  NaN stays NaN.
__device__ __forceinline__ void gate_of(float f, float& a, float& w) {
  float x, e;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(f * -1.4426950408889634f), "f"(116.f));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(1.f + e));
  w = e * a;
}
__device__ __forceinline__ float sqrt_of(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
template <int GATE>
__device__ __forceinline__ float input_of(float a, float w) {
  return GATE == MW_SCAN_COMPLEMENT ? w : sqrt_of(fmaf(w, a, w));
}
// a (1 - a) u'(a): -a w, or -a^2 w / u = -a^2 sqrt(w / (1 + a)) (finite where u is zero)
template <int GATE>
__device__ __forceinline__ float input_slope(float a, float w) {
  return GATE == MW_SCAN_COMPLEMENT ? -a * w : -a * a * sqrt_of(__fdividef(w, 1.f + a));
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

// ---------------------------------------------------------------------------------------------
// Long sequences.  A step is the affine map h -> a h + b, and maps compose associatively, so time is
// cut three ways: a thread walks kEvery steps of its channel(s) held in registers, the W warps of a
// block cover W * kEvery consecutive steps, and the C blocks of a cluster cover C such pieces in a
// row.  Each level hands its composed map (P, H) to the next one through shared memory (its own, then
// that of the cluster's blocks), takes the state it starts from, and walks its steps again with it:
// every tensor crosses HBM once however the time axis is cut, and no block waits for another outside
// its cluster.  The cluster then moves on to the next C * W * kEvery steps, with the loads of those
// already under way.
// ---------------------------------------------------------------------------------------------
constexpr int kScanWarps = 8;
constexpr int kMaxCluster = 16;

// what one lane of a row holds: VEC channels of type T
template <typename T, int VEC>
struct Lane;
template <>
struct Lane<float, 1> {
  using Raw = float;
  static __device__ __forceinline__ Raw zero() { return 0.f; }
  static __device__ __forceinline__ void get(Raw r, float (&v)[1]) { v[0] = r; }
  static __device__ __forceinline__ Raw put(const float (&v)[1]) { return v[0]; }
};
template <>
struct Lane<__nv_bfloat16, 1> {
  using Raw = unsigned short;
  static __device__ __forceinline__ Raw zero() { return 0; }
  static __device__ __forceinline__ void get(Raw r, float (&v)[1]) { v[0] = __uint_as_float((uint32_t)r << 16); }
  static __device__ __forceinline__ Raw put(const float (&v)[1]) { return __bfloat16_as_ushort(__float2bfloat16_rn(v[0])); }
};
template <>
struct Lane<__nv_bfloat16, 2> {
  using Raw = uint32_t;
  static __device__ __forceinline__ Raw zero() { return 0u; }
  static __device__ __forceinline__ void get(Raw r, float (&v)[2]) {
    v[0] = __uint_as_float(r << 16);
    v[1] = __uint_as_float(r & 0xffff0000u);
  }
  static __device__ __forceinline__ Raw put(const float (&v)[2]) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[0], v[1]);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// 8 bytes into the shared memory of block `rank` of the cluster, at this block's address `p`
__device__ __forceinline__ void store_to_rank(float2* p, int rank, float2 v) {
  uint32_t a = (uint32_t)__cvta_generic_to_shared(p), r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(r), "f"(v.x), "f"(v.y) : "memory");
}

// no block's shared memory is written by another before that block runs
__device__ __forceinline__ void cluster_start(int C) {
  if (C > 1) {
    cluster_arrive();
    cluster_wait();
  }
}

// h -> P h + H.  With CUT a zero P drops h whatever it is: infinities and NaN of what came before a
// reset do not reach the steps after it.
template <bool CUT>
__device__ __forceinline__ float affine(float P, float h, float H) {
  return CUT && P == 0.f ? H : fmaf(P, h, H);
}

// Composes the maps of the block's warps and of the cluster's blocks.  In: this thread's map (P, H).
// Out: the state its steps start from, given the state `carry` the cluster's piece starts from;
// `carry` becomes the state after the piece.  REVERSE: the pieces follow one another from the last
// warp of the last block to the first (the cotangent's direction).
template <int VEC, bool CUT, bool REVERSE>
struct Exchange {
  float2 warp_map[2][kScanWarps][VEC][32];
  float2 block_map[2][kMaxCluster][VEC][32];

  __device__ __forceinline__ void run(const float (&P)[VEC], const float (&H)[VEC], float (&carry)[VEC],
                                      float (&start)[VEC], int flip, int rank, int C) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < VEC; ++i) warp_map[flip][warp][i][lane] = make_float2(P[i], H[i]);
    __syncthreads();
    if (C > 1) {
      // warp w sends the block's whole map to ranks w, w + W, ...
      if (warp < C) {
        float2 whole[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          whole[i] = make_float2(1.f, 0.f);
#pragma unroll
          for (int k = 0; k < kScanWarps; ++k) {
            const float2 m = warp_map[flip][REVERSE ? kScanWarps - 1 - k : k][i][lane];
            whole[i].y = affine<CUT>(m.x, whole[i].y, m.y);
            whole[i].x *= m.x;
          }
        }
        for (int r = warp; r < C; r += kScanWarps)
#pragma unroll
          for (int i = 0; i < VEC; ++i) store_to_rank(&block_map[flip][rank][i][lane], r, whole[i]);
      }
      cluster_arrive();
    }
    // while the others' maps arrive: the maps of this block's warps before this one
    const int before = REVERSE ? kScanWarps - 1 - warp : warp;
    float pe[VEC], he[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) { pe[i] = 1.f; he[i] = 0.f; }
    for (int k = 0; k < before; ++k) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float2 m = warp_map[flip][REVERSE ? kScanWarps - 1 - k : k][i][lane];
        he[i] = affine<CUT>(m.x, he[i], m.y);
        pe[i] *= m.x;
      }
    }
    if (C > 1) {
      cluster_wait();
      const int first = REVERSE ? C - 1 - rank : rank;      // blocks before this one
      for (int k = 0; k < C; ++k) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          if (k == first) start[i] = carry[i];
          const float2 m = block_map[flip][REVERSE ? C - 1 - k : k][i][lane];
          carry[i] = affine<CUT>(m.x, carry[i], m.y);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        start[i] = carry[i];
        float p = pe[i], h = he[i];
        for (int k = before; k < kScanWarps; ++k) {
          const float2 m = warp_map[flip][REVERSE ? kScanWarps - 1 - k : k][i][lane];
          h = affine<CUT>(m.x, h, m.y);
          p *= m.x;
        }
        carry[i] = affine<CUT>(p, carry[i], h);
      }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) start[i] = affine<CUT>(pe[i], start[i], he[i]);
  }
};

// a step's rows lie 32-bit byte offsets apart inside a thread's kEvery steps (checked by the host)
template <typename Raw>
__device__ __forceinline__ Raw load_row(const void* base, int offset) {
  return __ldcs(reinterpret_cast<const Raw*>(static_cast<const char*>(base) + offset));
}
template <typename Raw>
__device__ __forceinline__ void store_row(void* base, int offset, Raw v) {
  __stcs(reinterpret_cast<Raw*>(static_cast<char*>(base) + offset), v);
}
template <bool V>
struct Flag { static constexpr bool value = V; };

// grid (C, channel blocks, batch), clusters of C blocks along x.  Pieces that lie wholly inside the sequence
// take a path without a test a step; the tests of the other path are warp-uniform.
template <typename T, int VEC, int GATE, bool CUT>
__global__ void __launch_bounds__(32 * kScanWarps, 2)
scan_chunk_kernel(const ScanArgs p) {
  using L = Lane<T, VEC>;
  using Raw = typename L::Raw;
  __shared__ Exchange<VEC, CUT, false> ex;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x, C = gridDim.x, b = blockIdx.z;
  const int c = (blockIdx.y * 32 + lane) * VEC;
  const bool live = c < p.D;
  const int n = length_of(p, b);
  const int piece = C * kScanWarps * kEvery;
  const int64_t nst = (p.T + kEvery - 1) / kEvery;
  const int v_row = (int)(p.v_t * sizeof(T)), f_row = (int)(p.f_t * sizeof(T)), y_row = (int)(p.y_t * sizeof(T));
  const int cc = live ? c : 0;       // lanes past the last channel read the first, and store nothing
  Raw rv[kEvery], rf[kEvery];
  auto load = [&](int t0) {
    const T* v = static_cast<const T*>(p.v) + b * p.v_b + cc + t0 * p.v_t;
    const T* f = static_cast<const T*>(p.f) + b * p.f_b + cc + t0 * p.f_t;
    if (t0 + kEvery <= n) {
#pragma unroll
      for (int j = 0; j < kEvery; ++j) {
        rv[j] = load_row<Raw>(v, j * v_row);
        rf[j] = load_row<Raw>(f, j * f_row);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kEvery; ++j) {
        rv[j] = rf[j] = L::zero();
        if (t0 + j < n) {
          rv[j] = load_row<Raw>(v, j * v_row);
          rf[j] = load_row<Raw>(f, j * f_row);
        }
      }
    }
  };
  int t0 = (rank * kScanWarps + warp) * kEvery;
  load(t0);
  cluster_start(C);
  float carry[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) carry[i] = p.h0 ? p.h0[(int64_t)b * p.D + cc + i] : 0.f;
  int flip = 0;
  for (int base = 0; base < p.T; base += piece, t0 += piece, flip ^= 1) {
    float a[kEvery][VEC], in[kEvery][VEC], P[VEC], H[VEC], h[VEC];
    const bool whole = t0 + kEvery <= n;
    auto compose = [&](auto full) {
#pragma unroll
      for (int j = 0; j < kEvery; ++j) {
        float v[VEC], f[VEC];
        L::get(rv[j], v);
        L::get(rf[j], f);
        const bool on = decltype(full)::value || t0 + j < n;
        const bool cut = CUT && on && p.reset[(int64_t)b * p.T + t0 + j] != 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float w;
          gate_of(f[i], a[j][i], w);
          in[j][i] = input_of<GATE>(a[j][i], w) * v[i];
          if (CUT && cut) a[j][i] = 0.f;
          if (!on) { a[j][i] = 1.f; in[j][i] = 0.f; }
          P[i] = j ? P[i] * a[j][i] : a[j][i];
          H[i] = j ? affine<CUT>(a[j][i], H[i], in[j][i]) : in[j][i];
        }
      }
    };
    if (whole) compose(Flag<true>()); else compose(Flag<false>());
    if (base + piece < p.T) load(t0 + piece);
    ex.run(P, H, carry, h, flip, rank, C);
    if (live && t0 < p.T) {
      if (p.states) {
        float* st = p.states + (b * nst + t0 / kEvery) * p.D + c;
#pragma unroll
        for (int i = 0; i < VEC; ++i) st[i] = h[i];
      }
      T* y = static_cast<T*>(p.y) + b * p.y_b + c + t0 * p.y_t;
      auto emit = [&](auto full) {
#pragma unroll
        for (int j = 0; j < kEvery; ++j) {
          float o[VEC];
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            h[i] = affine<CUT>(a[j][i], h[i], in[j][i]);
            o[i] = decltype(full)::value || t0 + j < n ? h[i] : 0.f;
          }
          if (decltype(full)::value || t0 + j < p.T) store_row<Raw>(y, j * y_row, L::put(o));
        }
      };
      if (whole) emit(Flag<true>()); else emit(Flag<false>());
    }
  }
  if (p.h_last && live && rank == 0 && warp == 0)
#pragma unroll
    for (int i = 0; i < VEC; ++i) p.h_last[(int64_t)b * p.D + c + i] = carry[i];
}

// The cotangent runs from the end: a step maps G (the cotangent of the state after it) to
// r a (G + dy), the cotangent of the state before it.  The states before each thread's steps were
// kept by the forward pass, so h needs no exchange.  Over the exchange a thread keeps, per step, 1 - a
// (from which a and u follow), dy and the factor of g in df; resets are a bit mask, the same in all lanes.
template <typename T, int VEC, int GATE, bool CUT>
__global__ void __launch_bounds__(32 * kScanWarps, 2)
scan_chunk_back_kernel(const ScanArgs p) {
  using L = Lane<T, VEC>;
  using Raw = typename L::Raw;
  __shared__ Exchange<VEC, CUT, true> ex;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x, C = gridDim.x, b = blockIdx.z;
  const int c = (blockIdx.y * 32 + lane) * VEC;
  const bool live = c < p.D;
  const int cc = live ? c : 0;
  const int n = length_of(p, b);
  const int piece = C * kScanWarps * kEvery;
  const int64_t nst = (p.T + kEvery - 1) / kEvery;
  const int pieces = (p.T + piece - 1) / piece;
  const int v_row = (int)(p.v_t * sizeof(T)), f_row = (int)(p.f_t * sizeof(T)), y_row = (int)(p.y_t * sizeof(T));
  const int dv_row = (int)(p.dv_t * sizeof(T)), df_row = (int)(p.df_t * sizeof(T));
  cluster_start(C);
  float carry[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) carry[i] = p.dh_last ? p.dh_last[(int64_t)b * p.D + cc + i] : 0.f;
  int flip = 0;
  for (int it = pieces - 1; it >= 0; --it, flip ^= 1) {
    const int t0 = it * piece + (rank * kScanWarps + warp) * kEvery;
    const bool whole = t0 + kEvery <= n;
    Raw rv[kEvery], rf[kEvery], rd[kEvery];
    {
      const T* v = static_cast<const T*>(p.v) + b * p.v_b + cc + t0 * p.v_t;
      const T* f = static_cast<const T*>(p.f) + b * p.f_b + cc + t0 * p.f_t;
      const T* d = static_cast<const T*>(p.dy) + b * p.y_b + cc + t0 * p.y_t;
      if (whole && p.dy) {
#pragma unroll
        for (int j = 0; j < kEvery; ++j) {
          rv[j] = load_row<Raw>(v, j * v_row);
          rf[j] = load_row<Raw>(f, j * f_row);
          rd[j] = load_row<Raw>(d, j * y_row);
        }
      } else {
#pragma unroll
        for (int j = 0; j < kEvery; ++j) {
          rv[j] = rf[j] = rd[j] = L::zero();
          if (t0 + j < n) {
            rv[j] = load_row<Raw>(v, j * v_row);
            rf[j] = load_row<Raw>(f, j * f_row);
            if (p.dy) rd[j] = load_row<Raw>(d, j * y_row);
          }
        }
      }
    }
    float h[VEC], P[VEC], E[VEC], G[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) h[i] = t0 < p.T ? p.states_in[(b * nst + t0 / kEvery) * p.D + cc + i] : 0.f;
    unsigned cuts = 0;
    if (CUT)
#pragma unroll
      for (int j = 0; j < kEvery; ++j)
        if (t0 + j < n && p.reset[(int64_t)b * p.T + t0 + j] != 0) cuts |= 1u << j;
    float w[kEvery][VEC], k[kEvery][VEC];
    auto compose = [&](auto full) {
#pragma unroll
      for (int j = 0; j < kEvery; ++j) {
        float v[VEC], f[VEC];
        L::get(rv[j], v);
        L::get(rf[j], f);
        const bool on = decltype(full)::value || t0 + j < n, cut = CUT && ((cuts >> j) & 1u);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float s;
          gate_of(f[i], s, w[j][i]);
          const float before = cut ? 0.f : h[i], in = input_of<GATE>(s, w[j][i]) * v[i];
          k[j][i] = fmaf(s * w[j][i], before, input_slope<GATE>(s, w[j][i]) * v[i]);
          if (on) h[i] = fmaf(s, before, in);
          if (!on) w[j][i] = 0.f;                     // a = 1: the cotangent passes
        }
      }
#pragma unroll
      for (int j = kEvery - 1; j >= 0; --j) {
        float d[VEC];
        L::get(rd[j], d);
        const bool cut = CUT && ((cuts >> j) & 1u);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float a = 1.f - w[j][i];
          P[i] = j == kEvery - 1 ? a : P[i] * a;
          E[i] = j == kEvery - 1 ? a * d[i] : a * (E[i] + d[i]);
          if (cut) P[i] = E[i] = 0.f;
        }
      }
    };
    if (whole) compose(Flag<true>()); else compose(Flag<false>());
    ex.run(P, E, carry, G, flip, rank, C);
    if (live && t0 < p.T) {
      T* dv = static_cast<T*>(p.dv) + b * p.dv_b + c + t0 * p.dv_t;
      T* df = static_cast<T*>(p.df) + b * p.df_b + c + t0 * p.df_t;
      auto emit = [&](auto full) {
#pragma unroll
        for (int j = kEvery - 1; j >= 0; --j) {
          float d[VEC], ov[VEC], of[VEC];
          L::get(rd[j], d);
          const bool on = decltype(full)::value || t0 + j < n, cut = CUT && ((cuts >> j) & 1u);
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const float a = 1.f - w[j][i], g = G[i] + d[i];
            ov[i] = on ? input_of<GATE>(a, w[j][i]) * g : 0.f;
            of[i] = on ? k[j][i] * g : 0.f;
            G[i] = cut ? 0.f : a * g;
          }
          if (decltype(full)::value || t0 + j < p.T) {
            store_row<Raw>(dv, j * dv_row, L::put(ov));
            store_row<Raw>(df, j * df_row, L::put(of));
          }
        }
      };
      if (whole) emit(Flag<true>()); else emit(Flag<false>());
    }
  }
  if (p.dh0 && live && rank == 0 && warp == 0)
#pragma unroll
    for (int i = 0; i < VEC; ++i) p.dh0[(int64_t)b * p.D + c + i] = carry[i];
}

mw_status check_desc(const mw_gated_scan_desc* d) {
  if (!d || d->batch < 0 || d->length < 0 || d->channels < 1 || d->reserved != 0) return MW_ERR_INVALID_ARG;
  if (d->input_gate != MW_SCAN_COMPLEMENT && d->input_gate != MW_SCAN_ENERGY) return MW_ERR_INVALID_ARG;
  if (d->dtype == 0) return MW_ERR_UNSUPPORTED;
  if (d->dtype != 1 && d->dtype != 2) return MW_ERR_INVALID_ARG;
  if (d->batch > 65535 || d->length > (1 << 30) || d->channels > (1 << 20)) return MW_ERR_UNSUPPORTED;
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

template <typename T, int VEC, int GATE, bool CUT>
mw_status launch_chunks(const ScanArgs& p, bool backward, cudaStream_t s) {
  const int columns = ceil_div(p.D, 32 * VEC);
  const int pieces = ceil_div(p.T, kScanWarps * kEvery);
  // blocks along time until there are two for every SM, as far as there are pieces for them
  int C = 1;
  while (C < kMaxCluster && C < pieces && (int64_t)columns * p.B * C < 2 * 148) C *= 2;
  void (*kernel)(const ScanArgs) = backward ? scan_chunk_back_kernel<T, VEC, GATE, CUT> : scan_chunk_kernel<T, VEC, GATE, CUT>;
  if (C > 8) MW_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)C, (unsigned)columns, (unsigned)p.B);
  cfg.blockDim = dim3(32 * kScanWarps);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)C;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ++g_launch_count;
  return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? MW_OK : MW_ERR_CUDA;
}

template <typename T, int VEC, int GATE>
mw_status run_scan(const ScanArgs& p, bool backward, cudaStream_t s) {
  // up to kEvery steps there is nothing to cut: a thread a channel (the chunks' kernels also hold the offsets
  // of kEvery rows in 32 bits, which only rows more than 2^26 bytes apart do not fit)
  const int64_t most = (int64_t)1 << 26;
  const bool near = p.v_t * (int64_t)sizeof(T) < most && p.f_t * (int64_t)sizeof(T) < most && p.y_t * (int64_t)sizeof(T) < most &&
                    p.dv_t * (int64_t)sizeof(T) < most && p.df_t * (int64_t)sizeof(T) < most;
  if (p.T <= kEvery || !near) {
    const dim3 grid((unsigned)ceil_div(p.D, 128), (unsigned)p.B);
    if (backward) scan_walk_back_kernel<T, GATE><<<grid, 128, 0, s>>>(p);
    else scan_walk_kernel<T, GATE><<<grid, 128, 0, s>>>(p);
    return launch_ok();
  }
  return p.reset ? launch_chunks<T, VEC, GATE, true>(p, backward, s) : launch_chunks<T, VEC, GATE, false>(p, backward, s);
}

template <typename T, int VEC>
mw_status gate_scan(const mw_gated_scan_desc* d, const ScanArgs& p, bool backward, cudaStream_t s) {
  return d->input_gate == MW_SCAN_COMPLEMENT ? run_scan<T, VEC, MW_SCAN_COMPLEMENT>(p, backward, s)
                                             : run_scan<T, VEC, MW_SCAN_ENERGY>(p, backward, s);
}

mw_status dispatch_scan(const mw_gated_scan_desc* d, const ScanArgs& p, bool backward, cudaStream_t s) {
  if (d->dtype == 1) return gate_scan<float, 1>(d, p, backward, s);
  // two bf16 channels a lane where every row of every tensor starts on a 4-byte boundary
  const int64_t odd = p.D | p.v_b | p.v_t | p.f_b | p.f_t | p.y_b | p.y_t | p.dv_b | p.dv_t | p.df_b | p.df_t;
  const uintptr_t at = (uintptr_t)p.v | (uintptr_t)p.f | (uintptr_t)p.y | (uintptr_t)p.dy | (uintptr_t)p.dv | (uintptr_t)p.df;
  return (odd & 1) == 0 && (at & 3) == 0 ? gate_scan<__nv_bfloat16, 2>(d, p, backward, s)
                                         : gate_scan<__nv_bfloat16, 1>(d, p, backward, s);
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
