// Gated linear recurrence (mw_gated_scan_*), per channel:
//   a = sigmoid(f),  u = 1 - a or sqrt(1 - a^2),  h_t = r_t a_t h_{t-1} + u_t v_t
// backward, with g_t the whole cotangent of h_t:
//   g_t = dy_t + r_{t+1} a_{t+1} g_{t+1},  dv = u g,  df = a (1 - a) g (r h_{t-1} + u'(a) v)
#include "mw_cluster.cuh"
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

// exp(-f).  The exponent is held below 116, where a is 1e-35 and 1 - a exactly 1: the exponential stays finite.
// NaN stays NaN.
__device__ __forceinline__ float decay_of(float f) {
  float x, e;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(f * -1.4426950408889634f), "f"(116.f));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
  return e;
}
// a = sigmoid(f) and w = 1 - a from exp(-f): one reciprocal gives both ends to their own relative accuracy.  Formed
// by a subtraction, 1 - a would lose the slow channels, where a is close to 1, and a the fast ones.  The product
// f log2(e) is rounded before the exponential, which makes the smaller of the two off by up to (|f| + 4) 2^-24 of
// itself (measured: 5.8e-7 at |f| = 10, 9.5e-7 at 20; 1.6e-7 with the library's exponential).  bf16 results hide it a
// thousand times over; a second term of the product would be two more instructions a gate.
__device__ __forceinline__ void gate_from(float e, float& a, float& w) {
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(1.f + e));
  w = e * a;
}
__device__ __forceinline__ void gate_of(float f, float& a, float& w) { gate_from(decay_of(f), a, w); }
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

// One thread per channel walks the whole sequence: the single steps of serving, short sequences, and rows so far
// apart that the kernels below cannot address them.  Bound by latency: the rows of kAhead steps are asked for before
// the first is used (eight wanted more registers than the waits were worth).
// One step of 64x2048 bf16 takes 2 us, 256x16x2048 14 us forward and 39 backward (50 and 86 MB).
constexpr int kAhead = 4;

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
  auto step = [&](int t, float vt, float ft, bool cut) {
    float a, w;
    gate_of(ft, a, w);
    const float in = input_of<GATE>(a, w) * vt;
    h = cut ? in : fmaf(a, h, in);
    y[t * p.y_t] = from_f32<T>(h);
  };
  static_assert(kEvery % kAhead == 0, "a kept state stands at the start of a stretch");
  int t = 0;
  for (; t + kAhead <= n; t += kAhead) {
    float vs[kAhead], fs[kAhead];
    bool cut[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      fs[j] = to_f32(f[(t + j) * p.f_t]);
      vs[j] = to_f32(v[(t + j) * p.v_t]);
      cut[j] = p.reset && p.reset[(int64_t)b * p.T + t + j];
    }
    if (p.states && t % kEvery == 0) p.states[(b * nst + t / kEvery) * p.D + c] = h;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) step(t + j, vs[j], fs[j], cut[j]);
  }
#pragma unroll 1
  for (; t < p.T; ++t) {
    if (p.states && t % kEvery == 0) p.states[(b * nst + t / kEvery) * p.D + c] = h;
    if (t < n) step(t, to_f32(v[t * p.v_t]), to_f32(f[t * p.f_t]), p.reset && p.reset[(int64_t)b * p.T + t]);
    else y[t * p.y_t] = from_f32<T>(0.f);
  }
  if (p.h_last) p.h_last[bc] = h;
}

// WHOLE: some stretches between kept states are whole (without them the kernel needs half the registers)
template <typename T, int GATE, bool WHOLE>
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
    float h = p.states_in[(b * nst + i) * p.D + c];
    if (WHOLE && t0 + kEvery <= n) {
      float e[kEvery], k[kEvery];                   // exp(-f) and df / g of each step
      unsigned cuts = 0;
#pragma unroll
      for (int q = 0; q < kEvery; q += kAhead) {
        float vs[kAhead], fs[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int t = t0 + q + j;
          fs[j] = to_f32(f[t * p.f_t]);
          vs[j] = to_f32(v[t * p.v_t]);
          if (p.reset && p.reset[(int64_t)b * p.T + t]) cuts |= 1u << (q + j);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          float a, w;
          e[q + j] = decay_of(fs[j]);
          gate_from(e[q + j], a, w);
          const float before = (cuts >> (q + j)) & 1u ? 0.f : h;
          k[q + j] = fmaf(a * w, before, input_slope<GATE>(a, w) * vs[j]);
          h = fmaf(a, before, input_of<GATE>(a, w) * vs[j]);
        }
      }
#pragma unroll
      for (int q = kEvery - kAhead; q >= 0; q -= kAhead) {
        float ds[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) ds[j] = dy ? to_f32(dy[(t0 + q + j) * p.y_t]) : 0.f;
#pragma unroll
        for (int j = kAhead - 1; j >= 0; --j) {
          const int t = t0 + q + j;
          float a, w;
          gate_from(e[q + j], a, w);
          g += ds[j];
          dv[t * p.dv_t] = from_f32<T>(input_of<GATE>(a, w) * g);
          df[t * p.df_t] = from_f32<T>(k[q + j] * g);
          g = (cuts >> (q + j)) & 1u ? 0.f : a * g;
        }
      }
      continue;
    }
    float before[kEvery];
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
constexpr int kMaxCluster = 8;
constexpr int64_t kFewBlocks = 148;      // one block an SM

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

// h -> P h + H.  A map over a reset has P = -0, which no product of gates is (they are positive, and what underflows
// is +0): it drops h whatever it is, so infinities and NaN of what came before a reset do not reach the steps
// after it, while those of a state that has merely decayed do.
constexpr float kCutFactor = -0.f;
__device__ __forceinline__ bool is_cut(float P) { return __float_as_uint(P) == 0x80000000u; }
template <bool CUT>
__device__ __forceinline__ float affine(float P, float h, float H) {
  return CUT && is_cut(P) ? H : fmaf(P, h, H);
}
// the factor of a map P after one of factor Q (a NaN before a reset is dropped with the rest)
template <bool CUT>
__device__ __forceinline__ float chained(float P, float Q) {
  return CUT && is_cut(P) ? P : P * Q;
}

// A product of gates that has underflowed, as the least positive number: an infinite h then stays infinite, as it
// does step by step (0 would make it NaN), and a finite one counts for 5e-7 at the very most.
__device__ __forceinline__ float held(float P) { return __uint_as_float(max(__float_as_uint(P), 1u)); }

// Composes the maps of the block's warps and of the cluster's blocks.  `state` holds what the cluster's next
// piece starts from, the same in all its blocks.  REVERSE: the pieces follow one another from the last warp
// of the last block to the first (the cotangent's direction).
//   - every warp leaves its map; after a barrier each composes those of the warps before it;
//   - the last warp in order then has the block's map and hands it to the copy engine, one copy to each block
//     of the cluster, counted on a barrier there (a cluster-wide barrier instead would also wait for every
//     block's stores to global memory, and measured two to four times slower a piece);
//   - one warp folds the blocks' maps into the state this block starts from and the next piece's.
// Everything is double-buffered by piece.  A buffer is written again two pieces on, by a block that has every
// map of the piece between, which no block sends before all its warps are done with this one.
template <int VEC, bool CUT, bool REVERSE>
struct Exchange {
  float2 warp_map[2][kScanWarps][32][VEC];
  float2 block_map[2][kMaxCluster][32][VEC];
  float2 outgoing[2][32][VEC];
  float block_start[2][32][VEC];
  float state[2][32][VEC];
  unsigned long long arrived[2];

  // before the first piece
  __device__ __forceinline__ void begin(const float (&first)[VEC], int C) {
    if (threadIdx.x < 32)
#pragma unroll
      for (int i = 0; i < VEC; ++i) state[0][threadIdx.x][i] = first[i];
    if (C > 1) {
      if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i)
          asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(shared_address(&arrived[i])) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      }
      cluster_sync();
    } else {
      __syncthreads();
    }
  }
  // after the last: no block leaves while its maps are still being read, or sent to it
  __device__ __forceinline__ void end(int C) {
    if (C > 1) cluster_sync();
    else __syncthreads();
  }

  // in: this thread's map (P, H) of piece `index`; out: the state its steps start from
  __device__ __forceinline__ void run(float (&P)[VEC], const float (&H)[VEC], float (&start)[VEC], int index,
                                      int rank, int C) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, flip = index & 1;
    constexpr uint32_t kBytes = 32 * VEC * sizeof(float2);
#pragma unroll
    for (int i = 0; i < VEC; ++i) P[i] = held(P[i]);
#pragma unroll
    for (int i = 0; i < VEC; ++i) warp_map[flip][warp][lane][i] = make_float2(P[i], H[i]);
    if (C > 1 && threadIdx.x == 0)
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_address(&arrived[flip])),
                   "r"(kBytes * (uint32_t)C)
                   : "memory");
    __syncthreads();
    const int before = REVERSE ? kScanWarps - 1 - warp : warp;
    float pe[VEC], he[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) { pe[i] = 1.f; he[i] = 0.f; }
    for (int k = 0; k < before; ++k) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float2 m = warp_map[flip][REVERSE ? kScanWarps - 1 - k : k][lane][i];
        he[i] = affine<CUT>(m.x, he[i], m.y);
        pe[i] = held(chained<CUT>(m.x, pe[i]));
      }
    }
    const bool last = before == kScanWarps - 1;
    if (C == 1) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float s = state[flip][lane][i];
        start[i] = affine<CUT>(pe[i], s, he[i]);
        if (last) state[flip ^ 1][lane][i] = affine<CUT>(P[i], start[i], H[i]);
      }
      return;
    }
    if (last) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) outgoing[flip][lane][i] = make_float2(held(chained<CUT>(P[i], pe[i])), affine<CUT>(P[i], he[i], H[i]));
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane < C)
        asm volatile(
            "cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                in_rank(shared_address(&block_map[flip][rank][0][0]), lane)),
            "r"(shared_address(&outgoing[flip][0][0])), "r"(kBytes), "r"(in_rank(shared_address(&arrived[flip]), lane))
            : "memory");
    }
    if (warp == 0) {
      const bool ok = wait_phase(shared_address(&arrived[flip]), (uint32_t)(index >> 1) & 1u);
      const int first = REVERSE ? C - 1 - rank : rank;      // blocks before this one
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        float s = ok ? state[flip][lane][i] : __int_as_float(0x7fffffff);      // (maps that never came: NaN)
        for (int k = 0; k < C; ++k) {
          if (k == first) block_start[flip][lane][i] = s;
          const float2 m = block_map[flip][REVERSE ? C - 1 - k : k][lane][i];
          s = affine<CUT>(m.x, s, m.y);
        }
        state[flip ^ 1][lane][i] = s;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VEC; ++i) start[i] = affine<CUT>(pe[i], block_start[flip][lane][i], he[i]);
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
  __shared__ __align__(16) Exchange<VEC, CUT, false> ex;
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
  float carry[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) carry[i] = p.h0 ? p.h0[(int64_t)b * p.D + cc + i] : 0.f;
  ex.begin(carry, C);
  int index = 0;
  for (int base = 0; base < p.T; base += piece, t0 += piece, ++index) {
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
          if (CUT && cut) a[j][i] = kCutFactor;
          if (!on) { a[j][i] = 1.f; in[j][i] = 0.f; }
          P[i] = j ? chained<CUT>(a[j][i], P[i]) : a[j][i];
          H[i] = j ? affine<CUT>(a[j][i], H[i], in[j][i]) : in[j][i];
        }
      }
    };
    if (whole) compose(Flag<true>()); else compose(Flag<false>());
    if (base + piece < p.T) load(t0 + piece);
    ex.run(P, H, h, index, rank, C);
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
  ex.end(C);
  if (p.h_last && live && rank == 0 && warp == 0)
#pragma unroll
    for (int i = 0; i < VEC; ++i) p.h_last[(int64_t)b * p.D + c + i] = ex.state[index & 1][lane][i];
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
  __shared__ __align__(16) Exchange<VEC, CUT, true> ex;
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
  float carry[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) carry[i] = p.dh_last ? p.dh_last[(int64_t)b * p.D + cc + i] : 0.f;
  ex.begin(carry, C);
  int index = 0;
  for (int it = pieces - 1; it >= 0; --it, ++index) {
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
    float e[kEvery][VEC], k[kEvery][VEC];         // exp(-f) and df / g of each step
    auto compose = [&](auto full) {
#pragma unroll
      for (int j = 0; j < kEvery; ++j) {
        float v[VEC], f[VEC], d[VEC];
        L::get(rv[j], v);
        L::get(rf[j], f);
        L::get(rd[j], d);
        const bool on = decltype(full)::value || t0 + j < n, cut = CUT && ((cuts >> j) & 1u);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float a, w;
          e[j][i] = decay_of(f[i]);
          gate_from(e[j][i], a, w);
          const float before = cut ? 0.f : h[i], in = input_of<GATE>(a, w) * v[i];
          k[j][i] = fmaf(a * w, before, input_slope<GATE>(a, w) * v[i]);
          if (on) h[i] = fmaf(a, before, in);
          if (!on) { a = 1.f; e[j][i] = 0.f; }        // the cotangent passes
          // d reaches the state before the first step through all gates up to its own
          if (CUT && cut) a = kCutFactor;
          P[i] = j ? held(chained<CUT>(P[i], a)) : a;
          if (!j) E[i] = 0.f;
          if (!CUT || !is_cut(P[i])) E[i] = fmaf(P[i], d[i], E[i]);
        }
      }
    };
    if (whole) compose(Flag<true>()); else compose(Flag<false>());
    ex.run(P, E, G, index, rank, C);
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
            float a, w;
            gate_from(e[j][i], a, w);
            const float g = G[i] + d[i];
            ov[i] = on ? input_of<GATE>(a, w) * g : 0.f;
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
  ex.end(C);
  if (p.dh0 && live && rank == 0 && warp == 0)
#pragma unroll
    for (int i = 0; i < VEC; ++i) p.dh0[(int64_t)b * p.D + c + i] = ex.state[index & 1][lane][i];
}

// ---------------------------------------------------------------------------------------------
// The same two kernels for rows that start on 16-byte boundaries.  They are bound by latency at 16 warps an SM
// (122 to 128 registers a thread; 60 to 63% of issue slots used), so instructions count twice: a third of those of the
// kernels above are loads, stores and their addresses, a row of 64 or 128 bytes at a time.  Here a warp brings its kEvery rows of each tensor into shared memory by
// asynchronous copies of 16 bytes a lane (four or eight rows an instruction), one piece ahead of its work,
// reads them there at constant offsets, leaves its results in their place and stores those 16 bytes a lane.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_started() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// a warp's rows of one tensor: 32 lanes of VEC channels each
template <typename T, int VEC, int STEPS>
struct Rows {
  static constexpr int kBytes = 32 * VEC * (int)sizeof(T);   // of a row
  static constexpr int kPieces = kBytes / 16;                // lanes that copy one row
  static constexpr int kAtOnce = 32 / kPieces;               // rows of one instruction
  static constexpr int kBlock = STEPS * kBytes;
  static constexpr int kEach = 16 / (int)sizeof(T);          // channels of one copy
  const char* base;
  int64_t row;
  __device__ __forceinline__ Rows(const void* p, int64_t batch, int64_t step, int b, int channel)
      : base(static_cast<const char*>(p) + (b * batch + channel) * (int64_t)sizeof(T)), row(step * (int64_t)sizeof(T)) {}
  // first channel, from the warp's, that this lane copies
  static __device__ __forceinline__ int channel() { return (int)(threadIdx.x % kPieces) * kEach; }
  // rows t0 .. t0 + kEvery - 1, zeros from row `end` on and where this lane has no channels
  __device__ __forceinline__ void fetch(uint32_t to, int t0, int end, bool live) const {
    const int lane = threadIdx.x & 31, first = lane / kPieces;
    const char* from = base + (int64_t)(t0 + first) * row;
    to += (uint32_t)(first * kBytes + (lane % kPieces) * 16);
#pragma unroll
    for (int r = 0; r < STEPS / kAtOnce; ++r) {
      const bool on = live && t0 + first + kAtOnce * r < end;
      copy16(to + (uint32_t)(r * kAtOnce * kBytes), on ? from : base, on);
      from += kAtOnce * row;
    }
  }
  __device__ __forceinline__ void store(const unsigned char* from, int t0, int end, bool live) const {
    const int lane = threadIdx.x & 31, first = lane / kPieces;
    char* to = const_cast<char*>(base) + (int64_t)(t0 + first) * row;
    from += first * kBytes + (lane % kPieces) * 16;
#pragma unroll
    for (int r = 0; r < STEPS / kAtOnce; ++r) {
      const uint4 v = *reinterpret_cast<const uint4*>(from + r * kAtOnce * kBytes);
      if (live && t0 + first + kAtOnce * r < end) __stcs(reinterpret_cast<uint4*>(to), v);
      to += kAtOnce * row;
    }
  }
};

template <typename T, int VEC, int GATE, bool CUT, int STEPS>
__global__ void __launch_bounds__(32 * kScanWarps, 2)
scan_wide_kernel(const ScanArgs p) {
  using R = Rows<T, VEC, STEPS>;
  constexpr int kBlockBytes = R::kBlock, kRowBytes = R::kBytes;
  using L = Lane<T, VEC>;
  using Raw = typename L::Raw;
  __shared__ __align__(16) Exchange<VEC, CUT, false> ex;
  extern __shared__ __align__(128) unsigned char ring[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x, C = gridDim.x, b = blockIdx.z;
  const int c0 = blockIdx.y * 32 * VEC, c = c0 + lane * VEC;
  const bool live = c < p.D;
  const int cc = live ? c : 0;
  const int n = length_of(p, b);
  const int piece = C * kScanWarps * STEPS;
  const int64_t nst = (p.T + kEvery - 1) / kEvery;
  // this warp's two stages of (v, f)
  unsigned char* mine = ring + warp * 4 * kBlockBytes;
  const uint32_t mine_at = shared_address(mine);
  const int cl = c0 + R::channel();       // the channels this lane copies
  const bool copies = cl < p.D;
  const R v_rows(p.v, p.v_b, p.v_t, b, copies ? cl : 0), f_rows(p.f, p.f_b, p.f_t, b, copies ? cl : 0),
      y_rows(p.y, p.y_b, p.y_t, b, copies ? cl : 0);
  int t0 = (rank * kScanWarps + warp) * STEPS;
  auto fetch = [&](int stage, int t) {
    v_rows.fetch(mine_at + (uint32_t)(stage * 2 * kBlockBytes), t, n, copies);
    f_rows.fetch(mine_at + (uint32_t)(stage * 2 * kBlockBytes + kBlockBytes), t, n, copies);
    copies_started();
  };
  fetch(0, t0);
  float carry[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) carry[i] = p.h0 ? p.h0[(int64_t)b * p.D + cc + i] : 0.f;
  ex.begin(carry, C);
  int index = 0;
  for (int base = 0; base < p.T; base += piece, t0 += piece, ++index) {
    const int stage = index & 1;
    __syncwarp();                      // every lane is done with the other stage
    if (base + piece < p.T) {
      fetch(stage ^ 1, t0 + piece);
      copies_done<1>();
    } else {
      copies_done<0>();
    }
    __syncwarp();
    unsigned char* at = mine + stage * 2 * kBlockBytes;
    unsigned char* word = at + lane * (int)sizeof(Raw);
    float a[STEPS][VEC], in[STEPS][VEC], P[VEC], H[VEC], h[VEC];
    const bool whole = t0 + STEPS <= n;
    auto compose = [&](auto full) {
#pragma unroll
      for (int j = 0; j < STEPS; ++j) {
        float v[VEC], f[VEC];
        L::get(*reinterpret_cast<const Raw*>(word + j * kRowBytes), v);
        L::get(*reinterpret_cast<const Raw*>(word + kBlockBytes + j * kRowBytes), f);
        const bool on = decltype(full)::value || t0 + j < n;
        const bool cut = CUT && on && p.reset[(int64_t)b * p.T + t0 + j] != 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float w;
          gate_of(f[i], a[j][i], w);
          in[j][i] = input_of<GATE>(a[j][i], w) * v[i];
          if (CUT && cut) a[j][i] = kCutFactor;
          if (!on) { a[j][i] = 1.f; in[j][i] = 0.f; }
          P[i] = j ? chained<CUT>(a[j][i], P[i]) : a[j][i];
          H[i] = j ? affine<CUT>(a[j][i], H[i], in[j][i]) : in[j][i];
        }
      }
    };
    if (whole) compose(Flag<true>()); else compose(Flag<false>());
    ex.run(P, H, h, index, rank, C);
    if (t0 < p.T) {
      auto emit = [&](auto full) {
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
          float o[VEC];
          if (j % kEvery == 0 && p.states && live && t0 + j < p.T) {
            float* st = p.states + (b * nst + (t0 + j) / kEvery) * p.D + c;
#pragma unroll
            for (int i = 0; i < VEC; ++i) st[i] = h[i];
          }
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            h[i] = affine<CUT>(a[j][i], h[i], in[j][i]);
            o[i] = decltype(full)::value || t0 + j < n ? h[i] : 0.f;
          }
          *reinterpret_cast<Raw*>(word + j * kRowBytes) = L::put(o);
        }
      };
      if (whole) emit(Flag<true>()); else emit(Flag<false>());
      __syncwarp();
      y_rows.store(at, t0, p.T, copies);
    }
  }
  ex.end(C);
  if (p.h_last && live && rank == 0 && warp == 0)
#pragma unroll
    for (int i = 0; i < VEC; ++i) p.h_last[(int64_t)b * p.D + c + i] = ex.state[index & 1][lane][i];
}

template <typename T, int GATE, bool CUT, int STEPS>
__global__ void __launch_bounds__(32 * kScanWarps, 2)
scan_wide_back_kernel(const ScanArgs p) {
  constexpr int VEC = 1;               // (two channels' e and k would leave 16 steps between exchanges)
  using R = Rows<T, VEC, STEPS>;
  constexpr int kBlockBytes = R::kBlock, kRowBytes = R::kBytes;
  using L = Lane<T, VEC>;
  using Raw = typename L::Raw;
  __shared__ __align__(16) Exchange<VEC, CUT, true> ex;
  extern __shared__ __align__(128) unsigned char ring[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x, C = gridDim.x, b = blockIdx.z;
  const int c0 = blockIdx.y * 32 * VEC, c = c0 + lane * VEC;
  const bool live = c < p.D;
  const int cc = live ? c : 0;
  const int n = length_of(p, b);
  const int piece = C * kScanWarps * STEPS;
  const int64_t nst = (p.T + kEvery - 1) / kEvery;
  const int pieces = (p.T + piece - 1) / piece;
  // this warp's two stages of (v, f, dy)
  unsigned char* mine = ring + warp * 6 * kBlockBytes;
  const uint32_t mine_at = shared_address(mine);
  const int cl = c0 + R::channel();
  const bool copies = cl < p.D;
  const int cs = copies ? cl : 0;
  const R v_rows(p.v, p.v_b, p.v_t, b, cs), f_rows(p.f, p.f_b, p.f_t, b, cs), d_rows(p.dy ? p.dy : p.v, p.y_b, p.y_t, b, cs),
      dv_rows(p.dv, p.dv_b, p.dv_t, b, cs), df_rows(p.df, p.df_b, p.df_t, b, cs);
  float next[VEC];                     // the state before this thread's steps of the next piece
  auto fetch = [&](int stage, int t) {
    const uint32_t to = mine_at + (uint32_t)(stage * 3 * kBlockBytes);
    v_rows.fetch(to, t, n, copies);
    f_rows.fetch(to + kBlockBytes, t, n, copies);
    d_rows.fetch(to + 2 * kBlockBytes, t, p.dy ? n : 0, copies);
    copies_started();
#pragma unroll
    for (int i = 0; i < VEC; ++i) next[i] = t < p.T ? p.states_in[(b * nst + t / kEvery) * p.D + cc + i] : 0.f;
  };
  int t0 = (pieces - 1) * piece + (rank * kScanWarps + warp) * STEPS;
  fetch(0, t0);
  float carry[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) carry[i] = p.dh_last ? p.dh_last[(int64_t)b * p.D + cc + i] : 0.f;
  ex.begin(carry, C);
  int index = 0;
  for (int it = pieces - 1; it >= 0; --it, ++index, t0 -= piece) {
    const int stage = index & 1;
    float h[VEC], P[VEC], E[VEC], G[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) h[i] = next[i];
    __syncwarp();                      // every lane is done with the other stage
    if (it > 0) {
      fetch(stage ^ 1, t0 - piece);
      copies_done<1>();
    } else {
      copies_done<0>();
    }
    __syncwarp();
    const bool whole = t0 + STEPS <= n;
    unsigned char* at = mine + stage * 3 * kBlockBytes;
    unsigned char* word = at + lane * (int)sizeof(Raw);
    unsigned cuts = 0;
    if (CUT)
#pragma unroll
      for (int j = 0; j < STEPS; ++j)
        if (t0 + j < n && p.reset[(int64_t)b * p.T + t0 + j] != 0) cuts |= 1u << j;
    float e[STEPS][VEC], k[STEPS][VEC];         // exp(-f) and df / g of each step
    auto compose = [&](auto full) {
#pragma unroll
      for (int j = 0; j < STEPS; ++j) {
        float v[VEC], f[VEC], d[VEC];
        L::get(*reinterpret_cast<const Raw*>(word + j * kRowBytes), v);
        L::get(*reinterpret_cast<const Raw*>(word + kBlockBytes + j * kRowBytes), f);
        L::get(*reinterpret_cast<const Raw*>(word + 2 * kBlockBytes + j * kRowBytes), d);
        const bool on = decltype(full)::value || t0 + j < n, cut = CUT && ((cuts >> j) & 1u);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float a, w;
          e[j][i] = decay_of(f[i]);
          gate_from(e[j][i], a, w);
          const float before = cut ? 0.f : h[i], in = input_of<GATE>(a, w) * v[i];
          k[j][i] = fmaf(a * w, before, input_slope<GATE>(a, w) * v[i]);
          if (on) h[i] = fmaf(a, before, in);
          if (!on) { a = 1.f; e[j][i] = 0.f; }        // the cotangent passes
          // d reaches the state before the first step through all gates up to its own
          if (CUT && cut) a = kCutFactor;
          P[i] = j ? held(chained<CUT>(P[i], a)) : a;
          if (!j) E[i] = 0.f;
          if (!CUT || !is_cut(P[i])) E[i] = fmaf(P[i], d[i], E[i]);
        }
      }
    };
    if (whole) compose(Flag<true>()); else compose(Flag<false>());
    ex.run(P, E, G, index, rank, C);
    if (t0 < p.T) {
      auto emit = [&](auto full) {
#pragma unroll
        for (int j = STEPS - 1; j >= 0; --j) {
          float d[VEC], ov[VEC], of[VEC];
          L::get(*reinterpret_cast<const Raw*>(word + 2 * kBlockBytes + j * kRowBytes), d);
          const bool on = decltype(full)::value || t0 + j < n, cut = CUT && ((cuts >> j) & 1u);
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            float a, w;
            gate_from(e[j][i], a, w);
            const float g = G[i] + d[i];
            ov[i] = on ? input_of<GATE>(a, w) * g : 0.f;
            of[i] = on ? k[j][i] * g : 0.f;
            G[i] = cut ? 0.f : a * g;
          }
          *reinterpret_cast<Raw*>(word + j * kRowBytes) = L::put(ov);
          *reinterpret_cast<Raw*>(word + kBlockBytes + j * kRowBytes) = L::put(of);
        }
      };
      if (whole) emit(Flag<true>()); else emit(Flag<false>());
      __syncwarp();
      dv_rows.store(at, t0, p.T, copies);
      df_rows.store(at + kBlockBytes, t0, p.T, copies);
    }
  }
  ex.end(C);
  if (p.dh0 && live && rank == 0 && warp == 0)
#pragma unroll
    for (int i = 0; i < VEC; ++i) p.dh0[(int64_t)b * p.D + c + i] = ex.state[index & 1][lane][i];
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

// Blocks along time: doubled while the grid leaves SMs without one, as far as there are pieces of the sequence
// for them.  Each doubling costs an exchange a piece: 8x2048x2048 bf16 (256 columns of blocks) takes 39 us with one
// block along time and 51 us with two, 1x65536x1024 (32 of them, energy gate) 465, 294, 155, 119 us with 1, 2, 4, 8.
int blocks_along_time(int64_t columns, int pieces) {
  int C = 1;
  while (C < kMaxCluster && C < pieces && columns * C < kFewBlocks) C *= 2;
  return C;
}

template <int STEPS>
mw_status launch_clusters(void (*kernel)(const ScanArgs), const ScanArgs& p, int columns, size_t ring, cudaStream_t s) {
  static_assert(kMaxCluster <= 8, "larger clusters are not portable");
  if (ring) MW_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ring));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks_along_time((int64_t)columns * p.B, ceil_div(p.T, kScanWarps * STEPS)), (unsigned)columns, (unsigned)p.B);
  cfg.blockDim = dim3(32 * kScanWarps);
  cfg.dynamicSmemBytes = ring;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cfg.gridDim.x;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ++g_launch_count;
  return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? MW_OK : MW_ERR_CUDA;
}

template <typename T, int VEC, int GATE, bool CUT>
mw_status launch_chunks(const ScanArgs& p, bool backward, cudaStream_t s) {
  return launch_clusters<kEvery>(backward ? scan_chunk_back_kernel<T, VEC, GATE, CUT> : scan_chunk_kernel<T, VEC, GATE, CUT>,
                                 p, ceil_div(p.D, 32 * VEC), 0, s);
}
template <typename T, int VEC, int GATE, bool CUT, int STEPS>
mw_status launch_wide(const ScanArgs& p, cudaStream_t s) {
  return launch_clusters<STEPS>(scan_wide_kernel<T, VEC, GATE, CUT, STEPS>, p, ceil_div(p.D, 32 * VEC),
                                (size_t)kScanWarps * 4 * Rows<T, VEC, STEPS>::kBlock, s);
}
template <typename T, int GATE, bool CUT, int STEPS>
mw_status launch_wide_back(const ScanArgs& p, cudaStream_t s) {
  return launch_clusters<STEPS>(scan_wide_back_kernel<T, GATE, CUT, STEPS>, p, ceil_div(p.D, 32),
                                (size_t)kScanWarps * 6 * Rows<T, 1, STEPS>::kBlock, s);
}

// `wide`: every row of every tensor starts on a 16-byte boundary; `pairs`: on a 4-byte one.
// (Inputs above L2, complement gate.)
//   - Where one exchange covers the sequence there is nothing to copy ahead of, and copies only add their latency:
//     direct loads (64x128x2048 bf16, forward and backward: 27 and 40 us; 28 and 72 with copies).  Two bf16 channels a
//     lane if that still gives every SM a block (one channel 38 and 51 us; but 1x512x1024 4.9 us, one channel 4.4).
//   - Longer ones copy ahead (2x8192x1024 f32 backward 61 us, direct loads 74; forward 37 and 39).
//   - bf16 then takes one channel a lane and uses the registers for twice the steps between two exchanges (1x65536x1024
//     forward 108 us; 134 with 16 steps, 200 with two channels; backward 195 and 205 with 16 steps) ...
//   - ... except forward with more columns than the device holds blocks at once, which gains more from half the
//     instructions (8x2048x2048 39 us with two channels, 45 with one; 4x4096x2048, with half the columns, 48 and 44).
template <typename T, int GATE, bool CUT>
mw_status cut_scan(const ScanArgs& p, bool backward, bool wide, bool pairs, cudaStream_t s) {
  constexpr bool kNarrow = sizeof(T) == 2;       // bf16: two channels a lane are possible
  const int pieces = ceil_div(p.T, kScanWarps * kEvery);
  const int64_t columns = (int64_t)ceil_div(p.D, kNarrow ? 64 : 32) * p.B;
  const int C = blocks_along_time(columns, pieces);
  if (!wide || pieces <= C) {
    if constexpr (kNarrow)
      if (pairs && columns * C >= kFewBlocks) return launch_chunks<T, 2, GATE, CUT>(p, backward, s);
    return launch_chunks<T, 1, GATE, CUT>(p, backward, s);
  }
  if constexpr (kNarrow) {
    if (backward) return launch_wide_back<T, GATE, CUT, 2 * kEvery>(p, s);
    return columns < kFewBlocks * 3 / 2 ? launch_wide<T, 1, GATE, CUT, 2 * kEvery>(p, s) : launch_wide<T, 2, GATE, CUT, kEvery>(p, s);
  } else {
    return backward ? launch_wide_back<T, GATE, CUT, kEvery>(p, s) : launch_wide<T, 1, GATE, CUT, kEvery>(p, s);
  }
}

template <typename T, int GATE>
mw_status run_scan(const ScanArgs& p, bool backward, cudaStream_t s) {
  // what every row's place is a multiple of, in bytes
  const int64_t e = sizeof(T);
  const int64_t places = (p.D | p.v_b | p.v_t | p.f_b | p.f_t | p.y_b | p.y_t | p.dv_b | p.dv_t | p.df_b | p.df_t) * e |
                         (int64_t)((uintptr_t)p.v | (uintptr_t)p.f | (uintptr_t)p.y | (uintptr_t)p.dy | (uintptr_t)p.dv | (uintptr_t)p.df);
  // A thread a channel where there is nothing to cut, up to kEvery steps, and up to four times as many (twice in the
  // backward pass) where the channels alone give every SM four blocks.  In us, walked and in chunks, bf16, inputs
  // above L2: 256x32x2048 forward 25 and 81, backward 71 and 113; 64x64x2048 17 and 22, 45 and 29; backward at 48
  // steps even (256x48x2048 104 and 113, 64x48x2048 35 and 29); with few channels 8x64x2048 6.1 and 4.1, 9.3 and 5.3.
  // The chunk kernels also hold the offsets of kEvery rows in 32 bits, which only rows more than 2^26 bytes
  // apart do not fit.
  const int64_t most = (int64_t)1 << 26;
  const bool near = p.v_t * e < most && p.f_t * e < most && p.y_t * e < most && p.dv_t * e < most && p.df_t * e < most;
  const dim3 grid((unsigned)ceil_div(p.D, 128), (unsigned)p.B);
  const int shortest = (int64_t)grid.x * grid.y < 4 * kFewBlocks ? kEvery : backward ? 2 * kEvery : 4 * kEvery;
  if (p.T <= shortest || !near) {
    if (!backward) scan_walk_kernel<T, GATE><<<grid, 128, 0, s>>>(p);
    else if (p.T >= kEvery) scan_walk_back_kernel<T, GATE, true><<<grid, 128, 0, s>>>(p);
    else scan_walk_back_kernel<T, GATE, false><<<grid, 128, 0, s>>>(p);
    return launch_ok();
  }
  const bool wide = (places & 15) == 0, pairs = (places & 3) == 0;
  return p.reset ? cut_scan<T, GATE, true>(p, backward, wide, pairs, s) : cut_scan<T, GATE, false>(p, backward, wide, pairs, s);
}

template <typename T>
mw_status gate_scan(const mw_gated_scan_desc* d, const ScanArgs& p, bool backward, cudaStream_t s) {
  return d->input_gate == MW_SCAN_COMPLEMENT ? run_scan<T, MW_SCAN_COMPLEMENT>(p, backward, s)
                                             : run_scan<T, MW_SCAN_ENERGY>(p, backward, s);
}

mw_status dispatch_scan(const mw_gated_scan_desc* d, const ScanArgs& p, bool backward, cudaStream_t s) {
  return d->dtype == 1 ? gate_scan<float>(d, p, backward, s) : gate_scan<__nv_bfloat16>(d, p, backward, s);
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
