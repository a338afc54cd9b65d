// Embedding lookup with scaling, and its gradient (mw_embedding_*):
//   out_i = s E[t_i],   dE_v = s sum_{t_i = v} dout_i
// Both directions move rows and compute next to nothing: HBM bounds them (lookup 2 N rows, gradient N rows read and V
// rows written). Measured, bf16: lookup of 16384 in 32768x2048 20 us (6.7 TB/s, tokens met twice included), the table's
// gradient 52 us (201 MB: 3.9 TB/s; zeros and sort 23, sums 22, joins 8, one after another), both of 5003 in 10007x515
// fp32 32 us (rows off 16-byte boundaries, half the tokens the same: four launches of 7 to 9 us). The gradient sorts
// (token, position) by a stable radix sort, so that a token's positions stand in a run, in order; runs are summed in
// float by warps that take 32 entries of the sorted list each, whatever the runs' lengths, and what a run leaves in
// several warps' shares is joined in order afterwards.
//
// Up to 65536 tokens are sorted by one cluster of eight blocks, in their shared memory, while the other blocks of the
// same launch fill the table's gradient with zeros: the sort (9 us) hides behind that. More go through three launches a
// digit. (By those launches, zeros first, 16384 tokens took 49 us before the first sum.)
#include "mw_cluster.cuh"
#include "mw_launch.cuh"

namespace mw {
namespace {

constexpr int kRadixThreads = 256, kRadixKeys = 8;                 // keys a thread
constexpr int kRadixTile = kRadixThreads * kRadixKeys;
constexpr int kRadixBits = 8, kRadixDigits = 1 << kRadixBits;
constexpr int kPiece = 32;                                         // sorted entries that one warp sums

struct EmbedArgs {
  int64_t n;
  int vocab, dim;
  int64_t ld_table, ld_out, ld_dtable;
  float scale;
};

// VEC elements of a row: as they are, and as floats
template <typename T, int VEC>
struct RawOf { using type = uint4; };
template <typename T>
struct RawOf<T, 1> { using type = T; };
template <typename T, int VEC>
__device__ __forceinline__ void widen(const typename RawOf<T, VEC>::type& raw, float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    v[0] = to_f32(raw);
  } else {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (VEC == 4) {
        v[i] = __uint_as_float(w[i]);
      } else {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T* at, float (&v)[VEC]) {
  if (VEC == 1) {
    v[0] = to_f32(at[0]);
  } else if (sizeof(T) == 4) {
    const float4 a = *reinterpret_cast<const float4*>(at);
    v[0] = a.x; v[1 % VEC] = a.y; v[2 % VEC] = a.z; v[3 % VEC] = a.w;
  } else {
    const uint4 a = *reinterpret_cast<const uint4*>(at);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ void put(float* at, float v) { *at = v; }
__device__ __forceinline__ void put(__nv_bfloat16* at, float v) { *at = __float2bfloat16_rn(v); }
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T* at, const float (&v)[VEC]) {
  if (VEC == 1) {
    put(at, v[0]);
  } else if (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i)
      reinterpret_cast<float4*>(at)[i] = make_float4(v[4 * i], v[(4 * i + 1) % VEC], v[(4 * i + 2) % VEC], v[(4 * i + 3) % VEC]);
  } else if (VEC == 4) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1 % VEC]), b = __floats2bfloat162_rn(v[2 % VEC], v[3 % VEC]);
    *reinterpret_cast<uint2*>(at) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[(2 * i) % VEC], v[(2 * i + 1) % VEC]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// the row of a token, or `vocab` where it names none
template <typename I>
__device__ __forceinline__ int row_of(I t, int vocab) { return t >= 0 && t < (I)vocab ? (int)t : vocab; }

// Rows of 64 accesses and more: a warp takes 256 accesses of a row, eight a lane, whose loads are all under way before
// the first store.
constexpr int kLookupAhead = 8;
template <typename T, typename I, int VEC>
__global__ void __launch_bounds__(256)
lookup_kernel(EmbedArgs a, const I* __restrict__ tokens, const T* __restrict__ table, T* __restrict__ out, int segments) {
  after_previous();
  using Raw = typename RawOf<T, VEC>::type;
  const int per = a.dim / VEC, lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), r = w / segments;
  if (r >= a.n) return;
  const int i0 = (int)(w - r * segments) * (32 * kLookupAhead) + lane;
  const int v = row_of(tokens[r], a.vocab);
  const T* from = table + v * a.ld_table;
  T* to = out + r * a.ld_out;
  Raw x[kLookupAhead];
#pragma unroll
  for (int k = 0; k < kLookupAhead; ++k)
    if (v < a.vocab && i0 + 32 * k < per) x[k] = *reinterpret_cast<const Raw*>(from + (i0 + 32 * k) * VEC);
#pragma unroll
  for (int k = 0; k < kLookupAhead; ++k) {
    float y[VEC];
#pragma unroll
    for (int q = 0; q < VEC; ++q) y[q] = 0.f;
    if (v < a.vocab && i0 + 32 * k < per) widen<T, VEC>(x[k], y);
#pragma unroll
    for (int q = 0; q < VEC; ++q) y[q] *= a.scale;
    if (i0 + 32 * k < per) store_vec<T, VEC>(to + (i0 + 32 * k) * VEC, y);
  }
}

// Shorter rows: a block takes `rows` of them, a thread four accesses at a time.
constexpr int kLookupPieces = 4;
template <typename T, typename I, int VEC>
__global__ void __launch_bounds__(256)
short_lookup_kernel(EmbedArgs a, const I* __restrict__ tokens, const T* __restrict__ table, T* __restrict__ out, int rows) {
  after_previous();
  using Raw = typename RawOf<T, VEC>::type;
  const int per = a.dim / VEC;
  const int64_t r0 = (int64_t)blockIdx.x * rows;
  const int here = (int)(a.n - r0 < rows ? a.n - r0 : rows);
  for (int i0 = threadIdx.x; i0 < here * per; i0 += 256 * kLookupPieces) {
    Raw x[kLookupPieces];
    bool in[kLookupPieces];
#pragma unroll
    for (int k = 0; k < kLookupPieces; ++k) {
      const int i = i0 + k * 256, r = i / per, c = (i - r * per) * VEC;
      const int v = i < here * per ? row_of(tokens[r0 + r], a.vocab) : a.vocab;
      in[k] = v < a.vocab;
      if (in[k]) x[k] = *reinterpret_cast<const Raw*>(table + v * a.ld_table + c);
    }
#pragma unroll
    for (int k = 0; k < kLookupPieces; ++k) {
      const int i = i0 + k * 256, r = i / per, c = (i - r * per) * VEC;
      float y[VEC];
#pragma unroll
      for (int q = 0; q < VEC; ++q) y[q] = 0.f;
      if (in[k]) widen<T, VEC>(x[k], y);
#pragma unroll
      for (int q = 0; q < VEC; ++q) y[q] *= a.scale;
      if (i < here * per) store_vec<T, VEC>(out + (r0 + r) * a.ld_out + c, y);
    }
  }
}

// ---- stable radix sort of (token, position) ---------------------------------------------------
// entry i of the unsorted list: its token's row and its position; of a sorted one: what the last pass left
template <typename I>
struct Entries {
  const I* tokens;            // first pass
  const uint32_t *key, *pos;  // later passes
  int vocab;
  __device__ __forceinline__ uint32_t key_at(uint32_t i) const {
    return tokens ? (uint32_t)row_of(tokens[i], vocab) : key[i];
  }
  __device__ __forceinline__ uint32_t pos_at(uint32_t i) const { return tokens ? i : pos[i]; }
};

template <typename I>
__global__ void __launch_bounds__(kRadixThreads)
radix_count_kernel(Entries<I> in, uint32_t n, int shift, uint32_t* __restrict__ counts) {
  __shared__ uint32_t count[kRadixDigits];
  count[threadIdx.x] = 0;
  __syncthreads();
  const uint32_t i0 = blockIdx.x * (uint32_t)kRadixTile;
#pragma unroll
  for (int k = 0; k < kRadixKeys; ++k) {
    const uint32_t i = i0 + k * kRadixThreads + threadIdx.x;
    if (i < n) atomicAdd(&count[(in.key_at(i) >> shift) & (kRadixDigits - 1)], 1u);
  }
  __syncthreads();
  counts[(size_t)threadIdx.x * gridDim.x + blockIdx.x] = count[threadIdx.x];
}

// counts -> first places, over [digit][block]; one block
__global__ void __launch_bounds__(1024) radix_scan_kernel(uint32_t* counts, uint32_t n) {
  __shared__ uint32_t warp_sum[32];
  __shared__ uint32_t carry;
  if (threadIdx.x == 0) carry = 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (uint32_t i0 = 0; i0 < n; i0 += 4096) {
    const uint32_t i = i0 + threadIdx.x * 4;
    uint32_t v[4], sum = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = i + k < n ? counts[i + k] : 0;
      const uint32_t t = v[k];
      v[k] = sum;
      sum += t;
    }
    uint32_t x = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += y;
    }
    __syncthreads();                       // (carry and warp_sum of the last round have been read)
    if (lane == 31) warp_sum[warp] = x;
    __syncthreads();
    uint32_t before = carry + x - sum;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
    uint32_t all = 0;
    if (threadIdx.x == 1023) all = before + sum;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n) counts[i + k] = before + v[k];
    __syncthreads();
    if (threadIdx.x == 1023) carry = all;
    __syncthreads();
  }
}

template <typename I>
__global__ void __launch_bounds__(kRadixThreads)
radix_place_kernel(Entries<I> in, uint32_t n, int shift, const uint32_t* __restrict__ first, uint32_t* __restrict__ key_out,
                   uint32_t* __restrict__ pos_out) {
  constexpr int kWarps = kRadixThreads / 32;
  __shared__ uint32_t count[kWarps][kRadixDigits];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int d = lane; d < kRadixDigits; d += 32) count[warp][d] = 0;
  __syncwarp();
  // a warp's keys are consecutive, 32 a round: a key's rank in its warp counts those of its digit before it
  const uint32_t i0 = blockIdx.x * (uint32_t)kRadixTile + warp * (32 * kRadixKeys) + lane;
  uint32_t key[kRadixKeys], rank[kRadixKeys];
#pragma unroll
  for (int k = 0; k < kRadixKeys; ++k) {
    const uint32_t i = i0 + k * 32;
    const bool on = i < n;
    key[k] = on ? in.key_at(i) : 0;
    const uint32_t d = on ? (key[k] >> shift) & (kRadixDigits - 1) : kRadixDigits;
    const uint32_t same = __match_any_sync(0xffffffffu, d);
    const uint32_t before = on ? count[warp][d] : 0;
    rank[k] = before + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (on && (same >> lane) == 1u) count[warp][d] = before + __popc(same);      // the last lane of the digit
    __syncwarp();
  }
  __syncthreads();
  {
    uint32_t at = first[(size_t)threadIdx.x * gridDim.x + blockIdx.x];
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t c = count[w][threadIdx.x];
      count[w][threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kRadixKeys; ++k) {
    const uint32_t i = i0 + k * 32;
    if (i < n) {
      const uint32_t at = count[warp][(key[k] >> shift) & (kRadixDigits - 1)] + rank[k];
      key_out[at] = key[k];
      pos_out[at] = in.pos_at(i);
    }
  }
}

// ---- the same sort by one cluster, beside blocks that write zeros ------------------------------
constexpr int kSortBlocks = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortRounds = 8;
constexpr int kSortBits = 9, kSortDigits = 1 << kSortBits;
constexpr int kSortMost = kSortBlocks * kSortThreads * kSortRounds;        // tokens
// shared memory: counts a warp, sums, first places; keys and positions of one pass
constexpr size_t kSortFixed = (size_t)kSortWarps * kSortDigits * 2 + 2 * kSortDigits * 4;
constexpr size_t sort_smem(int rounds) { return kSortFixed + (size_t)kSortThreads * rounds * 8; }

// zeros into `count` elements from `to` on, by `threads` threads
template <typename G>
__device__ __forceinline__ void zero_row(G* to, int dim, int thread, int threads, bool wide) {
  if (wide) {
    for (int c = thread; c < dim * (int)sizeof(G) / 16; c += threads) reinterpret_cast<uint4*>(to)[c] = make_uint4(0u, 0u, 0u, 0u);
  } else {
    for (int c = thread; c < dim; c += threads) to[c] = from_f64<G>(0.0);
  }
}

template <typename I, typename G>
__global__ void __cluster_dims__(kSortBlocks, 1, 1) __launch_bounds__(kSortThreads)
sort_kernel(const I* __restrict__ tokens, uint32_t n, int vocab, int passes, int bits, int rounds, uint32_t* __restrict__ key_out,
            uint32_t* __restrict__ pos_out, uint32_t* joins, G* dtable, int dim, int64_t ld, bool wide) {
  after_previous();
  extern __shared__ uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x >= kSortBlocks) {
    // a warp a row
    const int64_t warps = (int64_t)(gridDim.x - kSortBlocks) * kSortWarps;
    for (int64_t r = (int64_t)(blockIdx.x - kSortBlocks) * kSortWarps + warp; r < vocab; r += warps)
      zero_row(dtable + r * ld, dim, lane, 32, wide);
    return;
  }
  uint16_t(*count)[kSortDigits] = reinterpret_cast<uint16_t(*)[kSortDigits]>(smem);
  uint32_t* sum = reinterpret_cast<uint32_t*>(smem + (size_t)kSortWarps * kSortDigits * 2);
  uint32_t* first = sum + kSortDigits;
  uint2* entry = reinterpret_cast<uint2*>(smem + kSortFixed);        // (key, position) that the pass before sent here
  __shared__ uint32_t warp_sum[kSortWarps];
  const int rank = (int)blockIdx.x;
  const uint32_t share = (uint32_t)kSortThreads * rounds, base = rank * share;
  const int digits = 1 << bits;
  if (rank == 0 && threadIdx.x == 0) *joins = 0;
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * bits;
    for (int d = lane; d < digits; d += 32) count[warp][d] = 0;
    __syncwarp();
    // a warp's keys are consecutive, 32 a round: a key's rank in its warp counts those of its digit before it
    uint32_t key[kSortRounds], pos[kSortRounds], before[kSortRounds];
#pragma unroll
    for (int k = 0; k < kSortRounds; ++k) {
      const uint32_t i = (uint32_t)warp * 32 * rounds + k * 32 + lane;
      key[k] = 0xffffffffu;
      pos[k] = 0;
      if (k < rounds && base + i < n) {
        if (pass == 0) {
          key[k] = (uint32_t)row_of(tokens[base + i], vocab);
          pos[k] = base + i;
        } else {
          const uint2 e = entry[i];
          key[k] = e.x;
          pos[k] = e.y;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kSortRounds; ++k) {
      if (k >= rounds) break;
      const bool on = key[k] != 0xffffffffu;
      const uint32_t d = on ? (key[k] >> shift) & (digits - 1) : kSortDigits;
      const uint32_t same = __match_any_sync(0xffffffffu, d);
      const uint32_t had = on ? count[warp][d] : 0;
      before[k] = had + __popc(same & ((1u << lane) - 1u));
      __syncwarp();
      if (on && (same >> lane) == 1u) count[warp][d] = (uint16_t)(had + __popc(same));      // the last lane of the digit
      __syncwarp();
    }
    __syncthreads();
    if (threadIdx.x < digits) {
      uint32_t at = 0;
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = count[w][threadIdx.x];
        count[w][threadIdx.x] = (uint16_t)at;
        at += c;
      }
      sum[threadIdx.x] = at;
    }
    cluster_sync();
    {
      // first place of a digit: all smaller digits, and this one's in the blocks before
      uint32_t all = 0, mine = 0;
      if (threadIdx.x < digits) {
        const uint32_t at = shared_address(sum + threadIdx.x);
#pragma unroll
        for (int r = 0; r < kSortBlocks; ++r) {
          uint32_t c;
          asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(in_rank(at, r)) : "memory");
          all += c;
          if (r < rank) mine += c;
        }
      }
      uint32_t x = all;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, d);
        if (lane >= d) x += y;
      }
      if (lane == 31) warp_sum[warp] = x;
      __syncthreads();
      for (int w = 0; w < warp && w < kSortDigits / 32; ++w) mine += warp_sum[w];
      if (threadIdx.x < digits) first[threadIdx.x] = mine + x - all;
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kSortRounds; ++k) {
      if (k < rounds && key[k] != 0xffffffffu) {
        const uint32_t d = (key[k] >> shift) & (digits - 1);
        const uint32_t to = first[d] + count[warp][d] + before[k];
        if (pass + 1 == passes) {
          key_out[to] = key[k];
          pos_out[to] = pos[k];
        } else {
          const uint32_t r = to / share;
          asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(in_rank(shared_address(entry + (to - r * share)), (int)r)),
                       "r"(key[k]), "r"(pos[k])
                       : "memory");
        }
      }
    }
    cluster_sync();
  }
}

// ---- sums of runs -----------------------------------------------------------------------------
template <typename G>
__global__ void __launch_bounds__(256) zero_rows_kernel(G* dtable, int64_t rows, int dim, int64_t ld, bool wide) {
  for (int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); r < rows; r += (int64_t)gridDim.x * 8)
    zero_row(dtable + r * ld, dim, threadIdx.x & 31, 32, wide);
}

// VEC columns of a row, GVEC of them an access (1 where the rows of the gradient do not lie on boundaries)
template <typename G, int VEC, bool ADD, bool GWIDE>
__device__ __forceinline__ void write_sum(G* at, float (&v)[VEC], float scale) {
  if (ADD) {
    float old[VEC];
    if (GWIDE && VEC > 1 && VEC * sizeof(G) >= 16) {
      constexpr int kPer = VEC > 1 ? 16 / (int)sizeof(G) : 1;
#pragma unroll
      for (int k = 0; k < VEC; k += kPer) {
        float part[kPer];
        load_vec<G, kPer>(at + k, part);
#pragma unroll
        for (int i = 0; i < kPer; ++i) old[(k + i) % VEC] = part[i];
      }
    } else {
#pragma unroll
      for (int k = 0; k < VEC; ++k) old[k] = to_f32(at[k]);
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) v[k] = fmaf(scale, v[k], old[k]);
  } else {
#pragma unroll
    for (int k = 0; k < VEC; ++k) v[k] = scale * v[k];
  }
  if (GWIDE) {
    store_vec<G, VEC>(at, v);
  } else {
#pragma unroll
    for (int k = 0; k < VEC; ++k) put(at + k, v[k]);
  }
}

// A warp sums one piece of the sorted list over 32 VEC MULT columns, MULT accesses a lane and row, eight rows under way
// at a time. A run that lies whole in the piece goes to its row; what a piece holds of a run that came from the piece
// before goes to its first partial sum, of one that starts here and goes on to its second, and the piece is listed for
// the join.
template <typename T, typename G, int VEC, int MULT, bool ADD, bool GWIDE>
__global__ void __launch_bounds__(256)
run_sums_kernel(EmbedArgs a, const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos, const T* __restrict__ dout,
                G* __restrict__ dtable, float* __restrict__ partial, int col_groups, uint32_t* joins) {
  after_previous();
  constexpr int kAhead = 8;
  const int lane = threadIdx.x & 31;
  const uint32_t n = (uint32_t)a.n;
  const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const uint32_t p = (uint32_t)(w / col_groups), i0 = p * kPiece;
  if (i0 >= n) return;
  const int group = (int)(w - (int64_t)p * col_groups);
  const int c = (group * MULT * 32 + lane) * VEC;            // and every 32 VEC columns on
  int count = (int)(n - i0 < kPiece ? n - i0 : kPiece);
  const uint32_t my_key = lane < count ? key[i0 + lane] : 0xffffffffu;
  const uint32_t my_pos = lane < count ? pos[i0 + lane] : 0;
  const uint32_t before = i0 ? key[i0 - 1] : 0xffffffffu;
  const uint32_t after = i0 + kPiece < n ? key[i0 + kPiece] : 0xffffffffu;
  // tokens that name no row come last
  count = __popc(__ballot_sync(0xffffffffu, my_key < (uint32_t)a.vocab));
  float acc[MULT][VEC];
#pragma unroll
  for (int m = 0; m < MULT; ++m)
#pragma unroll
    for (int q = 0; q < VEC; ++q) acc[m][q] = 0.f;
  bool from_before = __shfl_sync(0xffffffffu, my_key, 0) == before;
  const int width = (a.dim + 3) / 4 * 4;
  for (int b = 0; b < count; b += kAhead) {
    using Raw = typename RawOf<T, VEC>::type;
    Raw x[kAhead][MULT];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint32_t r = __shfl_sync(0xffffffffu, my_pos, (b + k) & 31);
      const T* from = dout + r * a.ld_out + c;
#pragma unroll
      for (int m = 0; m < MULT; ++m)
        if (c + m * 32 * VEC < a.dim && b + k < count) x[k][m] = *reinterpret_cast<const Raw*>(from + m * 32 * VEC);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = b + k;
      if (i < count) {
        const uint32_t v = __shfl_sync(0xffffffffu, my_key, i & 31);
        const uint32_t next = i == kPiece - 1 ? after : __shfl_sync(0xffffffffu, my_key, (i + 1) & 31);
#pragma unroll
        for (int m = 0; m < MULT; ++m) {
          if (c + m * 32 * VEC < a.dim) {
            float y[VEC];
            widen<T, VEC>(x[k][m], y);
#pragma unroll
            for (int q = 0; q < VEC; ++q) acc[m][q] += y[q];
          }
        }
        if (next != v || i == kPiece - 1) {
          const bool goes_on = next == v;
#pragma unroll
          for (int m = 0; m < MULT; ++m) {
            const int at = c + m * 32 * VEC;
            if (at < a.dim) {
              if (from_before || goes_on)
                store_vec<float, VEC>(partial + ((size_t)p * 2 + (from_before ? 0 : 1)) * width + at, acc[m]);
              else
                write_sum<G, VEC, ADD, GWIDE>(dtable + v * a.ld_dtable + at, acc[m], a.scale);
            }
#pragma unroll
            for (int q = 0; q < VEC; ++q) acc[m][q] = 0.f;
          }
          if (goes_on && !from_before && group == 0 && lane == 0) joins[1 + atomicAdd(joins, 1u)] = p;
          from_before = false;
        }
      }
    }
  }
}

// A block joins 256 columns of a run that starts in a listed piece and goes on beyond it: the piece's second partial
// sum, then the first ones of the pieces after, each of eight rows of threads every eighth of them, the rows' sums in
// order.  (The order of the list is that of the atomics; what is summed, and how, is not.)
constexpr int kJoinRows = 8, kJoinColumns = 256, kJoinThreads = kJoinRows * kJoinColumns / 4;
template <typename G, bool ADD>
__global__ void __launch_bounds__(kJoinThreads)
join_runs_kernel(EmbedArgs a, const uint32_t* __restrict__ key, const float* __restrict__ partial, G* __restrict__ dtable,
                 const uint32_t* __restrict__ joins) {
  after_previous();
  __shared__ float4 sums[kJoinRows][kJoinColumns / 4];
  const uint32_t n = (uint32_t)a.n;
  const int across = threadIdx.x % (kJoinColumns / 4), down = threadIdx.x / (kJoinColumns / 4);
  const uint32_t groups = (uint32_t)(a.dim + kJoinColumns - 1) / kJoinColumns;
  const int width = (a.dim + 3) / 4 * 4;
  const uint64_t items = (uint64_t)joins[0] * groups;
  for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint32_t p = joins[1 + item / groups];
    const int c = (int)(item % groups) * kJoinColumns + across * 4;
    const uint32_t v = key[p * kPiece + kPiece];
    // the run's last piece: as many pieces after this one begin with it as stand in a row
    const uint32_t pieces = (n + kPiece - 1) / kPiece;
    uint32_t last_piece = p + 1;
    for (uint32_t q = p + 2; q < pieces; q += kJoinThreads) {
      const int more = __syncthreads_count(q + threadIdx.x < pieces && key[(q + threadIdx.x) * kPiece] == v);
      last_piece += (uint32_t)more;
      if (more < kJoinThreads) break;
    }
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < a.dim) {
#pragma unroll 8
      for (uint32_t q = p + 1 + down; q <= last_piece; q += kJoinRows) {
        const float4 x = *reinterpret_cast<const float4*>(partial + (size_t)q * 2 * width + c);
        acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
      }
    }
    sums[down][across] = acc;
    __syncthreads();
    if (down == 0 && c < a.dim) {
      float4 t = *reinterpret_cast<const float4*>(partial + ((size_t)p * 2 + 1) * width + c);
#pragma unroll
      for (int w = 0; w < kJoinRows; ++w) {
        const float4 x = sums[w][across];
        t.x += x.x; t.y += x.y; t.z += x.z; t.w += x.w;
      }
      const float y[4] = {t.x, t.y, t.z, t.w};
      G* to = dtable + v * a.ld_dtable + c;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (c + k < a.dim) {
          float one[1] = {y[k]};
          write_sum<G, 1, ADD, false>(to + k, one, a.scale);
        }
      }
    }
    __syncthreads();
  }
}

struct EmbedScratch {
  uint32_t *key[2], *pos[2], *counts, *joins;
  float* partial;
  uint32_t tiles, pieces;
};
size_t embed_layout(const mw_embedding_desc* d, char* base, EmbedScratch* l) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* p = base + at;
    at += align_up(bytes, 256);
    return p;
  };
  const size_t n = (size_t)d->tokens;
  l->tiles = (uint32_t)((n + kRadixTile - 1) / kRadixTile);
  l->pieces = (uint32_t)((n + kPiece - 1) / kPiece);
  for (int i = 0; i < 2; ++i) {
    l->key[i] = (uint32_t*)take(n * 4);
    l->pos[i] = (uint32_t*)take(n * 4);
  }
  l->counts = (uint32_t*)take((size_t)l->tiles * kRadixDigits * 4);
  l->joins = (uint32_t*)take(((size_t)l->pieces + 1) * 4);
  l->partial = (float*)take((size_t)l->pieces * 2 * align_up((size_t)d->dim, 4) * 4);
  return at + 256;
}

mw_status check_embed(const mw_embedding_desc* d) {
  if (!d || d->tokens < 0 || d->vocab < 1 || d->dim < 1 || d->reserved != 0 || !isfinite((float)d->scale)) return MW_ERR_INVALID_ARG;
  if (d->index_bytes != 4 && d->index_bytes != 8) return MW_ERR_INVALID_ARG;
  if (d->tokens > (1 << 30) || d->dtype == MW_F64 || d->vocab == INT32_MAX) return MW_ERR_UNSUPPORTED;
  if (d->dtype != MW_F32 && d->dtype != MW_BF16_F32ACC) return MW_ERR_INVALID_ARG;
  if (d->grad_dtype != 0 && d->grad_dtype != MW_F32 && d->grad_dtype != MW_BF16_F32ACC) return MW_ERR_INVALID_ARG;
  for (int64_t ld : {d->ld_table, d->ld_out, d->ld_dtable})
    if (ld != 0 && ld < d->dim) return MW_ERR_INVALID_ARG;
  return MW_OK;
}

EmbedArgs embed_args(const mw_embedding_desc* d) {
  EmbedArgs a;
  a.n = d->tokens; a.vocab = d->vocab; a.dim = d->dim;
  a.ld_table = d->ld_table ? d->ld_table : d->dim;
  a.ld_out = d->ld_out ? d->ld_out : d->dim;
  a.ld_dtable = d->ld_dtable ? d->ld_dtable : d->dim;
  a.scale = (float)d->scale;
  return a;
}

// whether pieces of 16 bytes lie on 16-byte boundaries in every row
bool wide_rows(const void* p, int64_t ld, int dim, size_t e) {
  return ((uintptr_t)p & 15) == 0 && (ld * (int64_t)e) % 16 == 0 && ((int64_t)dim * (int64_t)e) % 16 == 0;
}

template <typename T, typename I>
mw_status lookup(const mw_embedding_desc* d, const void* tokens, const void* table, void* out, cudaStream_t s) {
  const EmbedArgs a = embed_args(d);
  constexpr int kVec = 16 / sizeof(T);
  const bool wide = wide_rows(table, a.ld_table, a.dim, sizeof(T)) && wide_rows(out, a.ld_out, a.dim, sizeof(T));
  const int per = wide ? a.dim / kVec : a.dim;
  const I* t = (const I*)tokens;
  if (per >= 64) {
    const int segments = ceil_div(per, 32 * kLookupAhead);
    if (a.n * segments > ((int64_t)1 << 33)) return MW_ERR_UNSUPPORTED;
    return launch_after(wide ? lookup_kernel<T, I, kVec> : lookup_kernel<T, I, 1>, (unsigned)((a.n * segments + 7) / 8), 256, 0, s, a, t,
                        (const T*)table, (T*)out, segments);
  }
  // 1024 accesses a block
  const int rows = 1024 / per;
  return launch_after(wide ? short_lookup_kernel<T, I, kVec> : short_lookup_kernel<T, I, 1>, (unsigned)((a.n + rows - 1) / rows), 256, 0, s, a, t,
                      (const T*)table, (T*)out, rows);
}

// Clusters of the sort that the device holds at once (asked for once a device; at least two).  Allows its
// shared memory, too.
template <typename K>
mw_status sort_clusters(K kernel, int* out) {
  static int clusters[64] = {};
  int dev = 0;
  MW_CUDA_OK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64 || clusters[dev] == 0) {
    MW_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sort_smem(kSortRounds)));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kSortBlocks * 18);
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = sort_smem(kSortRounds);
    int c = 0;
    MW_CUDA_OK(cudaOccupancyMaxActiveClusters(&c, kernel, &cfg));
    if (c < 2) c = 2;
    if (dev < 0 || dev >= 64) { *out = c; return MW_OK; }
    clusters[dev] = c;
  }
  *out = clusters[dev];
  return MW_OK;
}

template <typename T, typename G, int VEC, bool ADD, bool GWIDE>
mw_status sum_runs(const EmbedArgs& a, const EmbedScratch& l, const uint32_t* key, const uint32_t* pos, const T* dout, G* dtable,
                   cudaStream_t s) {
  constexpr int kMult = VEC == 1 ? 4 : 1;
  const int groups = ceil_div(a.dim, 32 * VEC * kMult);
  const int64_t warps = (int64_t)l.pieces * groups;
  if (warps > ((int64_t)1 << 33)) return MW_ERR_UNSUPPORTED;
  MW_TRY(launch_after(run_sums_kernel<T, G, VEC, kMult, ADD, GWIDE>, (unsigned)((warps + 7) / 8), 256, 0, s, a, key, pos, dout, dtable, l.partial, groups, l.joins));
  const int64_t joins = (int64_t)l.pieces * ceil_div(a.dim, kJoinColumns);
  return launch_after(join_runs_kernel<G, ADD>, (unsigned)(joins < 148 * 4 ? joins : 148 * 4), kJoinThreads, 0, s, a, key, l.partial, dtable, l.joins);
}

template <typename T, typename G, typename I>
mw_status table_gradient(const mw_embedding_desc* d, const void* tokens, const void* dout, void* dtable, bool add, char* scratch,
                         cudaStream_t s) {
  const EmbedArgs a = embed_args(d);
  EmbedScratch l;
  embed_layout(d, scratch, &l);
  const uint32_t n = (uint32_t)a.n;
  G* g = (G*)dtable;
  const bool gwide = wide_rows(dtable, a.ld_dtable, a.dim, sizeof(G));
  if (!add && (n == 0 || n > (uint32_t)kSortMost)) {
    zero_rows_kernel<G><<<(unsigned)(a.vocab < 148 * 64 ? ceil_div(a.vocab, 8) : 148 * 8), 256, 0, s>>>(g, a.vocab, a.dim, a.ld_dtable, gwide);
    MW_TRY(launch_ok());
  }
  if (n == 0) return MW_OK;
  int bits = 1;                                   // keys are 0..vocab
  while ((uint32_t)a.vocab >> bits) ++bits;
  const uint32_t *key = l.key[0], *pos = l.pos[0];
  if (n <= (uint32_t)kSortMost) {
    const int passes = ceil_div(bits, kSortBits), rounds = ceil_div(n, kSortBlocks * kSortThreads);
    auto kernel = sort_kernel<I, G>;
    // blocks that write zeros: the clusters that run beside the sort's (one more would begin when the others end), and
    // not more than rows
    int fill = 0;
    if (!add) {
      MW_TRY(sort_clusters(kernel, &fill));
      fill = (fill - 1) * kSortBlocks;
      const int rows = ceil_div(ceil_div(a.vocab, kSortWarps), kSortBlocks) * kSortBlocks;
      if (fill > rows) fill = rows;
    } else {
      MW_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sort_smem(kSortRounds)));
    }
    MW_TRY(launch_after(kernel, (unsigned)(kSortBlocks + fill), kSortThreads, sort_smem(rounds), s, (const I*)tokens, n, a.vocab, passes,
                        ceil_div(bits, passes), rounds, l.key[0], l.pos[0], l.joins, g, a.dim, a.ld_dtable, gwide));
  } else {
    MW_CUDA_OK(cudaMemsetAsync(l.joins, 0, 4, s));
    Entries<I> in = {(const I*)tokens, nullptr, nullptr, a.vocab};
    int to = 0;
    for (int shift = 0; shift < bits; shift += kRadixBits) {
      radix_count_kernel<I><<<l.tiles, kRadixThreads, 0, s>>>(in, n, shift, l.counts);
      radix_scan_kernel<<<1, 1024, 0, s>>>(l.counts, l.tiles * kRadixDigits);
      radix_place_kernel<I><<<l.tiles, kRadixThreads, 0, s>>>(in, n, shift, l.counts, l.key[to], l.pos[to]);
      MW_TRY(launch_ok(3));
      in = {nullptr, l.key[to], l.pos[to], a.vocab};
      to ^= 1;
    }
    key = in.key;
    pos = in.pos;
  }
  const T* y = (const T*)dout;
  constexpr int kVec = 16 / sizeof(T);
  // (a row on 16-byte boundaries in dout's type and in the gradient's: eight or four columns an access in both)
  if (wide_rows(dout, a.ld_out, a.dim, sizeof(T))) {
    if (gwide) return add ? sum_runs<T, G, kVec, true, true>(a, l, key, pos, y, g, s) : sum_runs<T, G, kVec, false, true>(a, l, key, pos, y, g, s);
    return add ? sum_runs<T, G, kVec, true, false>(a, l, key, pos, y, g, s) : sum_runs<T, G, kVec, false, false>(a, l, key, pos, y, g, s);
  }
  return add ? sum_runs<T, G, 1, true, false>(a, l, key, pos, y, g, s) : sum_runs<T, G, 1, false, false>(a, l, key, pos, y, g, s);
}

template <typename T, typename G>
mw_status table_gradient(const mw_embedding_desc* d, const void* tokens, const void* dout, void* dtable, bool add, char* scratch,
                         cudaStream_t s) {
  return d->index_bytes == 4 ? table_gradient<T, G, int32_t>(d, tokens, dout, dtable, add, scratch, s)
                             : table_gradient<T, G, int64_t>(d, tokens, dout, dtable, add, scratch, s);
}

}  // namespace
}  // namespace mw

extern "C" mw_status mw_embedding_forward(const mw_embedding_desc* desc, const void* tokens, const void* table, void* out,
                                          void* stream) {
  using namespace mw;
  MW_TRY(check_embed(desc));
  if (desc->tokens == 0) return MW_OK;
  if (!tokens || !table || !out || out == table) return MW_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  if (desc->dtype == MW_F32)
    return desc->index_bytes == 4 ? lookup<float, int32_t>(desc, tokens, table, out, s)
                                  : lookup<float, int64_t>(desc, tokens, table, out, s);
  return desc->index_bytes == 4 ? lookup<__nv_bfloat16, int32_t>(desc, tokens, table, out, s)
                                : lookup<__nv_bfloat16, int64_t>(desc, tokens, table, out, s);
}

extern "C" mw_status mw_embedding_scratch_bytes(const mw_embedding_desc* desc, size_t* bytes) {
  using namespace mw;
  if (!bytes) return MW_ERR_INVALID_ARG;
  MW_TRY(check_embed(desc));
  EmbedScratch l;
  *bytes = embed_layout(desc, nullptr, &l);
  return MW_OK;
}

extern "C" mw_status mw_embedding_backward(const mw_embedding_desc* desc, const void* tokens, const void* dout, void* dtable,
                                           int32_t accumulate, void* scratch, size_t scratch_bytes, void* stream) {
  using namespace mw;
  MW_TRY(check_embed(desc));
  if ((accumulate != 0 && accumulate != 1) || !dtable || (desc->tokens > 0 && (!tokens || !dout))) return MW_ERR_INVALID_ARG;
  EmbedScratch l;
  if (!scratch || ((uintptr_t)scratch & 255u) || scratch_bytes < embed_layout(desc, nullptr, &l)) return MW_ERR_WORKSPACE;
  if (dtable == dout) return MW_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  char* ws = static_cast<char*>(scratch);
  const bool add = accumulate != 0;
  const int32_t g = desc->grad_dtype ? desc->grad_dtype : desc->dtype;
  if (desc->dtype == MW_F32)
    return g == MW_F32 ? table_gradient<float, float>(desc, tokens, dout, dtable, add, ws, s)
                       : table_gradient<float, __nv_bfloat16>(desc, tokens, dout, dtable, add, ws, s);
  return g == MW_F32 ? table_gradient<__nv_bfloat16, float>(desc, tokens, dout, dtable, add, ws, s)
                     : table_gradient<__nv_bfloat16, __nv_bfloat16>(desc, tokens, dout, dtable, add, ws, s);
}
