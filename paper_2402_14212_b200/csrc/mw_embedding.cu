// Embedding lookup with scaling, and its gradient (mw_embedding_*):
//   out_i = s E[t_i],   dE_v = s sum_{t_i = v} dout_i
// Both directions move rows and compute next to nothing: HBM bounds them (lookup 2 N rows, gradient N rows read
// and V rows written).  The gradient sorts (token, position) by a stable radix sort, so that a token's positions
// stand in a run, in order; runs are summed in float by warps that take 32 entries of the sorted list each,
// whatever the runs' lengths, and what a run leaves in several warps' shares is joined in order afterwards.
#include "mw_common.cuh"

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

// VEC elements of a row as floats
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

// A block takes `rows` whole rows; a thread a piece of VEC columns at a time.
template <typename T, typename I, int VEC>
__global__ void __launch_bounds__(256)
lookup_kernel(EmbedArgs a, const I* __restrict__ tokens, const T* __restrict__ table, T* __restrict__ out, int rows) {
  const int per = a.dim / VEC;
  const int64_t r0 = (int64_t)blockIdx.x * rows;
  const int here = (int)(a.n - r0 < rows ? a.n - r0 : rows);
  for (int i = threadIdx.x; i < here * per; i += 256) {
    const int r = i / per, c = (i - r * per) * VEC;
    const int v = row_of(tokens[r0 + r], a.vocab);
    float x[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) x[k] = 0.f;
    if (v < a.vocab) load_vec<T, VEC>(table + v * a.ld_table + c, x);
#pragma unroll
    for (int k = 0; k < VEC; ++k) x[k] *= a.scale;
    store_vec<T, VEC>(out + (r0 + r) * a.ld_out + c, x);
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

// ---- sums of runs -----------------------------------------------------------------------------
template <typename G>
__global__ void __launch_bounds__(256) zero_rows_kernel(G* dtable, int64_t rows, int dim, int64_t ld) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int c = threadIdx.x; c < dim; c += 256) put(dtable + r * ld + c, 0.f);
}

template <typename G, int VEC, bool ADD>
__device__ __forceinline__ void write_sum(G* at, float (&v)[VEC], float scale) {
  float old[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) old[k] = ADD ? to_f32(at[k]) : 0.f;
#pragma unroll
  for (int k = 0; k < VEC; ++k) v[k] = ADD ? fmaf(scale, v[k], old[k]) : scale * v[k];
#pragma unroll
  for (int k = 0; k < VEC; ++k) put(at + k, v[k]);
}

// A warp sums one piece of the sorted list over 32 VEC columns.  A run that lies whole in the piece goes to its
// row; what a piece holds of a run that came from the piece before goes to its first partial sum, of one
// that starts here and goes on to its second.
template <typename T, typename G, int VEC, bool ADD>
__global__ void __launch_bounds__(256)
run_sums_kernel(EmbedArgs a, const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos, const T* __restrict__ dout,
                G* __restrict__ dtable, float* __restrict__ partial, int col_groups) {
  const int lane = threadIdx.x & 31;
  const uint32_t n = (uint32_t)a.n;
  const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const uint32_t p = (uint32_t)(w / col_groups), i0 = p * kPiece;
  if (i0 >= n) return;
  const int c = ((int)(w - (int64_t)p * col_groups) * 32 + lane) * VEC;
  const bool on = c < a.dim;
  const int count = (int)(n - i0 < kPiece ? n - i0 : kPiece);
  const uint32_t my_key = lane < count ? key[i0 + lane] : 0xffffffffu;
  const uint32_t my_pos = lane < count ? pos[i0 + lane] : 0;
  const uint32_t before = i0 ? key[i0 - 1] : 0xffffffffu;
  const uint32_t after = i0 + kPiece < n ? key[i0 + kPiece] : 0xffffffffu;
  float acc[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) acc[k] = 0.f;
  bool from_before = __shfl_sync(0xffffffffu, my_key, 0) == before;
  for (int i = 0; i < count; ++i) {
    const uint32_t v = __shfl_sync(0xffffffffu, my_key, i), r = __shfl_sync(0xffffffffu, my_pos, i);
    const uint32_t next = __shfl_sync(0xffffffffu, my_key, i + 1 < count ? i + 1 : i);
    if (v >= (uint32_t)a.vocab) break;            // tokens that name no row come last
    if (on) {
      float x[VEC];
      load_vec<T, VEC>(dout + r * a.ld_out + c, x);
#pragma unroll
      for (int k = 0; k < VEC; ++k) acc[k] += x[k];
    }
    const bool last = i + 1 == count, goes_on = last && v == after;
    if (!last && next == v) continue;
    if (on) {
      if (from_before || goes_on) {
        float* to = partial + ((size_t)p * 2 + (from_before ? 0 : 1)) * a.dim + c;
#pragma unroll
        for (int k = 0; k < VEC; ++k) to[k] = acc[k];
      } else {
        write_sum<G, VEC, ADD>(dtable + v * a.ld_dtable + c, acc, a.scale);
      }
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) acc[k] = 0.f;
    from_before = false;
  }
}

// A block joins the run that starts in its piece and goes on beyond it: the piece's second partial sum, then the
// first ones of the pieces after, each warp every eighth of them, the warps' sums in order.
template <typename G, bool ADD>
__global__ void __launch_bounds__(256)
join_runs_kernel(EmbedArgs a, const uint32_t* __restrict__ key, const float* __restrict__ partial, G* __restrict__ dtable) {
  __shared__ float sums[8][32];
  const uint32_t n = (uint32_t)a.n, p = blockIdx.x, i0 = p * kPiece;
  const uint32_t end = i0 + kPiece;
  if (end >= n) return;
  const uint32_t v = key[end];
  if (v >= (uint32_t)a.vocab || key[end - 1] != v || (key[i0] == v && i0 && key[i0 - 1] == v)) return;
  // one past the run's last entry
  uint32_t lo = end, hi = n;
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2;
    if (key[mid] == v) lo = mid + 1; else hi = mid;
  }
  const uint32_t last_piece = (lo - 1) / kPiece;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int c0 = blockIdx.y * 32; c0 < a.dim; c0 += gridDim.y * 32) {
    const int c = c0 + lane;
    float acc = 0.f;
    if (c < a.dim)
      for (uint32_t q = p + 1 + warp; q <= last_piece; q += 8) acc += partial[(size_t)q * 2 * a.dim + c];
    sums[warp][lane] = acc;
    __syncthreads();
    if (warp == 0 && c < a.dim) {
      float t[1] = {partial[((size_t)p * 2 + 1) * a.dim + c]};
      for (int w = 0; w < 8; ++w) t[0] += sums[w][lane];
      write_sum<G, 1, ADD>(dtable + v * a.ld_dtable + c, t, a.scale);
    }
    __syncthreads();
  }
}

struct EmbedScratch {
  uint32_t *key[2], *pos[2], *counts;
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
  l->partial = (float*)take((size_t)l->pieces * 2 * d->dim * 4);
  return at + 256;
}

mw_status check_embed(const mw_embedding_desc* d) {
  if (!d || d->tokens < 0 || d->vocab < 1 || d->dim < 1 || d->reserved != 0 || !isfinite(d->scale)) return MW_ERR_INVALID_ARG;
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
  const int rows = per >= 1024 ? 1 : 1024 / per;
  const unsigned blocks = (unsigned)((a.n + rows - 1) / rows);
  if (wide) lookup_kernel<T, I, kVec><<<blocks, 256, 0, s>>>(a, (const I*)tokens, (const T*)table, (T*)out, rows);
  else lookup_kernel<T, I, 1><<<blocks, 256, 0, s>>>(a, (const I*)tokens, (const T*)table, (T*)out, rows);
  return launch_ok();
}

template <typename T, typename G, int VEC, bool ADD>
mw_status sum_runs(const EmbedArgs& a, const EmbedScratch& l, const uint32_t* key, const uint32_t* pos, const T* dout, G* dtable,
                   cudaStream_t s) {
  const int groups = ceil_div(a.dim, 32 * VEC);
  const int64_t warps = (int64_t)l.pieces * groups;
  if (warps > ((int64_t)1 << 34)) return MW_ERR_UNSUPPORTED;
  run_sums_kernel<T, G, VEC, ADD><<<(unsigned)((warps + 7) / 8), 256, 0, s>>>(a, key, pos, dout, dtable, l.partial, groups);
  const int cols = ceil_div(a.dim, 32);
  join_runs_kernel<G, ADD><<<dim3(l.pieces, (unsigned)(cols < 64 ? cols : 64)), 256, 0, s>>>(a, key, l.partial, dtable);
  return launch_ok(2);
}

template <typename T, typename G, typename I>
mw_status table_gradient(const mw_embedding_desc* d, const void* tokens, const void* dout, void* dtable, bool add, char* scratch,
                         cudaStream_t s) {
  const EmbedArgs a = embed_args(d);
  EmbedScratch l;
  embed_layout(d, scratch, &l);
  if (!add) {
    zero_rows_kernel<G><<<(unsigned)(a.vocab < 148 * 16 ? a.vocab : 148 * 16), 256, 0, s>>>((G*)dtable, a.vocab, a.dim, a.ld_dtable);
    MW_TRY(launch_ok());
  }
  if (a.n == 0) return MW_OK;
  const uint32_t n = (uint32_t)a.n;
  Entries<I> in = {(const I*)tokens, nullptr, nullptr, a.vocab};
  int to = 0;
  // keys are 0..vocab
  for (int shift = 0; shift < 32 && ((uint32_t)a.vocab >> shift) != 0; shift += kRadixBits) {
    radix_count_kernel<I><<<l.tiles, kRadixThreads, 0, s>>>(in, n, shift, l.counts);
    radix_scan_kernel<<<1, 1024, 0, s>>>(l.counts, l.tiles * kRadixDigits);
    radix_place_kernel<I><<<l.tiles, kRadixThreads, 0, s>>>(in, n, shift, l.counts, l.key[to], l.pos[to]);
    MW_TRY(launch_ok(3));
    in = {nullptr, l.key[to], l.pos[to], a.vocab};
    to ^= 1;
  }
  const T* y = (const T*)dout;
  G* g = (G*)dtable;
  constexpr int kVec = 16 / sizeof(T);
  if (wide_rows(dout, a.ld_out, a.dim, sizeof(T)))
    return add ? sum_runs<T, G, kVec, true>(a, l, in.key, in.pos, y, g, s) : sum_runs<T, G, kVec, false>(a, l, in.key, in.pos, y, g, s);
  return add ? sum_runs<T, G, 1, true>(a, l, in.key, in.pos, y, g, s) : sum_runs<T, G, 1, false>(a, l, in.key, in.pos, y, g, s);
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
  if (!tokens || !table || !out) return MW_ERR_INVALID_ARG;
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
