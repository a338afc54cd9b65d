// Orthogonalised momentum update (mw_orth_*):
//   U from gradient and momentum, X_0 = U / ||U||_F, `steps` times
//     A = X X^T,   B = c1 A + c2 A^2,   X <- c0 X + B X          (X with its shorter side as rows)
//   W' = keep W - step X
// Two small kernels form X_0; all products of all steps and matrices are one persistent launch.
//
// Numbers.  The products run on the tensor cores with fp16 operands and fp32 accumulators.  fp16 has
// three more bits than bf16 at the same rate, and what it lacks in range a power of two supplies: X is
// held times Sx (64 sqrt(n): rows of X have norm about one), A and B times Sa.  Rounding is kept out of
// the sums that cancel: X is stored as a pair (leading term and remainder), the c0 X of its update reads
// both, and only the product B X sees the leading term alone; in the last two steps, where the spectrum
// has reached its plateau, A is stored as A - alpha I and B as B + beta I (with c0 - beta in front of X), so
// that what is rounded is the small difference.  One-term operands then give X to about 1e-3 (2e-3 at
// rank-deficient U), where bf16 operands gave 1e-2 to 6e-2 on the same matrices: less than the 2e-3 that
// rounding X to bf16 costs, which is why bf16 weights of 32 rows and more take them by default, but more than 32-bit
// products would leave.  Two-term operands (leading term and remainder, three products of four) give fp32 accuracy, at three
// times the work: 2 of 4096 x 4096 with bf16 weights 2.9 ms with one term, 9.0 ms with two.
//
// A and B are symmetric: tiles on and above the diagonal are computed, the others stored as their
// transposes, 3 m^2 n + m^3 flops a step instead of 4 m^2 n + 2 m^3.
//
// One CTA pair (cta_group::2) owns a 256 x 256 tile; the tiles of one phase follow the other's in one
// list that the pairs take round-robin.  A tile waits only for the ROWS of tiles it reads (counters in
// global memory), so a phase starts while the last tiles of the one before it still run; every wait is
// bounded, and a tile depends on earlier tiles of the list only, which co-resident pairs complete.
#include <cuda_fp16.h>
#include <math.h>

#include <mutex>
#include <new>

#include "mw_tc_gemm.cuh"
#include "mw_tc_ptx.cuh"

namespace mw {
namespace {
constexpr int kOrthMaxSteps = 16;
}
}  // namespace mw

struct mw_orth {
  mw_orth_desc d;
  int m, n;            // shorter and longer side
  bool tall;           // rows > cols: the iterate is the transpose
  int steps, terms;
  double c[3];
  int mp, np;          // padded sides: multiples of 256 and 128
  bool small;          // one CTA a matrix, everything in shared memory
  uint32_t unmet_ms = 0;     // self-test: a wait that nothing meets, and its limit (0: none)
  // tensor maps of a workspace, encoded when the workspace first comes along; calls on one plan may come from
  // several threads, so they are read and written under the lock
  std::mutex lock;
  const void* mapped = nullptr;
  CUtensorMap maps[13];
};

namespace mw {
namespace {

constexpr int kNormBlocks = 592;      // most partial sums of ||U||^2 per matrix
constexpr int kPtrGroup = 64;         // matrices of one launch of the small kernels
constexpr int kTmemColumns = 512;
constexpr int kTile = 256;            // rows and columns of a pair's tile
constexpr int kHalf = 128;            // ... of one CTA's share
constexpr int kBK = 64;
constexpr int kOrthThreads = 384;     // producer warp, issuing warp, two idle ones; eight epilogue warps
constexpr int kOrthFirstEpi = 4;
constexpr int kOrthEpi = 8;
// registers a thread: the launch gives 384 x 168 = 64512, handed over as 128 x 104 + 256 x 200 = 64512
constexpr int kFewRegisters = 104, kManyRegisters = 200;
// K blocks that one accumulator takes of a two-term product.  The tensor core truncates its accumulator at
// every instruction; over 64 K blocks of fp32-accurate products that came to errors of 1e-5 to 1e-4 of X, in
// pieces of 4 blocks that the epilogue adds, rounding to nearest, to 2e-6 (an accumulator of their own for the
// cross products changed nothing).  Pieces want accumulators to run ahead into while the epilogue stores a tile:
// two-term tiles are 128 columns wide, which makes four of them (64 matrices of 1024 x 1024: 6.1 ms; 6.5 ms with two
// of 256 columns, where the products wait for the epilogue).  The two-term epilogue spills: 268 bytes a thread
// stored, 344 loaded, of sums and mirrored rows held at once.
constexpr int kPieceBlocks = 4;
__host__ __device__ constexpr int set_columns(int terms) { return terms == 1 ? 256 : 128; }
__host__ __device__ constexpr int set_count(int terms) { return kTmemColumns / set_columns(terms); }
constexpr int kOrthStagesMax = 4;
constexpr uint32_t kPlaneBytes = kHalf * kBK * 2;      // one operand plane of one stage and CTA
constexpr int kPass = 32;                              // columns an epilogue warp takes at a time
constexpr uint32_t kPassPlane = 32 * kPass * 2;        // one fp16 plane of such a block
constexpr uint32_t kBuffer = 2 * kPassPlane;
// buffers of an epilogue warp: two-term products need the room for their stages more, and have the time
__host__ __device__ constexpr int staging_buffers(int terms) { return terms == 1 ? 3 : 1; }
constexpr int kMaxSide = 32768;
constexpr uint64_t kOrthWaitNs = 2000000000ull;

// operands: K-major rows, MN-major rows; blocks that an epilogue warp reads and writes
// (MAP_XK64, MAP_A64: 64 rows for the second operand of a tile of 128 columns)
enum { MAP_XK = 0, MAP_XMN = 2, MAP_XO = 4, MAP_A = 6, MAP_B, MAP_AO, MAP_BO, MAP_XK64, MAP_A64 = 12, MAP_COUNT };

struct OrthPtrs {
  const void* u[kPtrGroup];
  const float* g[kPtrGroup];
  const float* m[kPtrGroup];
  float* mo[kPtrGroup];
  const void* w[kPtrGroup];      // params (null: X itself is stored) and outputs
  void* out[kPtrGroup];
};

// factors of the three products' epilogues (see the top of the file)
struct OrthFactors {
  float a_scale, b_acc, x_acc, out_scale;
  float a_diag[kOrthMaxSteps], b_add[kOrthMaxSteps], b_diag[kOrthMaxSteps], x_add[kOrthMaxSteps];
};

struct alignas(64) OrthParams {
  CUtensorMap map[MAP_COUNT];
  int count, tm, tn, steps, per_step, total;
  int bn_sym, bn_x, sym_tiles;   // tile widths; tiles of a symmetric product (tn counts those of B X)
  int kb_m, kb_n;                // K blocks of a sum over m and over n
  int piece_blocks;              // K blocks of one accumulator (0: all)
  int mp, np, stages;
  uint32_t stage_bytes;
  OrthFactors f;
  unsigned* done;                // [step][phase][matrix][row of tiles]
  DeviceStatus* st;
  uint64_t wait_ns;
  unsigned unmet;                // self-test: counts that B's tiles wait for and nothing adds
};

struct OrthUnit { int step, phase, mat, ti, tj, n0, bn, nkb, pieces; };      // tj: the row of tiles that column n0 mirrors to

// place t of a triangle of tiles (i, j >= i): row by row, or column by column
__device__ __forceinline__ void triangle_rows(int t, int tm, int& i, int& j) {
  i = 0;
  while (t >= tm - i) { t -= tm - i; ++i; }
  j = i + t;
}
__device__ __forceinline__ void triangle_columns(int t, int& i, int& j) {
  j = 0;
  while (t > j) { t -= j + 1; ++j; }
  i = t;
}

__device__ __forceinline__ OrthUnit orth_unit(const OrthParams& p, int u) {
  OrthUnit w;
  w.step = u / p.per_step;
  int r = u - w.step * p.per_step;
  const int sym = p.count * p.sym_tiles;
  if (r < 2 * sym) {
    w.phase = r >= sym;
    r -= w.phase * sym;
    w.mat = r / p.sym_tiles;
    r -= w.mat * p.sym_tiles;
    w.bn = p.bn_sym;
    int half = 0;
    if (w.bn < kTile) { half = r & 1; r >>= 1; }
    // A's rows are completed early for B; B waits for them in the order they come
    if (w.phase == 0) triangle_rows(r, p.tm, w.ti, w.tj);
    else triangle_columns(r, w.ti, w.tj);
    w.n0 = w.tj * kTile + half * w.bn;
    w.nkb = w.phase == 0 ? p.kb_n : p.kb_m;
  } else {
    r -= 2 * sym;
    w.phase = 2;
    const int per = p.tm * p.tn;
    w.mat = r / per;
    r -= w.mat * per;
    w.ti = r / p.tn;
    w.n0 = (r - w.ti * p.tn) * p.bn_x;
    w.tj = 0;
    w.nkb = p.kb_m;
    w.bn = p.np - w.n0 < p.bn_x ? kHalf : p.bn_x;
  }
  w.pieces = p.piece_blocks ? (w.nkb + p.piece_blocks - 1) / p.piece_blocks : 1;
  return w;
}

__device__ __forceinline__ const unsigned* row_counter(const OrthParams& p, int step, int phase, int mat, int row) {
  return p.done + (((size_t)step * 3 + phase) * p.count + mat) * p.tm + row;
}

__device__ __forceinline__ void umma_f16(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  umma_bf16<true>(d, a, b, idesc, acc);       // kind::f16: the instruction descriptor names the type
}

__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half2(uint32_t v) {
  return __half22float2(*reinterpret_cast<const __half2*>(&v));
}

// byte offset of 16-byte piece c of row r in a block of 64-byte rows under the tensor map's 64-byte swizzle: the
// lanes of a warp, a row each, then meet distinct banks
__device__ __forceinline__ uint32_t piece_at(uint32_t r, uint32_t c) { return r * 64u + ((c ^ ((r >> 1) & 3u)) << 4); }
// wait_done without pauses at first: a tile's rows are often about to be complete
__device__ __forceinline__ bool wait_rows(const unsigned* counter, unsigned target, const WaitCtx& wc) {
  for (int i = 0; i < 64; ++i) {
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(counter) : "memory");
    if (v >= target) return true;
  }
  return wait_done(counter, target, wc);
}
// barriers of the epilogue warps alone; the first tells all of them whether any gave up
__device__ __forceinline__ bool epilogue_any(bool failed) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.or.aligned.pred q, 1, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)failed), "n"(kOrthEpi * 32)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ void epilogue_sync() { asm volatile("barrier.cta.sync.aligned 2, %0;" ::"n"(kOrthEpi * 32) : "memory"); }
// counts after everything this thread has written (or knows written) is visible to the device
__device__ __forceinline__ void count_up(unsigned* counter) {
  asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(counter) : "memory");
}

template <typename T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <int TERMS>
__global__ void __launch_bounds__(kOrthThreads, 1)
orth_products_kernel(const __grid_constant__ OrthParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[kOrthStagesMax];
  __shared__ __align__(8) uint64_t empty_bar[kOrthStagesMax];
  constexpr int kSets = set_count(TERMS), kSetColumns = set_columns(TERMS);
  __shared__ __align__(8) uint64_t acc_full[kSets];
  __shared__ __align__(8) uint64_t acc_empty[kSets];
  __shared__ __align__(8) uint64_t add_full[kOrthEpi * staging_buffers(TERMS)];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_cta_rank();
  const uint32_t tiles = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int pairs = (int)(gridDim.x >> 1), pair = (int)(blockIdx.x >> 1);

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(smem_u32(&full_bar[s]), 1);
      mbar_init(smem_u32(&empty_bar[s]), 1);
    }
    for (int s = 0; s < kSets; ++s) {
      mbar_init(smem_u32(&acc_full[s]), 1);
      mbar_init(smem_u32(&acc_empty[s]), kOrthEpi * 2);
    }
    for (int s = 0; s < kOrthEpi * staging_buffers(TERMS); ++s) mbar_init(smem_u32(&add_full[s]), 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)),
                 "r"((uint32_t)kTmemColumns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  WaitCtx wc;
  wc.st = p.st;
  wc.abort_flag = &abort_flag;
  wc.limit_ns = p.wait_ns;
  const unsigned sym_rows = (unsigned)(p.tm * (kTile / p.bn_sym)) * 2 + p.unmet, x_rows = (unsigned)p.tn * 2;      // one count a CTA and tile

  if (warp < kOrthFirstEpi) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegisters));
  else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegisters));

  if (warp == 0) {
    // ---------------- TMA producer ----------------
    uint32_t stage = 0, phase = 0;
    const uint32_t full0 = smem_u32(&full_bar[0]), empty0 = smem_u32(&empty_bar[0]);
    const uint32_t full0_remote = map_to_cta(full0, 0u);
    bool ok = true;
    for (int u = pair; u < p.total && ok; u += pairs) {
      const OrthUnit w = orth_unit(p, u);
      // the rows this tile reads, each polled by a lane of its own
      if (w.phase == 0) {
        if (w.step > 0 && lane < 2)
          ok = wait_rows(row_counter(p, w.step - 1, 2, w.mat, lane ? w.tj : w.ti), x_rows, wc);
      } else if (w.phase == 1) {
        if (lane < 2) ok = wait_rows(row_counter(p, w.step, 0, w.mat, lane ? w.tj : w.ti), sym_rows, wc);
      } else {
        if (lane == 0) ok = wait_rows(row_counter(p, w.step, 1, w.mat, w.ti), sym_rows, wc);
        if (w.step > 0)
          for (int r = lane; r < p.tm && ok; r += 32) ok = wait_rows(row_counter(p, w.step - 1, 2, w.mat, r), x_rows, wc);
      }
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (lane == 0) {
        asm volatile("fence.proxy.async;" ::: "memory");     // the rows' stores, then our copies
        const int buf = w.step & 1;
        const CUtensorMap* ta = w.phase == 0 ? &p.map[MAP_XK + buf] : (w.phase == 1 ? &p.map[MAP_A] : &p.map[MAP_B]);
        const int plane_a = w.mat * (w.phase == 0 ? 2 : TERMS);
        const CUtensorMap* tb = w.phase == 2 ? &p.map[MAP_XMN + buf]
                                             : (w.bn == kTile ? ta : (w.phase == 0 ? &p.map[MAP_XK64 + buf] : &p.map[MAP_A64]));
        const int am0 = w.ti * kTile + (int)rank * kHalf;
        const int half = w.bn >> 1;
        const int bn0 = w.n0 + (int)rank * half;
        const uint32_t b_off = TERMS * kPlaneBytes, b_plane = (uint32_t)half * (kBK * 2);
        const uint32_t tx = 2u * TERMS * (kPlaneBytes + b_plane);
        for (int kb = 0; kb < w.nkb; ++kb) {
          if (!mbar_wait<true>(empty0 + 8u * stage, phase ^ 1u, wc, 1u)) { ok = false; break; }
          if (rank == 0) mbar_expect_tx(full0 + 8u * stage, tx);
          const uint32_t fb = full0_remote + 8u * stage;
          const uint32_t base = tiles + stage * p.stage_bytes;
          const int k0 = kb * kBK;
          tma_load_3d<true>(base, ta, fb, k0, am0, plane_a);
          if (w.phase != 2) {
            tma_load_3d<true>(base + b_off, tb, fb, k0, bn0, plane_a);
          } else {
            for (int t = 0; t < TERMS; ++t)
              for (int g = 0; g < half; g += 64)
                tma_load_3d<true>(base + b_off + (uint32_t)t * b_plane + (uint32_t)g * (kBK * 2), tb, fb, bn0 + g, k0,
                                  w.mat * 2 + t);
          }
          if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; }
        }
      }
      ok = __all_sync(0xffffffffu, ok);
    }
  } else if (warp == 1) {
    // ---------------- issuing lane (even CTA) ----------------
    if (lane == 0 && rank == 0) {
      uint32_t stage = 0, phase = 0;
      const uint32_t full0 = smem_u32(&full_bar[0]), empty0 = smem_u32(&empty_bar[0]);
      int j = 0;
      bool ok = true;
      for (int u = pair; u < p.total && ok; u += pairs) {
        const OrthUnit w = orth_unit(p, u);
        const bool mn = w.phase == 2;
        // fp32 accumulator, fp16 operands, B's major-ness, N / 8, M / 16
        const uint32_t idesc = (1u << 4) | ((mn ? 1u : 0u) << 16) | ((uint32_t)(w.bn >> 3) << 17) |
                               ((uint32_t)(kTile >> 4) << 24);
        const uint32_t a_base = 1u << 16, b_base = (mn ? (8192u >> 4) : 1u) << 16;
        const uint32_t b_adv = mn ? (2048u >> 4) : (32u >> 4);
        const uint32_t b_off = TERMS * kPlaneBytes, b_plane = (uint32_t)(w.bn >> 1) * (kBK * 2);
        const int piece = p.piece_blocks ? p.piece_blocks : w.nkb;
        for (int kb0 = 0; kb0 < w.nkb && ok; kb0 += piece, ++j) {
          const uint32_t set = (uint32_t)j % kSets, aphase = ((uint32_t)j / kSets) & 1u;
          if (!mbar_wait<true>(smem_u32(&acc_empty[set]), aphase ^ 1u, wc, 2u)) { ok = false; break; }
          tc_fence_after();
          const uint32_t d = tmem_base + set * (uint32_t)kSetColumns;
          const int kb1 = kb0 + piece < w.nkb ? kb0 + piece : w.nkb;
          bool ready = mbar_try_wait<true>(full0 + 8u * stage, phase);
          for (int kb = kb0; kb < kb1; ++kb) {
            if (!ready && !mbar_wait<true>(full0 + 8u * stage, phase, wc, 3u)) { ok = false; break; }
            tc_fence_after();
            const uint32_t sb = tiles + stage * p.stage_bytes;
            const uint32_t a0 = (sb >> 4) | a_base, b0 = ((sb + b_off) >> 4) | b_base;
            umma_f16(d, a0, b0, idesc, kb > kb0);
            if (TERMS == 2) {
              umma_f16(d, a0, b0 + (b_plane >> 4), idesc, 1u);
              umma_f16(d, a0 + (kPlaneBytes >> 4), b0, idesc, 1u);
            }
            // the next stage's barrier is polled while the first products run
            const uint32_t freed = empty0 + 8u * stage;
            if (++stage == (uint32_t)p.stages) { stage = 0; phase ^= 1u; }
            ready = kb + 1 < kb1 && mbar_try_wait<true>(full0 + 8u * stage, phase);
#pragma unroll
            for (int k = 1; k < kBK / 16; ++k) {
              const uint32_t a = a0 + (uint32_t)k * (32u >> 4), b = b0 + (uint32_t)k * b_adv;
              umma_f16(d, a, b, idesc, 1u);
              if (TERMS == 2) {
                umma_f16(d, a, b + (b_plane >> 4), idesc, 1u);
                umma_f16(d, a + (kPlaneBytes >> 4), b, idesc, 1u);
              }
            }
            umma_commit<true>(freed);
          }
          if (ok) umma_commit<true>(smem_u32(&acc_full[set]));
        }
      }
    }
  } else if (warp >= kOrthFirstEpi) {
    // ---------------- epilogue ----------------
    // A tensor-memory lane quarter and one half of the tile's columns each, taken kPass columns at a time (sixteen
    // warps with a quarter each measured a fifth slower).  The
    // copy engine brings a block's addend (both planes of X, or A) into one of the warp's buffers, each lane
    // replaces its row by the result, and the engine takes it away again.  With three buffers (one term) addends
    // are fetched ahead: of X's four passes three before the sum is there and the fourth once the first's
    // result has been read; of A's two, then one pass ahead, the third buffer being for transposed blocks.
    const int ew = warp - kOrthFirstEpi, quarter = warp & 3, side = ew >> 2;
    constexpr int kBuffers = staging_buffers(TERMS);
    const uint32_t sbuf = tiles + (uint32_t)p.stages * p.stage_bytes + (uint32_t)ew * (kBuffers * kBuffer);
    const uint32_t add_bar = smem_u32(&add_full[ew * kBuffers]);
    uint32_t add_phase = 0;              // a bit per buffer
    int j = 0;
    bool failed = false;                 // a wait ran out: all epilogue warps leave together
    // lane 0: start an addend's copy into a buffer whose last result the engine has read
    auto fetch = [&](const CUtensorMap* map, uint32_t buffer, int col, int row, int plane, int planes) {
      mbar_expect_tx(add_bar + 8u * buffer, (uint32_t)planes * kPassPlane);
      tma_load_3d<false>(sbuf + buffer * kBuffer, map, add_bar + 8u * buffer, col, row, plane);
    };
    auto hand_over = [&](const CUtensorMap* map, uint32_t src, int col, int row, int plane) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) bulk_store_3d(map, src, col, row, plane);
    };
    // eight elements of this lane's row, first .. first + 7, into rows of the transposed block: element i goes
    // to row i, column `lane`, so the two-byte stores of a warp fill one 64-byte row
    auto store_turned = [&](uint32_t base, uint32_t first, const uint32_t (&pk)[4]) {
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t at = base + piece_at(first + i, (uint32_t)lane >> 3) + ((uint32_t)lane & 7u) * 2u;
        asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"((unsigned short)(i & 1 ? pk[i / 2] >> 16 : pk[i / 2] & 0xffffu)) : "memory");
      }
    };
    for (int u = pair; u < p.total; u += pairs) {
      const OrthUnit w = orth_unit(p, u);
      const int row0 = w.ti * kTile + (int)rank * kHalf + quarter * 32, row = row0 + lane;
      const int cols = w.bn >> 1, n0 = w.n0 + side * cols;      // this warp's columns
      const int addends = w.phase == 0 ? 0 : (w.phase == 1 ? TERMS : 2);
      const CUtensorMap* from = w.phase == 1 ? &p.map[MAP_AO] : &p.map[MAP_XO + (w.step & 1)];
      const CUtensorMap* to = w.phase == 0 ? &p.map[MAP_AO] : (w.phase == 1 ? &p.map[MAP_BO] : &p.map[MAP_XO + ((w.step + 1) & 1)]);
      const int plane0 = w.mat * (w.phase == 2 ? 2 : TERMS);
      // the addend's rows are complete before its first block is fetched, ahead of the sum
      bool ok = true;
      if (ew == 0 && lane == 0) {
        if (w.phase == 1) ok = wait_rows(row_counter(p, w.step, 0, w.mat, w.ti), sym_rows, wc);
        else if (w.phase == 2 && w.step > 0) ok = wait_rows(row_counter(p, w.step - 1, 2, w.mat, w.ti), x_rows, wc);
      }
      __syncwarp();
      if (epilogue_any(!ok || failed)) break;
      if (lane == 0 && addends) {
        asm volatile("fence.proxy.async;" ::: "memory");
        const int ahead = TERMS == 2 ? 1 : (w.phase == 2 ? 3 : 2);
        for (int k = 0; k < ahead && k * kPass < cols; ++k) fetch(from, (uint32_t)k, n0 + k * kPass, row0, plane0, addends);
      }
      // Two terms: the pieces of the sum meet in registers, and each accumulator goes straight back.
      // One term: a pass reads its columns from the one accumulator, which goes back after the last.
      float acc[TERMS == 2 ? 2 : 1][32];
      uint32_t t0 = 0, set = 0;
      auto await_sum = [&]() {
        set = (uint32_t)j % kSets;
        const uint32_t aphase = ((uint32_t)j / kSets) & 1u;
        ++j;
        ok = __all_sync(0xffffffffu, mbar_wait<true>(smem_u32(&acc_full[set]), aphase, wc, 4u));
        tc_fence_after();
        t0 = tmem_base + ((uint32_t)(quarter * 32) << 16) + set * (uint32_t)kSetColumns + (uint32_t)(side * cols);
      };
      auto give_back = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (rank != 0) mbar_arrive_cluster(map_to_cta(smem_u32(&acc_empty[set]), 0u));
          else mbar_arrive(smem_u32(&acc_empty[set]));
        }
      };
      if (TERMS == 1) {
        if (ok) await_sum();
      } else {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int i = 0; i < 32; ++i) acc[TERMS == 2 ? c : 0][i] = 0.f;
#pragma unroll 1
        for (int s = 0; s < w.pieces && ok; ++s) {
          await_sum();
          if (!ok) break;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t r[32];
            tmem_ld32_issue(t0 + (uint32_t)(c * 32), r);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[TERMS == 2 ? c : 0][i] += __uint_as_float(r[i]);
          }
          give_back();
        }
      }
      const float alpha = w.phase == 0 ? p.f.a_scale : (w.phase == 1 ? p.f.b_acc : p.f.x_acc);
      const float scale = w.phase == 1 ? p.f.b_add[w.step] : p.f.x_add[w.step];
      const float diag = w.phase == 0 ? p.f.a_diag[w.step] : p.f.b_diag[w.step];
      const int planes = w.phase == 2 ? 2 : TERMS;
      const bool mirror = w.phase < 2 && w.ti != w.tj;
      // (unrolled for two terms, whose sums sit in registers)
#pragma unroll(TERMS == 2 ? 2 : 1)
      for (int k = 0; k < (TERMS == 2 ? 2 : 4); ++k) {
        const int c0 = k * kPass;
        if (c0 < cols && ok) {
          const int col = n0 + c0;
          const uint32_t buffer = TERMS == 2 ? 0u : (w.phase == 2 ? (uint32_t)k % 3u : (uint32_t)k & 1u);
          const uint32_t at = sbuf + buffer * kBuffer;
          if (TERMS == 2) {
            if (lane == 0 && k > 0) {
              bulk_wait_read_all();
              if (addends) fetch(from, 0u, col, row0, plane0, addends);
            }
            __syncwarp();
          } else if (k > 0 && (w.phase < 2 || k == 1)) {
            if (lane == 0) {
              bulk_wait_read_all();
              if (w.phase == 2 && 3 * kPass < cols) fetch(from, 0u, n0 + 3 * kPass, row0, plane0, addends);
              if (w.phase == 1 && k < 3 && c0 + kPass < cols) fetch(from, (uint32_t)(k + 1) & 1u, col + kPass, row0, plane0, addends);
            }
            __syncwarp();
          }
          float v[kPass];
          if (TERMS == 1) {
            uint32_t r[32];
            tmem_ld32_issue(t0 + (uint32_t)c0, r);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = alpha * __uint_as_float(r[i]);
            if (c0 + kPass >= cols) give_back();
          } else {
#pragma unroll
            for (int i = 0; i < kPass; ++i) v[i] = alpha * acc[TERMS == 2 ? k : 0][i];
          }
          if (addends) {
            ok = __all_sync(0xffffffffu, mbar_wait<false>(add_bar + 8u * buffer, (add_phase >> buffer) & 1u, wc, 6u));
            add_phase ^= 1u << buffer;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              if (t < addends) {
#pragma unroll
                for (uint32_t q = 0; q < kPass / 8; ++q) {
                  uint32_t r[4];
                  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                               : "r"(at + (uint32_t)t * kPassPlane + piece_at((uint32_t)lane, q)));
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    const float2 f = unpack_half2(r[i]);
                    v[8 * q + 2 * i] = fmaf(scale, f.x, v[8 * q + 2 * i]);
                    v[8 * q + 2 * i + 1] = fmaf(scale, f.y, v[8 * q + 2 * i + 1]);
                  }
                }
              }
            }
          }
          if (w.phase < 2 && w.ti == w.tj) {
#pragma unroll
            for (int i = 0; i < kPass; ++i)
              if (col + i == row) v[i] += diag;
          }
          // the result's terms, 16 bytes of a row at a time
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (t < planes) {
#pragma unroll
              for (uint32_t q = 0; q < kPass / 8; ++q) {
                uint32_t pk[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  pk[i] = pack_half2(v[8 * q + 2 * i], v[8 * q + 2 * i + 1]);
                  const float2 f = unpack_half2(pk[i]);
                  v[8 * q + 2 * i] -= f.x;
                  v[8 * q + 2 * i + 1] -= f.y;
                }
                st_shared_v4(at + (uint32_t)t * kPassPlane + piece_at((uint32_t)lane, q), pk[0], pk[1], pk[2], pk[3]);
                if (TERMS == 1 && mirror) store_turned(sbuf + 2u * kBuffer, 8u * q, pk);
              }
            }
          }
          hand_over(to, at, col, row0, plane0);
          if (TERMS == 2 && mirror) {
            // the rows are read back, and turned in their place once the engine has them
            uint32_t pk[2][kPass / 2];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (uint32_t q = 0; q < kPass / 8; ++q)
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(pk[t][4 * q]), "=r"(pk[t][4 * q + 1]), "=r"(pk[t][4 * q + 2]), "=r"(pk[t][4 * q + 3])
                             : "r"(at + (uint32_t)t * kPassPlane + piece_at((uint32_t)lane, q))
                             : "memory");
            if (lane == 0) bulk_wait_read_all();
            __syncwarp();
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (uint32_t q = 0; q < kPass / 8; ++q) {
                const uint32_t four[4] = {pk[t][4 * q], pk[t][4 * q + 1], pk[t][4 * q + 2], pk[t][4 * q + 3]};
                store_turned(at + (uint32_t)t * kPassPlane, 8u * q, four);
              }
          }
          if (mirror) hand_over(to, TERMS == 2 ? at : sbuf + 2u * kBuffer, row0, col, plane0);
        }
      }
      // one count for the whole CTA, once all its stores have been written (a release a warp would be eight
      // fences on end)
      if (lane == 0) bulk_wait_all();
      __syncwarp();
      failed = !ok;
      epilogue_sync();
      if (ew == 0 && lane == 0) {
        unsigned* cnt = const_cast<unsigned*>(row_counter(p, w.step, w.phase, w.mat, 0));
        count_up(cnt + w.ti);
        if (mirror) count_up(cnt + w.tj);
      }
    }
    if (lane == 0) bulk_wait_all();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0 && lane == 0 && abort_flag) {
    // a wait ran out: copies still in flight get a bounded time to land before the CTA retires
    for (int s = 0; s < p.stages; ++s)
      for (uint32_t i = 0; i < 4096u && !mbar_try_wait<true>(smem_u32(&full_bar[s]), 0u); ++i) __nanosleep(256);
  }
  cluster_sync_all();
  tc_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)kTmemColumns)
                 : "memory");
}

// Blocks of 32 rows by 64 columns of X, eight consecutive columns a thread.  A tall matrix holds X's columns
// as rows: its block is turned in shared memory.
// eight values of a row that starts at `at` and ends `left` values later (WIDE: all eight, 16-byte aligned)
template <typename T, bool WIDE>
__device__ __forceinline__ void load8(const T* at, int left, float (&v)[8]) {
  if (WIDE && left >= 8) {
    if (sizeof(T) == 4) {
      const float4 a = reinterpret_cast<const float4*>(at)[0], b = reinterpret_cast<const float4*>(at)[1];
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(at);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < left ? to_f32(at[j]) : 0.f;
  }
}
template <typename T, bool WIDE>
__device__ __forceinline__ void store8(T* at, int left, const float (&v)[8]) {
  if (WIDE && left >= 8) {
    if (sizeof(T) == 4) {
      reinterpret_cast<float4*>(at)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(at)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
      *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) at[j] = narrow<T>(v[j]);
  }
}
// position of this thread's eight values: in the matrix (rows of `width` values) and in the block
struct Eight { int row, col, left; };
__device__ __forceinline__ Eight eight_of(int tall, int height, int width, int row0, int col0) {
  Eight e;
  e.row = tall ? col0 + (int)(threadIdx.x >> 2) : row0 + (int)(threadIdx.x >> 3);
  e.col = tall ? row0 + (int)(threadIdx.x & 3) * 8 : col0 + (int)(threadIdx.x & 7) * 8;
  e.left = e.row < height ? width - e.col : 0;
  return e;
}

// ---------------------------------------------------------------------------------------------
// M' = beta M + G (or U given) and partial sums of ||U||^2, one per block, in double: a fixed order,
// and no overflow whatever the gradients' scale.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ float update_of(float g, float m2, float beta, int nesterov) {
  return nesterov ? fmaf(beta, m2, g) : m2;
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(256)
orth_momentum_kernel(const __grid_constant__ OrthPtrs ptr, int64_t n, float beta, int nesterov,
                     double* __restrict__ partials) {
  __shared__ double buf[8];
  const int i = blockIdx.y;
  double s = 0.0;
  for (int64_t k = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; k < n; k += (int64_t)gridDim.x * 2048) {
    const int left = n - k < 8 ? (int)(n - k) : 8;
    float u[8];
    if (ptr.u[i]) {
      load8<T, WIDE>(static_cast<const T*>(ptr.u[i]) + k, left, u);
    } else {
      float g[8], m[8];
      load8<float, WIDE>(ptr.g[i] + k, left, g);
      load8<float, WIDE>(ptr.m[i] + k, left, m);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = fmaf(beta, m[j], g[j]);
        u[j] = update_of(g[j], m[j], beta, nesterov);
      }
      store8<float, WIDE>(ptr.mo[i] + k, left, m);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) s += (double)u[j] * (double)u[j];
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < 8; ++w) t += buf[w];
    partials[(int64_t)i * gridDim.x + blockIdx.x] = t;
  }
}

// X_0 = Sx U / ||U||_F as fp16 leading term and remainder, padded with zeros
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256)
orth_start_kernel(const __grid_constant__ OrthPtrs ptr, int m, int n, int mp, int np, int tall, float beta, int nesterov,
                  const double* __restrict__ partials, int parts, double sx, __half* __restrict__ x) {
  __shared__ float tile[64][33];
  __shared__ double buf[9];
  const int i = blockIdx.z, row0 = blockIdx.y * 32, col0 = blockIdx.x * 64;
  double t = 0.0;
  for (int k = threadIdx.x; k < parts; k += 256) t += partials[(int64_t)i * parts + k];
#pragma unroll
  for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = t;
  const Eight e = eight_of(tall, tall ? n : m, tall ? m : n, row0, col0);
  const int64_t at = (int64_t)e.row * (tall ? m : n) + e.col;
  float v[8];
  if (e.left <= 0) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
  } else if (ptr.u[i]) {
    load8<T, WIDE>(static_cast<const T*>(ptr.u[i]) + at, e.left, v);
  } else {
    float g[8], m2[8];
    load8<float, WIDE>(ptr.g[i] + at, e.left, g);
    load8<float, WIDE>(ptr.mo[i] + at, e.left, m2);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = update_of(g[j], m2[j], beta, nesterov);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0.0;
    for (int w = 0; w < 8; ++w) s += buf[w];
    buf[8] = s > 0.0 ? sx / sqrt(s) : (s == 0.0 ? 0.0 : s);      // NaN stays NaN
  }
  const int a = threadIdx.x >> 3, b = (threadIdx.x & 7) * 8;
  if (tall)
#pragma unroll
    for (int j = 0; j < 8; ++j) tile[threadIdx.x >> 2][(threadIdx.x & 3) * 8 + j] = v[j];
  __syncthreads();
  if (tall)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = tile[b + j][a];
  const double r = buf[8];
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bool in0 = row0 + a < m && col0 + b + 2 * j < n, in1 = row0 + a < m && col0 + b + 2 * j + 1 < n;
    const float x0 = in0 ? (float)((double)v[2 * j] * r) : 0.f, x1 = in1 ? (float)((double)v[2 * j + 1] * r) : 0.f;
    hi[j] = pack_half2(x0, x1);
    const float2 f = unpack_half2(hi[j]);
    lo[j] = pack_half2(x0 - f.x, x1 - f.y);
  }
  __half* to = x + (int64_t)i * 2 * mp * np + (int64_t)(row0 + a) * np + col0 + b;
  *reinterpret_cast<uint4*>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  *reinterpret_cast<uint4*>(to + (int64_t)mp * np) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}

// W' = keep W - step X, or X itself, from the two planes of the last X.  Where a wait of the products ran out there is
// no X, and the outputs, which may be the weights themselves, stay as they are.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256)
orth_apply_kernel(const __grid_constant__ OrthPtrs ptr, int m, int n, int mp, int np, int tall, const __half* __restrict__ x,
                  float out_scale, float keep, float step, const DeviceStatus* __restrict__ st) {
  __shared__ float tile[64][33];
  if (st->code != 0) return;
  const int i = blockIdx.z, row0 = blockIdx.y * 32, col0 = blockIdx.x * 64;
  const int a = threadIdx.x >> 3, b = (threadIdx.x & 7) * 8;
  const __half* from = x + (int64_t)i * 2 * mp * np + (int64_t)(row0 + a) * np + col0 + b;
  const uint4 hi = *reinterpret_cast<const uint4*>(from), lo = *reinterpret_cast<const uint4*>(from + (int64_t)mp * np);
  const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
  float v[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 p = unpack_half2(h[j]), q = unpack_half2(l[j]);
    v[2 * j] = p.x + q.x;
    v[2 * j + 1] = p.y + q.y;
  }
  if (tall) {
#pragma unroll
    for (int j = 0; j < 8; ++j) tile[b + j][a] = v[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = tile[threadIdx.x >> 2][(threadIdx.x & 3) * 8 + j];
  }
  const Eight e = eight_of(tall, tall ? n : m, tall ? m : n, row0, col0);
  if (e.left <= 0) return;
  const int64_t at = (int64_t)e.row * (tall ? m : n) + e.col;
  if (ptr.w[i]) {
    float w[8];
    load8<T, WIDE>(static_cast<const T*>(ptr.w[i]) + at, e.left, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = fmaf(-step, v[j] * out_scale, keep * w[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= out_scale;
  }
  store8<T, WIDE>(static_cast<T*>(ptr.out[i]) + at, e.left, v);
}

// ---------------------------------------------------------------------------------------------
// Small matrices (up to 128 x 256, X and A within one SM's shared memory): one CTA a matrix does everything in one
// launch -- momentum, norm, all steps, update.  A phase of the kernel above costs a trip through L2, 9 to
// 16 us whatever the tile; here X, A and B stay in shared memory and each phase is a product, a read of the
// accumulator and a rewrite in place.  X is laid out in groups of 64 columns, [128 rows][128 bytes] each under
// the 128-byte swizzle: row by row that is a K-major operand of X X^T, and column by column an MN-major
// operand of B X, so one copy serves both products.
// ---------------------------------------------------------------------------------------------
struct OrthSmall {
  OrthFactors f;
  int m, n, tall, steps, nesterov;
  float beta, keep, step;
  double sx;
  DeviceStatus* st;
  uint64_t wait_ns;
  unsigned unmet;       // self-test: the first product is not started
};
constexpr uint32_t kGroupBytes = 128 * 128;

__host__ __device__ constexpr uint32_t small_bytes(int m, int n, int terms) {
  return (uint32_t)(2 * ((n + 63) / 64) + terms * ((m + 63) / 64)) * kGroupBytes;
}
constexpr int kSmallRows = 128, kSmallColumns = 256;
// byte offset of the 16 bytes that hold columns c .. c + 7 (c a multiple of 8) of row r
__device__ __forceinline__ uint32_t small_at(int r, int c) {
  return (uint32_t)(c >> 6) * kGroupBytes + (uint32_t)r * 128u + (uint32_t)((((c & 63) >> 3) ^ (r & 7)) << 4);
}

template <typename T, int TERMS>
__global__ void __launch_bounds__(256)
orth_small_kernel(const __grid_constant__ OrthPtrs ptr, const __grid_constant__ OrthSmall p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  __shared__ double buf[9];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, i = blockIdx.x;
  const int m = p.m, n = p.n, width = p.tall ? m : n;
  const int mg = (m + 63) / 64, ng = (n + 63) / 64;
  uint8_t* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* x_hi = base;
  uint8_t* x_lo = x_hi + ng * kGroupBytes;
  uint8_t* a_hi = x_lo + ng * kGroupBytes;
  uint8_t* a_lo = a_hi + mg * kGroupBytes;                 // (two terms only)
  // accumulator columns of X X^T and A^2, then of B X
  const uint32_t columns = mg * 64 + ng * 64 <= 128 ? 128u : (mg * 64 + ng * 64 <= 256 ? 256u : 512u);
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&bar), 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(columns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // M', U and ||U||; X starts as zeros in its padding
  const T* u_in = static_cast<const T*>(ptr.u[i]);
  const float *g = ptr.g[i], *mom = ptr.m[i];
  float* mom_out = ptr.mo[i];
  double s = 0.0;
  for (int k = threadIdx.x; k < m * n; k += 256) {
    float u;
    if (u_in) {
      u = to_f32(u_in[k]);
    } else {
      const float m2 = fmaf(p.beta, mom[k], g[k]);
      mom_out[k] = m2;
      u = update_of(g[k], m2, p.beta, p.nesterov);
    }
    s += (double)u * (double)u;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) buf[warp] = s;
  for (uint32_t k = threadIdx.x; k < 2u * ng * kGroupBytes / 16; k += 256)
    reinterpret_cast<uint4*>(x_hi)[k] = make_uint4(0u, 0u, 0u, 0u);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < 8; ++w) t += buf[w];
    buf[8] = t > 0.0 ? p.sx / sqrt(t) : (t == 0.0 ? 0.0 : t);      // NaN stays NaN
  }
  __syncthreads();
  const double r = buf[8];
  const uint32_t tmem = tmem_slot;
  for (int k = threadIdx.x; k < m * n; k += 256) {
    const int a = k / width, b = k - a * width, row = p.tall ? b : a, col = p.tall ? a : b;
    const float u = u_in ? to_f32(u_in[k]) : update_of(g[k], mom_out[k], p.beta, p.nesterov);
    const float x = (float)((double)u * r);
    const __half h = __float2half_rn(x);
    const uint32_t at = small_at(row, col & ~7) + (uint32_t)(col & 7) * 2u;
    *reinterpret_cast<__half*>(x_hi + at) = h;
    *reinterpret_cast<__half*>(x_lo + at) = __float2half_rn(x - __half2float(h));
  }
  WaitCtx wc;
  wc.st = p.st;
  wc.abort_flag = &abort_flag;
  wc.limit_ns = p.wait_ns;
  const int quarter = warp & 3, side = warp >> 2, row = quarter * 32 + lane;
  const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
  const uint32_t xh = smem_u32(x_hi) >> 4, xl = smem_u32(x_lo) >> 4, ah = smem_u32(a_hi) >> 4, al = smem_u32(a_lo) >> 4;
  uint32_t phase = 0;
  bool ok = true;
  for (int step = 0; step < p.steps && ok; ++step) {
#pragma unroll 1
    for (int ph = 0; ph < 3 && ok; ++ph) {
      // the operands are written by all threads: make them visible to the tensor core
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tc_fence_before();
      __syncthreads();
      const uint32_t d = tmem + (ph == 2 ? (uint32_t)(mg * 64) : 0u);
      if (threadIdx.x == 0 && !p.unmet) {
        tc_fence_after();
        const int N = ph == 2 ? ng * 64 : mg * 64, ks = ph == 0 ? ng * 4 : (m + 15) / 16;
        const uint32_t idesc = (1u << 4) | ((ph == 2 ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((128u >> 4) << 24);
        for (int k = 0; k < ks; ++k) {
          // K-major: 16 columns are 32 bytes of a group; MN-major: 16 rows are 2048 bytes
          const uint32_t kk = (uint32_t)(k >> 2) * (kGroupBytes >> 4) + (uint32_t)(k & 3) * 2u | (1u << 16);
          const uint32_t kn = (uint32_t)k * (2048u >> 4) | ((kGroupBytes >> 4) << 16);
          const uint32_t a0 = (ph == 0 ? xh : ah) + kk, b0 = ph == 2 ? xh + kn : (ph == 0 ? xh : ah) + kk;
          umma_bf16<false>(d, a0, b0, idesc, k > 0);
          if (TERMS == 2) {
            const uint32_t a1 = (ph == 0 ? xl : al) + kk, b1 = ph == 2 ? xl + kn : (ph == 0 ? xl : al) + kk;
            umma_bf16<false>(d, a0, b1, idesc, 1u);
            umma_bf16<false>(d, a1, b0, idesc, 1u);
          }
        }
        umma_commit<false>(smem_u32(&bar));
      }
      ok = __syncthreads_and(mbar_wait<false>(smem_u32(&bar), phase, wc, 7u));
      phase ^= 1u;
      if (!ok) break;
      tc_fence_after();
      const int cols = ph == 2 ? ng * 64 : mg * 64;
      uint8_t* hi = ph == 2 ? x_hi : a_hi;
      uint8_t* lo = ph == 2 ? x_lo : a_lo;
      const int planes = ph == 2 ? 2 : TERMS;
      const float alpha = ph == 0 ? p.f.a_scale : (ph == 1 ? p.f.b_acc : p.f.x_acc);
      const float scale = ph == 1 ? p.f.b_add[step] : p.f.x_add[step];
      const float diag = ph == 0 ? p.f.a_diag[step] : (ph == 1 ? p.f.b_diag[step] : 0.f);
      for (int c = side * 32; c < cols; c += 64) {
        uint32_t q[32];
        tmem_ld32_issue(d + lanes + (uint32_t)c, q);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t at = small_at(row, c + 8 * e);
          float v[8];
#pragma unroll
          for (int t = 0; t < 8; ++t) v[t] = alpha * __uint_as_float(q[8 * e + t]);
          if (ph) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              if (t < planes) {
                const uint4 w = *reinterpret_cast<const uint4*>((t ? lo : hi) + at);
                const uint32_t four[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                  const float2 f = unpack_half2(four[z]);
                  v[2 * z] = fmaf(scale, f.x, v[2 * z]);
                  v[2 * z + 1] = fmaf(scale, f.y, v[2 * z + 1]);
                }
              }
            }
          }
#pragma unroll
          for (int t = 0; t < 8; ++t)
            if (c + 8 * e + t == row) v[t] += diag;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (t < planes) {
              uint32_t four[4];
#pragma unroll
              for (int z = 0; z < 4; ++z) {
                four[z] = pack_half2(v[2 * z], v[2 * z + 1]);
                const float2 f = unpack_half2(four[z]);
                v[2 * z] -= f.x;
                v[2 * z + 1] -= f.y;
              }
              *reinterpret_cast<uint4*>((t ? lo : hi) + at) = make_uint4(four[0], four[1], four[2], four[3]);
            }
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
  if (!ok) return;                 // no X: the outputs stay as they are
  const T* w = static_cast<const T*>(ptr.w[i]);
  T* out = static_cast<T*>(ptr.out[i]);
  for (int k = threadIdx.x; k < m * n; k += 256) {
    const int a = k / width, b = k - a * width, rr = p.tall ? b : a, cc = p.tall ? a : b;
    const uint32_t at = small_at(rr, cc & ~7) + (uint32_t)(cc & 7) * 2u;
    const float x = (__half2float(*reinterpret_cast<const __half*>(x_hi + at)) +
                     __half2float(*reinterpret_cast<const __half*>(x_lo + at))) * p.f.out_scale;
    out[k] = narrow<T>(w ? fmaf(-p.step, x, p.keep * to_f32(w[k])) : x);
  }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
struct OrthWs {
  double* partials;
  unsigned* done;
  size_t done_bytes;
  __half *x[2], *a, *b;
};

size_t orth_layout(const mw_orth* p, char* base, OrthWs* w) {
  if (p->small) return 1024;              // device status alone
  size_t off = 1024;
  auto take = [&](size_t bytes) {
    char* q = base ? base + off : nullptr;
    off += align_up(bytes, 1024);
    return q;
  };
  const size_t c = (size_t)p->d.count, mn = (size_t)p->mp * p->np, mm = (size_t)p->mp * p->mp;
  OrthWs l;
  l.done_bytes = (size_t)p->steps * 3 * c * (p->mp / kTile) * sizeof(unsigned);
  l.done = reinterpret_cast<unsigned*>(take(l.done_bytes));
  l.partials = reinterpret_cast<double*>(take(c * kNormBlocks * sizeof(double)));
  for (auto& x : l.x) x = reinterpret_cast<__half*>(take(c * 2 * mn * 2));
  l.a = reinterpret_cast<__half*>(take(c * p->terms * mm * 2));
  l.b = reinterpret_cast<__half*>(take(c * p->terms * mm * 2));
  if (w) *w = l;
  return off;
}

// [planes][rows][cols] fp16 seen as (column, row, plane)
mw_status half_map(const __half* base, int rows, int cols, int64_t planes, int bx, int by, int bz, CUtensorMapSwizzle sw,
                   CUtensorMap* out) {
  auto fn = encode_fn();
  if (!fn) return MW_ERR_CUDA;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)cols * 2, (cuuint64_t)rows * cols * 2};
  cuuint32_t box[3] = {(cuuint32_t)bx, (cuuint32_t)by, (cuuint32_t)bz};
  cuuint32_t estr[3] = {1u, 1u, 1u};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<__half*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? MW_OK : MW_ERR_CUDA;
}

// the maps of a workspace into `out`
mw_status orth_maps(mw_orth* p, const OrthWs& l, const void* ws, CUtensorMap* out) {
  std::lock_guard<std::mutex> held(p->lock);
  if (p->mapped == ws) {
    for (int i = 0; i < MAP_COUNT; ++i) out[i] = p->maps[i];
    return MW_OK;
  }
  p->mapped = nullptr;
  const int64_t c = p->d.count;
  const int t = p->terms;
  const auto S128 = CU_TENSOR_MAP_SWIZZLE_128B, S64 = CU_TENSOR_MAP_SWIZZLE_64B;
  for (int b = 0; b < 2; ++b) {
    MW_TRY(half_map(l.x[b], p->mp, p->np, 2 * c, kBK, kHalf, t, S128, &p->maps[MAP_XK + b]));
    MW_TRY(half_map(l.x[b], p->mp, p->np, 2 * c, 64, kBK, 1, S128, &p->maps[MAP_XMN + b]));
    MW_TRY(half_map(l.x[b], p->mp, p->np, 2 * c, kPass, 32, 2, S64, &p->maps[MAP_XO + b]));
    const __half* s = b ? l.b : l.a;
    MW_TRY(half_map(s, p->mp, p->mp, t * c, kBK, kHalf, t, S128, &p->maps[MAP_A + b]));
    MW_TRY(half_map(s, p->mp, p->mp, t * c, kPass, 32, t, S64, &p->maps[MAP_AO + b]));
  }
  for (int b = 0; b < 2; ++b) MW_TRY(half_map(l.x[b], p->mp, p->np, 2 * c, kBK, 64, t, S128, &p->maps[MAP_XK64 + b]));
  MW_TRY(half_map(l.a, p->mp, p->mp, t * c, kBK, 64, t, S128, &p->maps[MAP_A64]));
  p->mapped = ws;
  for (int i = 0; i < MAP_COUNT; ++i) out[i] = p->maps[i];
  return MW_OK;
}

// CTA pairs that the device holds at once (cached per device)
template <int TERMS>
mw_status orth_pairs(size_t smem, int* out) {
  static int pairs[kMaxDevices] = {};
  const int dev = current_device();
  if (pairs[dev] == 0) {
    auto kernel = orth_products_kernel<TERMS>;
    MW_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (unsigned)sm_count());
    cfg.blockDim = dim3(kOrthThreads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int c = 0;
    MW_CUDA_OK(cudaOccupancyMaxActiveClusters(&c, kernel, &cfg));
    if (c < 1) return MW_ERR_CUDA;
    pairs[dev] = c < sm_count() / 2 ? c : sm_count() / 2;
  }
  *out = pairs[dev];
  return MW_OK;
}

template <int TERMS>
mw_status orth_launch(OrthParams& prm, size_t smem, cudaStream_t s) {
  int pairs = 0;
  MW_TRY(orth_pairs<TERMS>(smem, &pairs));
  // Tiles of 256 columns, whose products run at the full rate; of 128 where all of a product's fit the device
  // at once, so that a phase, which then lasts as long as one tile, is shorter (one 1024 x 1024 in bf16: 213 us
  // with 128 columns, 257 us with 256; 16 of them, whose tiles do not fit: 487 us with 256)
  const int tri = prm.tm * (prm.tm + 1) / 2;
  const int64_t sym = (int64_t)prm.count * tri, x128 = (int64_t)prm.count * prm.tm * ceil_div(prm.np, kHalf);
  prm.bn_sym = TERMS == 2 || 2 * sym <= pairs ? kHalf : kTile;
  prm.bn_x = TERMS == 2 || x128 <= pairs ? kHalf : kTile;
  prm.sym_tiles = tri * (kTile / prm.bn_sym);
  prm.tn = ceil_div(prm.np, prm.bn_x);
  prm.per_step = prm.count * (2 * prm.sym_tiles + prm.tm * prm.tn);       // (mw_orth_create bounds the total)
  prm.total = prm.per_step * prm.steps;
  const int64_t widest = (int64_t)prm.count * (prm.tm * prm.tn > prm.sym_tiles ? prm.tm * prm.tn : prm.sym_tiles);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * (unsigned)(widest < pairs ? widest : pairs));
  cfg.blockDim = dim3(kOrthThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeCooperative;      // tiles wait for one another: all pairs are resident
  attr[1].val.cooperative = tc_cooperative();
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  ++g_launch_count;
  return cudaLaunchKernelEx(&cfg, orth_products_kernel<TERMS>, prm) == cudaSuccess ? MW_OK : MW_ERR_CUDA;
}

double pow2_floor(double v) { return exp2(floor(log2(v))); }

// Sx: rows of X have norm about one, so sqrt(n) brings their entries to about one; 64 more leaves the remainders
// of small entries in fp16's range
double orth_sx(int n) {
  const double sx = 64.0 * exp2(ceil(log2(sqrt((double)n))));
  return sx < 16384.0 ? sx : 16384.0;
}

OrthFactors orth_factors(const mw_orth* p, double sx) {
  OrthFactors f;
  // Sa: the entries of B are at most |c1| s + |c2| s^2 with s <= 2 the largest eigenvalue of A
  double sa = 1024.0;
  const double most = 2.0 * fabs(p->c[1]) + 4.0 * fabs(p->c[2]);
  if (most * sa > 32768.0) sa = pow2_floor(32768.0 / most);
  f.a_scale = (float)(sa / (sx * sx));
  f.b_acc = (float)(p->c[2] / sa);
  f.x_acc = (float)(1.0 / sa);
  f.out_scale = (float)(1.0 / sx);
  const bool shifts = p->d.coef[0] == 0.0 && p->d.coef[1] == 0.0 && p->d.coef[2] == 0.0;
  for (int k = 0; k < p->steps; ++k) {
    // (the shifts are identities; these values lie in the middle of the spectra that the default
    // polynomial has produced by then: of 5 sets tried on 20 matrices, the smallest largest error)
    double al = 0.0, be = 0.0;
    if (shifts && p->steps >= 5 && k == p->steps - 1) { al = 0.7; be = 2.0; }
    else if (shifts && p->steps >= 5 && k == p->steps - 2) { al = 0.3; be = 1.0; }
    f.a_diag[k] = (float)(-al * sa);
    f.b_add[k] = (float)(p->c[1] + 2.0 * p->c[2] * al);
    f.b_diag[k] = (float)(sa * (p->c[1] * al + p->c[2] * al * al + be));
    f.x_add[k] = (float)(p->c[0] - be);
  }
  return f;
}

template <typename T>
mw_status orth_run(mw_orth* p, const void* const* params, const void* const* grads, const void* const* momentum,
                   void* const* out, void* const* momentum_out, const void* const* project_in, double lr, double beta,
                   double wd, double scale, char* ws, cudaStream_t s) {
  const int m = p->m, n = p->n, count = p->d.count;
  if (p->small) {
    MW_CUDA_OK(cudaMemsetAsync(ws, 0, 256, s));       // status
    auto kernel = p->terms == 1 ? orth_small_kernel<T, 1> : orth_small_kernel<T, 2>;
    const size_t smem = 1024 + small_bytes(m, n, p->terms);
    MW_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    static thread_local OrthSmall q;
    q.sx = orth_sx(n);
    q.f = orth_factors(p, q.sx);
    q.m = m; q.n = n; q.tall = p->tall; q.steps = p->steps; q.nesterov = p->d.nesterov;
    q.beta = (float)beta; q.keep = (float)(1.0 - lr * wd); q.step = (float)(lr * scale);
    q.st = reinterpret_cast<DeviceStatus*>(ws);
    q.wait_ns = p->unmet_ms ? p->unmet_ms * 1000000ull : kOrthWaitNs;
    q.unmet = p->unmet_ms != 0;
    for (int first = 0; first < count; first += kPtrGroup) {
      const int c = count - first < kPtrGroup ? count - first : kPtrGroup;
      static thread_local OrthPtrs ptr;
      for (int i = 0; i < c; ++i) {
        const int k = first + i;
        ptr.u[i] = project_in ? project_in[k] : nullptr;
        ptr.g[i] = grads ? static_cast<const float*>(grads[k]) : nullptr;
        ptr.m[i] = momentum ? static_cast<const float*>(momentum[k]) : nullptr;
        ptr.mo[i] = momentum_out ? static_cast<float*>(momentum_out[k]) : nullptr;
        ptr.w[i] = params ? params[k] : nullptr;
        ptr.out[i] = out[k];
      }
      kernel<<<(unsigned)c, 256, smem, s>>>(ptr, q);
      MW_TRY(launch_ok());
    }
    return MW_OK;
  }
  OrthWs l;
  orth_layout(p, ws, &l);
  // status and counters (ahead of the maps: their encoder wants a context, which a thread's first runtime call makes)
  MW_CUDA_OK(cudaMemsetAsync(ws, 0, 1024 + l.done_bytes, s));
  static thread_local OrthParams q;
  MW_TRY(orth_maps(p, l, ws, q.map));
  const int64_t mn = (int64_t)m * n, rowlen = p->tall ? m : n;
  const double sx = orth_sx(n);
  // blocks of the momentum pass: about eight an SM over all matrices
  const int64_t want = (mn + 2047) / 2048, share = ceil_div(8 * 148, count < kPtrGroup ? count : kPtrGroup);
  int parts = (int)(want < kNormBlocks ? want : kNormBlocks);
  if (parts > share) parts = (int)share;
  for (int first = 0; first < count; first += kPtrGroup) {
    const int c = count - first < kPtrGroup ? count - first : kPtrGroup;
    static thread_local OrthPtrs ptr;
    // 16-byte accesses where every row of every matrix starts on such a boundary
    bool wide = (rowlen * (int64_t)sizeof(T)) % 16 == 0;
    for (int i = 0; i < c; ++i) {
      const int k = first + i;
      ptr.u[i] = project_in ? project_in[k] : nullptr;
      ptr.g[i] = grads ? static_cast<const float*>(grads[k]) : nullptr;
      ptr.m[i] = momentum ? static_cast<const float*>(momentum[k]) : nullptr;
      ptr.mo[i] = momentum_out ? static_cast<float*>(momentum_out[k]) : nullptr;
      wide = wide && (((uintptr_t)ptr.u[i] | (uintptr_t)ptr.g[i] | (uintptr_t)ptr.m[i] | (uintptr_t)ptr.mo[i]) & 15) == 0;
    }
    double* part = l.partials + (size_t)first * parts;
    auto k1 = wide ? orth_momentum_kernel<T, true> : orth_momentum_kernel<T, false>;
    auto k2 = wide ? orth_start_kernel<T, true> : orth_start_kernel<T, false>;
    k1<<<dim3((unsigned)parts, (unsigned)c), 256, 0, s>>>(ptr, mn, (float)beta, p->d.nesterov, part);
    k2<<<dim3((unsigned)(p->np / 64), (unsigned)(p->mp / 32), (unsigned)c), 256, 0, s>>>(
        ptr, m, n, p->mp, p->np, p->tall, (float)beta, p->d.nesterov, part, parts, sx,
        l.x[0] + (size_t)first * 2 * p->mp * p->np);
    MW_TRY(launch_ok(2));
  }
  q.count = count;
  q.tm = p->mp / kTile;
  q.steps = p->steps;
  q.kb_m = ceil_div(m, kBK);
  q.kb_n = ceil_div(n, kBK);
  q.piece_blocks = p->terms == 2 ? kPieceBlocks : 0;
  q.mp = p->mp; q.np = p->np;
  q.f = orth_factors(p, sx);
  q.done = l.done;
  q.st = reinterpret_cast<DeviceStatus*>(ws);
  q.wait_ns = p->unmet_ms ? p->unmet_ms * 1000000ull : kOrthWaitNs;
  q.unmet = p->unmet_ms != 0;
  q.stage_bytes = (uint32_t)p->terms * (kPlaneBytes + (uint32_t)set_columns(p->terms) / 2u * kBK * 2u);
  q.stages = 4;
  const size_t smem = 1024 + (size_t)q.stages * q.stage_bytes + kOrthEpi * staging_buffers(p->terms) * kBuffer;
  MW_TRY(p->terms == 1 ? orth_launch<1>(q, smem, s) : orth_launch<2>(q, smem, s));
  for (int first = 0; first < count; first += kPtrGroup) {
    const int c = count - first < kPtrGroup ? count - first : kPtrGroup;
    static thread_local OrthPtrs ptr;
    bool wide = (rowlen * (int64_t)sizeof(T)) % 16 == 0;
    for (int i = 0; i < c; ++i) {
      ptr.w[i] = params ? params[first + i] : nullptr;
      ptr.out[i] = out[first + i];
      wide = wide && (((uintptr_t)ptr.w[i] | (uintptr_t)ptr.out[i]) & 15) == 0;
    }
    auto k3 = wide ? orth_apply_kernel<T, true> : orth_apply_kernel<T, false>;
    k3<<<dim3((unsigned)ceil_div(n, 64), (unsigned)ceil_div(m, 32), (unsigned)c), 256, 0, s>>>(
        ptr, m, n, p->mp, p->np, p->tall, l.x[p->steps & 1] + (size_t)first * 2 * p->mp * p->np, q.f.out_scale,
        (float)(1.0 - lr * wd), (float)(lr * scale), q.st);
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
  if (d.rows > kMaxSide || d.cols > kMaxSide || d.count > 65535) return MW_ERR_UNSUPPORTED;
  if (d.prec == MW_F64) return MW_ERR_UNSUPPORTED;
  if (d.prec != MW_F32 && d.prec != MW_BF16_F32ACC) return MW_ERR_INVALID_ARG;
  for (double c : d.coef)
    if (!isfinite(c)) return MW_ERR_INVALID_ARG;
  {
    // tiles of all steps are counted in 32 bits
    const int64_t m = d.rows < d.cols ? d.rows : d.cols, n = d.rows < d.cols ? d.cols : d.rows;
    const int64_t tm = (m + kTile - 1) / kTile, tn = (n + kTile - 1) / kTile;
    if (d.count * (tm * (tm + 1) + tm * tn) * (d.steps ? d.steps : 5) > (1 << 30)) return MW_ERR_UNSUPPORTED;
  }
  mw_orth* p = new (std::nothrow) mw_orth();
  if (!p) return MW_ERR_CUDA;
  p->d = d;
  p->tall = d.rows > d.cols;
  p->m = p->tall ? d.cols : d.rows;
  p->n = p->tall ? d.rows : d.cols;
  p->steps = d.steps ? d.steps : 5;
  // bf16 weights: one term where its error stays below the rounding to bf16 and a second one costs.  Rows share the
  // error between them: 2.3e-3 of X at the most for 26 rows, 9e-3 for two (2e-6 with two terms, whatever the size); and in
  // one CTA a matrix the second term is cheap (64 of 64 x 64 projected in 37 us, 33 with one; 16 of 31 x 1024, which
  // is not, 197 and 139).
  const bool few = p->m < 32, in_one = p->m <= kSmallRows && p->n <= kSmallColumns;
  p->terms = d.terms ? d.terms : (d.prec == MW_F32 || few || in_one ? 2 : 1);
  static_assert(small_bytes(kSmallRows, kSmallColumns, 2) <= 200u * 1024u, "X and A in one SM's shared memory");
  p->small = in_one;
  p->mp = (int)align_up((size_t)p->m, kTile);
  p->np = (int)align_up((size_t)p->n, kHalf);
  const bool given = d.coef[0] != 0.0 || d.coef[1] != 0.0 || d.coef[2] != 0.0;
  const double quintic[3] = {3.4445, -4.7750, 2.0315};
  for (int i = 0; i < 3; ++i) p->c[i] = given ? d.coef[i] : quintic[i];
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

extern "C" mw_status mw_orth_selftest_unmet_wait(mw_orth* plan, uint32_t limit_ms) {
  if (!plan || limit_ms > 1000) return MW_ERR_INVALID_ARG;
  plan->unmet_ms = limit_ms;
  return MW_OK;
}

extern "C" mw_status mw_orth_status(const mw_orth* plan, const void* workspace, void* stream) {
  using namespace mw;
  if (!plan || !workspace) return MW_ERR_INVALID_ARG;
  DeviceStatus host;
  MW_CUDA_OK(cudaMemcpyAsync(&host, workspace, sizeof(host), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
  MW_CUDA_OK(cudaStreamSynchronize((cudaStream_t)stream));
  return (mw_status)host.code;
}
