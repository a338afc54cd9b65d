// Softmax cross entropy over a vocabulary, and its gradient (mw_token_loss_*):
//   z = s h W^T,  loss_i = log sum_j exp z_ij - z_{i,t_i},  dz_ij = g_i (p_ij - [j = t_i]),  dh = s dz W,  dW = s dz^T h
//
// Rows that have a target are put together first, so that the others cost nothing and nothing of them is read. The
// products run on the tensor cores (CTA pairs, 256 x 256 tiles, one persistent launch a product) and bound the time: 2
// N V D flops for the loss, three times that with both gradients. Measured (1374 TFLOP/s is what a library product of
// 8192^3 bf16 reaches under the power cap, 1658 in a burst): loss of 8192 rows of 32768x2048 bf16 0.80 ms, 1.37
// PFLOP/s, where the library's product of the logits alone takes 0.83 ms; with both gradients 2.8 ms, 1.15 PFLOP/s;
// 3700 rows of 131072x4096 10.4 ms, 1.13 PFLOP/s; 2048 rows of 32768x1024 fp32 1.13 ms, 1.09 PFLOP/s of the three
// products a product. The tensor pipe is busy for 86 to 93% of the cycles.
//
// Loss alone: a tile's epilogue leaves, for each row and 128 columns, a power of two k and the sum of 2^(z' - k) (z' =
// z log2 e) of all logits but the target's; a last kernel joins them. Nothing else of the logits is written. Up to 256
// rows of bf16 are read as they lie, without being put together: two launches, 34 us for 16 rows of 32768x2048 (the
// vocabulary's way through memory is 20 us). Up to 8 rows of fp32 stay off the tensor cores ("very few rows" below).
//
// Gradient: the logits are not computed twice. A piece of rows at a time, the epilogue also writes 2^(z' - k) in half
// precision (float for float operands); once the row's sum is known those become dz in their place, by a factor per 128
// columns, and two products take them in. That costs 4 bytes of traffic an element (0.175 ms of the 2.8 above), less
// than the 2 D flops of computing it again (0.75 ms) from D of about 400 up.
//
// Numbers. bf16 operands are taken as half-precision numbers times a power of two (one a row of h, one for W): their 8
// bits fit, and dz keeps 11 bits where bf16 would leave 8 (dh and dW of bf16 are as far from 64 bits as the last
// rounding leaves any result: 1.7e-3). Float operands are split in two such terms (22 bits), three products of four.
// Sums are float; the tensor core cuts its accumulator off at every step, so a sum goes to registers, rounded to
// nearest, a piece of K at a time. The loss is log1p of the other terms' sum over the target's, so that rows sure of
// their target keep its digits. Rows do not share their powers of two: a large row of h, or a heavy or infinite weight
// among the rows', takes no digits from the others' losses and dh (where dW's sums run over such rows, h goes into them
// as an operand of its own). An epilogue's lane has a row and takes its power out: 3% of a call whose tiles are one K
// block long (16384 rows of 5000x64, 285 and 294 us), nothing of 2048 columns.
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "mw_launch.cuh"
#include "mw_tc_ptx.cuh"

namespace mw {
namespace {

constexpr int kIndexRows = 1024;          // rows of one block that looks for targets
// The power of two of a block of logits whose largest is m (in powers of two): what its exponentials are relative to.
// Of nothing but -inf it is small, so that the empty block sets no row's scale, and differences to any power are
// finite; beside an infinity or a NaN alone the values stay as they are.
constexpr float kNoPower = -3e38f;
__device__ __forceinline__ float power_of(float m) { return m == -INFINITY ? kNoPower : (m < INFINITY ? ceilf(m) : 0.f); }
constexpr int64_t kPieceBytes = (int64_t)1 << 30;
constexpr int64_t kHeldBytes = (int64_t)40 << 20;          // of rows that stay in L2 (126 MB) while the vocabulary passes

// ---- tiles ------------------------------------------------------------------------------------
constexpr int kTile = 256;                // rows and columns of a pair's tile
constexpr int kHalf = 128;                // ... of one CTA's share of either operand
constexpr int kBK = 64;
constexpr int kSumColumns = 128;          // logits that share a power of two and a sum
constexpr int kLossThreads = 384;         // copies of A, products, copies of B, an idle warp; eight epilogue warps
constexpr int kFirstEpi = 4, kEpi = 8;
// registers a thread: the launch gives 384 x 168 = 64512, handed over as 128 x 104 + 256 x 200 = 64512
constexpr int kFewRegisters = 104, kManyRegisters = 200;
constexpr uint32_t kPlaneBytes = kHalf * kBK * 2;       // one term of one operand of one stage and CTA
constexpr uint32_t kBufferBytes = 32 * 128;             // 32 rows of 128 bytes of an epilogue warp
constexpr uint64_t kLossWaitNs = 2000000000ull;
// self-test of this thread's calls: the product of which a CTA's rows are not copied, and how long they are waited for
thread_local uint32_t unmet_ms = 0;
thread_local int unmet_product = 0;
enum { P_SUMS = 0, P_EXP, P_DH, P_DW };
// How operands are held. M_ONE: one term (bf16 as it is in the loss alone, half precision times a power of two in the
// gradient). M_TWO: fp32 as two half-precision terms. M_FEW: the gradient of few rows of bf16, whose time is the
// vocabulary's way through memory: W is read in place, by both products that want it, exponentials are float and dz two
// bf16 terms against one of W and h. That saves writing W once more and reading that, and costs wider exponentials and
// a product more of dz each. So it is for 16-byte aligned W of 24 MB and more, with eight columns to a row at least,
// and up to 128 rows (half precision beside it: 1 row of 66235x2624 364 and 245 us, 128 rows 401 and 309; 128 rows of
// 16384x1024 77 and 73; but 16 rows of 33550x320 61 and 64 us, 128 rows 72 and 84, of 4096x512 44 and 49). M_THIN: very
// few rows, without the tensor cores (below).
enum { M_ONE = 1, M_TWO, M_FEW, M_THIN };
__host__ __device__ constexpr bool of_logits(int kind) { return kind == P_SUMS || kind == P_EXP; }
__host__ __device__ constexpr int terms_a(int mode, int kind) { return mode == M_TWO || (mode == M_FEW && kind >= P_DH) ? 2 : 1; }
__host__ __device__ constexpr int terms_b(int mode) { return mode == M_TWO ? 2 : 1; }
__host__ __device__ constexpr int products_of(int mode) { return mode == M_TWO ? 3 : (mode == M_FEW ? 2 : 1); }      // of dz
constexpr int kFewRows = 128;
constexpr int kThinRows = 8, kThinColumns = 64;
constexpr int64_t kFewNumbers = 12 << 20;
// Up to 128 rows are one CTA's: the other of a pair would multiply nothing, and the products of 256 rows take as long
// as the vocabulary's way through memory (loss of 16 rows of 32768x2048 bf16 36.5 us by pairs, 33.7 by CTAs, fp32 174
// and 155; gradients of 128 rows fp32 358 and 340; of 128 rows of 4096x512 fp32, whose 16 tiles leave most CTAs idle,
// 60 and 69).
__host__ __device__ constexpr uint32_t plane_b(bool pair) { return pair ? kPlaneBytes : 2 * kPlaneBytes; }     // a term of B in a CTA
// Shared memory: the stages' shares of A, theirs of B, the epilogue's buffers (of which the sums alone need none). A of
// few rows is short: its instructions read on into what follows, and nobody reads what comes of that.
constexpr int kStagesMax = 12;
constexpr size_t kSmemMost = 225 * 1024;
constexpr int stages_for(int buffers, uint32_t stage) {
  const size_t room = kSmemMost - 1024 - (size_t)kEpi * buffers * kBufferBytes;
  const int n = (int)(room / stage);
  return n < kStagesMax ? n : kStagesMax;
}
// Buffers of an epilogue warp: one, which leaves the most stages, unless a tile has so few K blocks that its way out is
// what takes the time (dW of 66235x2048 bf16: 200 rows 97 us with one, 95 with two and four; 500 rows 112, 124, 144;
// the exponentials of 2048 rows of 32768x768 91, 86, 96 and of 32768x1024 99, 103, 121; of fp32 x1024 282, 277, 444).
constexpr int buffers_for(int mode, int kind, int blocks_k) {
  if (kind == P_SUMS) return 0;
  return (kind == P_EXP && blocks_k <= (mode == M_TWO ? 24 : 12)) || (kind == P_DW && blocks_k <= 4) ? 2 : 1;
}

// K blocks that one accumulator takes. Each instruction cuts the sum off at its last place, always towards zero: the
// losses of 8192x32768x2048 bf16 are 1.6e-6 from 64 bits with 128 instructions an accumulator, 7.8e-7 with 64 and
// 3.8e-7 with 32, at 811, 810 and 837 us; two terms with 96 instructions leave 1.8e-6 in dW of 2048x32768x1024, with 48
// 8.7e-7 (1.10 and 1.12 ms). Few rows, whose losses no others average out, take half as many, and a quarter where a CTA
// has them all and it costs nothing: 16 rows of 32768x2048 1.6e-7 (3.4e-7 with half, 7.5e-7 with all) in 33.8 us, 200
// rows 3.7e-7 (1.8e-7 in 49 us of 43). dz of bf16 operands has 11 bits: its sums have 512 instructions, 2^-15 at the
// worst, and are read out seldom.
constexpr int piece_blocks(int mode, int kind, int rows) {
  const bool few = rows <= kTile;
  return mode == M_TWO ? (few ? 2 : 4) : (of_logits(kind) ? (rows <= kHalf ? 4 : (few ? 8 : 16)) : 128 / products_of(mode));
}

// what the kernels of one call share, behind the status block
struct LossInfo {
  DeviceStatus st;
  unsigned pad[59];
  int live;                 // rows that are not left out
  unsigned g_max, g_far;    // bits of the largest finite |g|, and how far those of the smallest lie below 2^31
  unsigned w_max;           // bits of the largest finite |W|
  unsigned reach;           // 1024 + the largest power of two of |g| |h|, a row's largest (0: zeros alone)
  unsigned uneven;          // some row of h is of an unusual size
  unsigned done;            // blocks whose losses are in
  unsigned pad2[57];
};

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((unsigned)(127 + e) << 23); }      // of -126..127
// v 2^e, whose factor may lie beyond a float's range
__device__ __forceinline__ float scaled_by(float v, int e) {
  e = e < -250 ? -250 : (e > 250 ? 250 : e);
  return v * power_of_two(e / 2) * power_of_two(e - e / 2);
}
// the power of two that brings numbers of at most this size to 2^13 .. 2^14 (the smallest, 2^-113 and less, below that)
__device__ __forceinline__ int range_exponent(unsigned max_bits) {
  const int e = (int)(max_bits >> 23) - 127;         // 2^e <= max < 2^(e + 1)
  if (max_bits == 0 || e > 127) return 0;
  return 13 - e > 126 ? 126 : 13 - e;
}
// ... of a row of h, or of W whole, whose numbers have the usual size, which is written while it is looked at; where the
// largest lies elsewhere it is written again. What is lost lies below 2^-25 of what is written, so the least that is left
// as it is sets the digits of small numbers: 2^-29 of the largest of its row for h, whose rows are written again at once
// (two terms: largest numbers of 2^-4 to 2^7, bf16 2^-2 to 2^9); 2^-23 of the largest for W, which takes a pass more (2^-10
// and 2^-8 on).
__host__ __device__ constexpr int usual_exponent(int terms) { return terms == 1 ? 6 : 8; }
constexpr int kLeastOfRow = 4, kLeastOfWeight = -2;
__device__ __forceinline__ bool unusual(unsigned most, int terms, int least) {
  const int e = (int)(most >> 23) - 127 + usual_exponent(terms);
  return most != 0 && (e > 14 || e < least);
}
__device__ __forceinline__ int operand_exponent(unsigned most, int terms, int least) {
  return unusual(most, terms, least) ? range_exponent(most) : usual_exponent(terms);
}
// ... of a row's dz, by its weight (any finite one above 2^-113 to 2^13 .. 2^14). dz of few rows, bf16 numbers with their
// range, has one power by the largest weight, and of very few rows, floats, none.
__device__ __forceinline__ int weight_exponent(unsigned bits) {
  const int e = (int)(bits >> 23) - 127;
  return e > 127 ? 0 : (13 - e > 126 ? 126 : 13 - e);
}
__device__ __forceinline__ int weight_exponent(float g) { return weight_exponent(__float_as_uint(fabsf(g))); }
// Rows of h and of dz have powers of two of their own: the logits' epilogue and the last kernel of dh, whose lanes have
// a row, take them out. dW's sums run over the rows. Where these are of one size, dz and h have one power each in
// truth; else dW takes h from an operand of its own, in which each row lies as far down as its dz was taken up, under
// one power for all: the rows whose |g| |h| is largest are brought to 2^13 .. 2^14, and what others lose there is small
// beside those.
__device__ __forceinline__ bool of_one_size(const LossInfo* info) {
  return info->uneven == 0 && weight_exponent(info->g_max) == weight_exponent(0x7fffffffu - info->g_far);
}
__device__ __forceinline__ int common_exponent(const LossInfo* info) { return info->reach ? 13 + 1024 - (int)info->reach : 0; }
// what dW's sums are too large by (NaN where a wait ran out before)
__device__ __forceinline__ float dweight_factor(const LossInfo* info, double scale, bool scaled, int terms) {
  if (info->st.code != 0) return __int_as_float(0x7fffffff);
  const int same = weight_exponent(info->g_max);
  const int e = !scaled ? same : (of_one_size(info) ? usual_exponent(terms) + same : common_exponent(info));
  return fminf(fmaxf((float)ldexp(scale, -e), -3e38f), 3e38f);
}

struct LossArgs {
  int64_t rows;
  int vocab, dim;
  int64_t ld_h, ld_w, ld_dh, ld_dw;
  float scale;
  int scaled;               // operands were multiplied by powers of two
};

struct alignas(64) ProductArgs {
  CUtensorMap a, b, out, acc;
  CUtensorMap b_common;     // P_DW: h where its rows are not of one size
  const LossInfo* info;
  DeviceStatus* st;
  float* total;             // NaN where a wait ran out
  uint64_t wait_ns;
  int unmet;                // self-test: A of the first CTA is not copied
  int first, piece;         // rows of this piece begin at `first` of the live ones
  int vocab, dim;
  int tiles_m, tiles_n;     // of the whole piece (P_DW: of the vocabulary and the columns)
  int blocks_k;
  int workers;              // CTA pairs that the device holds, or CTAs where each has tiles of its own
  int share_room;           // blocks of 256 x 256 sums
  int sum_blocks;           // P_SUMS, P_EXP: blocks of 128 logits a row
  uint32_t idesc;
  int stages, buffers;
  int most_blocks;          // K blocks of one accumulator
  int shares;               // P_DW: of K, where the tiles are few (their sums then lie in blocks, as dh's)
  int group_rows;           // P_SUMS, P_EXP: tiles of rows that go through the vocabulary together, at the most
  int tile_n;               // columns of a tile: 256, fewer for few rows of the loss alone
  int direct;               // few rows of the loss alone: h as it is, rows that are left out among the others
  LossInfo* clear;          // ... and what the other kernels share is cleared here
  const void* targets;
  int index_bytes;
  uint32_t a_stage, a_term; // bytes of A in a stage of a CTA, and from a term to the next
  int a_rows;               // rows of A that are copied into a CTA
  float scale;
  int scaled;
  float2* sums;             // [row][sum_blocks]: power, sum
  float* target_z;
  const int* target;
  const int* row_exponent;  // of h as an operand, by row; null: 0
  // P_DW: the gradient itself where the copy engine cannot write it, and the sums over pieces
  void* dw;
  int64_t ld_dw;
  int dw_bf16, dw_engine;
  float* partial;
  int64_t ld_partial;
};

// How dh's tiles are laid over the pairs (CTAs, of few rows): waves of whole tiles, then the rest of them with K in
// shares, so that the last wave is as short as the others leave it (4096 rows and 2048 columns are 128 tiles on 74
// pairs: 1.75 waves with the last 54 in four, 2 without). The shares' sums, beyond the first, lie in blocks of their
// own and are added in order.
struct DhPlan { int whole, rest, shares; };
constexpr int share_blocks(int pairs) { return 4 * pairs; }      // most of them
// (a warp calls it, a lane a number of shares)
__device__ __forceinline__ DhPlan dh_plan(int live, int tiles_n, int blocks_k, int workers, int room, int products) {
  const int tiles = (live + kTile - 1) / kTile * tiles_n;
  DhPlan d;
  d.whole = tiles / workers * workers;
  d.rest = tiles - d.whole;
  // cycles: a K block's products, what a tile costs beyond them, a sum's way through memory at 4.6 KB a cycle
  const int s = (int)(threadIdx.x & 31) + 1, per = (blocks_k + s - 1) / s;
  const bool can = s == 1 || (per >= 8 && d.rest * s <= room);
  const unsigned cost = (unsigned)((d.rest * s + workers - 1) / workers) * (unsigned)(per * products * 512 + 3000) + (unsigned)(d.rest * s) * 114u;
  const unsigned least = __reduce_min_sync(0xffffffffu, can ? cost : 0xffffffffu);
  d.shares = __ffs(__ballot_sync(0xffffffffu, can && cost == least));
  return d;
}

struct Unit { int m0, n0, kb0, kb1, share; };        // share: its block, -1 for the first

template <int KIND>
__device__ __forceinline__ int live_rows(const ProductArgs& p) {
  if (KIND == P_SUMS && p.direct) return p.piece;
  const int n = p.info->live - p.first;
  return n < 0 ? 0 : (n < p.piece ? n : p.piece);
}
template <int KIND>
__device__ __forceinline__ int unit_count(const ProductArgs& p, int live, const DhPlan& plan) {
  if (KIND == P_DW) return live > 0 || p.first == 0 ? p.tiles_m * p.tiles_n * p.shares : 0;
  if (KIND == P_DH) return plan.whole + plan.rest * plan.shares;
  return (live + kTile - 1) / kTile * p.tiles_n;
}
// Tiles that run at the same time share operands in L2. Logits: as many tiles of rows as L2 holds go through the
// vocabulary together, which is read once for them (8192x32768x2048 bf16: 33 MB of rows at once 771 us, 8 tiles of rows
// 807 us). dh: tiles of the same rows of dz, or of the same share of K. dW: a tile of the vocabulary with all its
// columns.
template <int KIND>
__device__ __forceinline__ Unit unit_at(const ProductArgs& p, int u, int live, const DhPlan& plan) {
  Unit w;
  w.share = -1;
  if (KIND == P_SUMS || KIND == P_EXP) {
    const int tm = (live + kTile - 1) / kTile, groups = (tm + p.group_rows - 1) / p.group_rows, most = (tm + groups - 1) / groups;
    const int per = most * p.tiles_n, group = u / per, r = u - group * per;
    const int left = tm - group * most, rows = left < most ? left : most;
    w.m0 = (group * most + r % rows) * kTile;
    w.n0 = r / rows * (KIND == P_SUMS ? p.tile_n : kTile);
    w.kb0 = 0;
    w.kb1 = p.blocks_k;
  } else if (KIND == P_DH) {
    int tile = u, share = 0, per = p.blocks_k;
    if (u >= plan.whole) {
      share = (u - plan.whole) / plan.rest;
      tile = u - share * plan.rest;
      per = (p.blocks_k + plan.shares - 1) / plan.shares;
      if (share) w.share = (tile - plan.whole) * (plan.shares - 1) + share - 1;
    }
    w.m0 = tile / p.tiles_n * kTile;
    w.n0 = tile % p.tiles_n * kTile;
    w.kb0 = share * per;
    w.kb1 = w.kb0 + per < p.blocks_k ? w.kb0 + per : p.blocks_k;
  } else {
    const int tiles = p.tiles_m * p.tiles_n, share = u / tiles, tile = u - share * tiles;
    const int blocks = (live + kBK - 1) / kBK, per = (blocks + p.shares - 1) / p.shares;
    if (p.shares > 1) w.share = tile * p.shares + share;
    w.m0 = tile / p.tiles_n * kTile;
    w.n0 = tile % p.tiles_n * kTile;
    w.kb0 = share * per;
    w.kb1 = w.kb0 + per < blocks ? w.kb0 + per : blocks;
  }
  return w;
}

// K blocks of each of a tile's pieces: as even as they come, since a short one leaves the products waiting for the
// epilogue
__device__ __forceinline__ int piece_of(const ProductArgs& p, const Unit& w) {
  const int n = w.kb1 - w.kb0, pieces = (n + p.most_blocks - 1) / p.most_blocks;
  return pieces > 1 ? (n + pieces - 1) / pieces : p.most_blocks;
}

// byte offset of 16-byte piece c of row r in a block of 128-byte rows under the 128-byte swizzle
__device__ __forceinline__ uint32_t piece_at(uint32_t r, uint32_t c) { return r * 128u + ((c ^ (r & 7u)) << 4); }
__device__ __forceinline__ void bulk_store_2d(const CUtensorMap* tm, uint32_t src, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(tm)),
               "r"(src), "r"(c0), "r"(c1)
               : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void tmem_ld32_floats(uint32_t taddr, float* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
        "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]), "=f"(r[19]),
        "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]),
        "=f"(r[30]), "=f"(r[31])
      : "r"(taddr)
      : "memory");
}
// whether a phase is complete, without waiting for it
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// one lane of a warp whose lanes are all here: what it does may use the registers that the warp has in common
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t half2_bits(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t bf162_bits(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// A buffer's 32 rows of 128 bytes to rows that do not lie on the copy engine's boundaries, E elements a lane and row.
// (The loop is the time of a tile whose K is short: eight rows are read before the first is written, and addresses are
// additions.)
template <typename V, int E>
__device__ __forceinline__ void store_rows(uint32_t at, V* to, int64_t ld, int rows, int cols, int lane) {
  constexpr uint32_t kPer = 16 / sizeof(V);          // elements of a 16-byte piece
  bool on[E];
#pragma unroll
  for (int x = 0; x < E; ++x) on[x] = lane + 32 * x < cols;
  to += lane;
#pragma unroll 1
  for (int r0 = 0; r0 < 32 && r0 < rows; r0 += 8) {
    V v[8][E];
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int x = 0; x < E; ++x) {
        const uint32_t e = (uint32_t)(lane + 32 * x), from = at + (uint32_t)r0 * 128u + piece_at((uint32_t)r, e / kPer) + e % kPer * (uint32_t)sizeof(V);
        if constexpr (sizeof(V) == 2) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v[r][x]) : "r"(from));
        else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v[r][x]) : "r"(from));
      }
#pragma unroll
    for (int r = 0; r < 8; ++r, to += ld) {
      if (r0 + r < rows) {
#pragma unroll
        for (int x = 0; x < E; ++x)
          if (on[x]) to[32 * x] = v[r][x];
      }
    }
  }
}

template <int MODE, int KIND, bool PAIR>
__global__ void __launch_bounds__(kLossThreads, 1)
loss_products_kernel(const __grid_constant__ ProductArgs p) {
  extern __shared__ uint8_t smem_raw[];
  constexpr int kTermsA = terms_a(MODE, KIND), kTermsB = terms_b(MODE);
  constexpr bool kFloats = MODE != M_ONE;          // exponentials are float
  // two blocks a fence (not where that spills a tile's floats)
  constexpr bool kPairs = (MODE == M_ONE && KIND == P_EXP) || (MODE != M_TWO && KIND == P_DW);
  constexpr uint32_t b_stage = kTermsB * plane_b(PAIR);
  constexpr int kShareB = PAIR ? kHalf : kTile;          // of a tile's columns
  __shared__ __align__(8) uint64_t full_bar[kStagesMax];
  __shared__ __align__(8) uint64_t empty_bar[kStagesMax];
  __shared__ __align__(8) uint64_t acc_full[2];
  __shared__ __align__(8) uint64_t acc_empty[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cluster_cta_rank() : 0u;
  const int stages = p.stages;
  const uint32_t a_stage = p.a_stage;
  const uint32_t a_tiles = (smem_u32(smem_raw) + 1023u) & ~1023u, b_tiles = a_tiles + (uint32_t)stages * a_stage;
  const int pairs = (int)(PAIR ? gridDim.x >> 1 : gridDim.x), pair = (int)(PAIR ? blockIdx.x >> 1 : blockIdx.x);

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(smem_u32(&full_bar[s]), 1);
      mbar_init(smem_u32(&empty_bar[s]), 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&acc_full[s]), 1);
      mbar_init(smem_u32(&acc_empty[s]), PAIR ? kEpi * 2 : kEpi);
    }
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = tmem_slot;
  WaitCtx wc;
  wc.st = p.st;
  wc.abort_flag = &abort_flag;
  wc.limit_ns = p.wait_ns;
  after_previous();
  if (KIND == P_SUMS && p.direct && blockIdx.x == 0 && threadIdx.x < sizeof(LossInfo) / 4)
    reinterpret_cast<unsigned*>(p.clear)[threadIdx.x] = 0;
  const int live = live_rows<KIND>(p);
  DhPlan plan = {0, 0, 1};
  if (KIND == P_DH) plan = dh_plan(live, p.tiles_n, p.blocks_k, p.workers, p.share_room, products_of(MODE));
  const int units = unit_count<KIND>(p, live, plan);

  constexpr bool kTurnedA = KIND == P_DW, kTurnedB = KIND == P_DH || KIND == P_DW;      // K across the rows in memory
  // (registers change hands inside the branches: where paths meet the compiler counts on the fewer)
  if (warp < kFirstEpi) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegisters));
  // The copies' and the products' loops are run by whole warps, and one lane is elected for the instructions
  // themselves: addresses are then the warp's, in uniform registers, where a loop of one lane moves every operand there
  // first (61 cycles a product and 66 a commit; a K block's four and their waits came to 470 of the 512 that the
  // products take).
  if (warp == 0 || warp == 2) {
    // ---------------- copies: A's by one warp, B's by another ----------------
    const bool of_a = warp == 0;
    uint32_t stage = 0, phase = 0;
    const uint32_t full0 = smem_u32(&full_bar[0]), empty0 = smem_u32(&empty_bar[0]);
    const uint32_t full0_even = PAIR ? map_to_cta(full0, 0u) : full0;
    const int share_n = KIND == P_SUMS ? (PAIR ? p.tile_n / 2 : p.tile_n) : kShareB;
    const uint32_t tx = (PAIR ? 2u : 1u) * (a_stage + b_stage / kShareB * (uint32_t)share_n);
    const int some = p.unmet && of_a && blockIdx.x == 0 ? 0 : units;
    const CUtensorMap* by_rows = KIND == P_DW && p.scaled && !of_one_size(p.info) ? &p.b_common : &p.b;
    bool ok = true;
    for (int u = pair; u < some && ok; u += pairs) {
      const Unit w = unit_at<KIND>(p, u, live, plan);
      const int am = w.m0 + (int)rank * kHalf, bn = w.n0 + (int)rank * share_n;
      for (int kb = w.kb0; kb < w.kb1; ++kb) {
        ok = __all_sync(0xffffffffu, mbar_wait<PAIR>(empty0 + 8u * stage, phase ^ 1u, wc, 1u));
        if (!ok) break;
        if (elect_one()) {
          if (of_a && rank == 0) mbar_expect_tx(full0 + 8u * stage, tx);
          const uint32_t fb = full0_even + 8u * stage;
          const uint32_t to = of_a ? a_tiles + stage * a_stage : b_tiles + stage * b_stage;
          if (KIND == P_SUMS || KIND == P_EXP) {
            if (of_a) tma_load_3d<PAIR>(to, &p.a, fb, kb * kBK, p.first + am, 0);
            else tma_load_3d<PAIR>(to, &p.b, fb, kb * kBK, bn, 0);
          } else if (KIND == P_DH) {
            if (of_a) tma_load_4d<PAIR>(to, &p.a, fb, 0, am, kb, 0);
            else tma_load_4d<PAIR>(to, &p.b, fb, 0, kb * kBK, bn >> 6, 0);
          } else {
            if (of_a) tma_load_4d<PAIR>(to, &p.a, fb, 0, kb * kBK, am >> 6, 0);
            else tma_load_4d<PAIR>(to, by_rows, fb, 0, p.first + kb * kBK, bn >> 6, 0);
          }
        }
        __syncwarp();
        if (++stage == (uint32_t)stages) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // ---------------- products (even CTA, for both) ----------------
    if (rank == 0) {
      uint32_t stage = 0, phase = 0;
      const uint32_t full0 = smem_u32(&full_bar[0]), empty0 = smem_u32(&empty_bar[0]);
      constexpr uint32_t a_base = (kTurnedA ? (8192u >> 4) : 1u) << 16, b_base = (kTurnedB ? (8192u >> 4) : 1u) << 16;
      constexpr uint32_t a_adv = kTurnedA ? (2048u >> 4) : (32u >> 4), b_adv = kTurnedB ? (2048u >> 4) : (32u >> 4);
      constexpr uint32_t term_b = plane_b(PAIR) >> 4;
      const uint32_t term_a = p.a_term >> 4;
      int j = 0;
      bool ok = true;
      for (int u = pair; u < units && ok; u += pairs) {
        const Unit w = unit_at<KIND>(p, u, live, plan);
        const int piece = piece_of(p, w);
        for (int kb0 = w.kb0; kb0 < w.kb1 && ok; kb0 += piece, ++j) {
          const uint32_t set = (uint32_t)j & 1u, aphase = ((uint32_t)j >> 1) & 1u;
          ok = __all_sync(0xffffffffu, mbar_wait<PAIR>(smem_u32(&acc_empty[set]), aphase ^ 1u, wc, 2u));
          if (!ok) break;
          tc_fence_after();
          const uint32_t d = tmem_base + set * (uint32_t)kTile;
          const int kb1 = kb0 + piece < w.kb1 ? kb0 + piece : w.kb1;
          for (int kb = kb0; kb < kb1; ++kb) {
            ok = __all_sync(0xffffffffu, mbar_wait<PAIR>(full0 + 8u * stage, phase, wc, 3u));
            if (!ok) break;
            const uint32_t a0 = (a_tiles + stage * a_stage) >> 4 | a_base, b0 = (b_tiles + stage * b_stage) >> 4 | b_base;
            // (sixteens of K behind the last row are zeros)
            const int steps = KIND == P_DW && live - kb * kBK < kBK ? (live - kb * kBK + 15) / 16 : kBK / 16;
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < kBK / 16; ++k) {
                if (KIND == P_DW && k >= steps) break;
                const uint32_t a = a0 + (uint32_t)k * a_adv, b = b0 + (uint32_t)k * b_adv;
                umma_bf16<PAIR>(d, a, b, p.idesc, k > 0 || kb > kb0);
                if (kTermsB == 2) umma_bf16<PAIR>(d, a, b + term_b, p.idesc, 1u);
                if (kTermsA == 2) umma_bf16<PAIR>(d, a + term_a, b, p.idesc, 1u);
              }
              umma_commit<PAIR>(empty0 + 8u * stage);
              if (kb + 1 == kb1) umma_commit<PAIR>(smem_u32(&acc_full[set]));
            }
            __syncwarp();
            if (++stage == (uint32_t)stages) { stage = 0; phase ^= 1u; }
          }
        }
      }
    }
  } else if (warp >= kFirstEpi) {
    // ---------------- epilogue ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegisters));
    // A lane has a row of 32 and a warp half the tile's columns, all of them in registers: an accumulator is handed
    // back as soon as it has been read.
    const int ew = warp - kFirstEpi, quarter = warp & 3, side = ew >> 2;
    const int buffers = p.buffers;
    const uint32_t sbuf = b_tiles + (uint32_t)stages * b_stage + (uint32_t)(ew * buffers) * kBufferBytes;
    uint32_t turn = 0;
    int j = 0;
    bool ok = true;
    float factor = 1.f;
    int exponent = 0;                               // factor's, but for a row's own (logits)
    if (KIND == P_DW) factor = dweight_factor(p.info, p.scale, p.scaled, kTermsB);
    if (of_logits(KIND)) {
      factor = (float)frexp((double)p.scale * 1.4426950408889634, &exponent);
      if (p.scaled) exponent -= operand_exponent(p.info->w_max, kTermsB, kLeastOfWeight);
    }
    const float mantissa = factor;
    const bool rises = mantissa >= 0.f;             // (the same of all rows, whose logits then go the same way)
    // Blocks of 32 rows of 128 bytes, this lane's row in eight pieces of 16 bytes, into the warp's buffers in turn:
    // `group` of them at a time, since the fence between their stores and the copy engine is what a short tile waits
    // for.
    auto free_buffers = [&](int group) {
      if (lane == 0) {
        if (buffers > group) bulk_wait_read_but_one();
        else bulk_wait_read_all();
      }
      __syncwarp();
    };
    auto next_buffer = [&]() -> uint32_t {
      const uint32_t at = sbuf + turn * kBufferBytes;
      if (++turn == (uint32_t)buffers) turn = 0;
      return at;
    };
    auto hand_over = [&]() {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
    };
    // 32 floats, 64 halves or 64 bf16 numbers from acc + c on
    auto lay_floats = [&](const float* v, uint32_t at) {
#pragma unroll
      for (uint32_t q = 0; q < 8; ++q)
        st_shared_v4(at + piece_at((uint32_t)lane, q), __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]), __float_as_uint(v[4 * q + 2]),
                     __float_as_uint(v[4 * q + 3]));
    };
    auto lay_pairs = [&](const float* v, uint32_t at, auto pack) {
#pragma unroll
      for (uint32_t q = 0; q < 8; ++q)
        st_shared_v4(at + piece_at((uint32_t)lane, q), pack(v[8 * q], v[8 * q + 1]), pack(v[8 * q + 2], v[8 * q + 3]), pack(v[8 * q + 4], v[8 * q + 5]),
                     pack(v[8 * q + 6], v[8 * q + 7]));
    };
    // all of a lane's columns from `acc` to `map`, those before `most`, two blocks a fence where the warp has the
    // buffers
    auto store_all = [&](const float* acc, auto lay, auto columns, const CUtensorMap* map, int col, int row, int most) {
      constexpr int kCols = decltype(columns)::value;
      if (kPairs && buffers >= 2) {
#pragma unroll
        for (int c = 0; c < kSumColumns; c += 2 * kCols) {
          if (c < most) {
            free_buffers(2);
            const uint32_t first = next_buffer(), second = next_buffer();
            lay(acc + c, first);
            lay(acc + c + kCols, second);
            hand_over();
            if (lane == 0) {
              bulk_store_2d(map, first, col + c, row);
              if (c + kCols < most) bulk_store_2d(map, second, col + c + kCols, row);
              else asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
          }
        }
      } else {
#pragma unroll
        for (int c = 0; c < kSumColumns; c += kCols) {
          if (c < most) {
            free_buffers(1);
            const uint32_t at = next_buffer();
            lay(acc + c, at);
            hand_over();
            if (lane == 0) bulk_store_2d(map, at, col + c, row);
          }
        }
      }
    };
    using Wide = std::integral_constant<int, 64>;
    using Narrow = std::integral_constant<int, 32>;
    auto halves = [](float a, float b) { return half2_bits(a, b); };
    auto bf16s = [](float a, float b) { return bf162_bits(a, b); };
    for (int u = pair; u < units && ok; u += pairs) {
      const Unit w = unit_at<KIND>(p, u, live, plan);
      const int row0 = w.m0 + (int)rank * kHalf + quarter * 32, row = row0 + lane;
      // what a tile of logits wants to know of its rows, on its way while the accumulator is waited for
      int own = 0, target = -1;
      if (of_logits(KIND) && row < live) {
        if (p.row_exponent) own = p.row_exponent[p.first + row];
        if (KIND == P_SUMS && p.direct) {
          const int64_t x = p.index_bytes == 4 ? (int64_t) static_cast<const int32_t*>(p.targets)[row] : static_cast<const int64_t*>(p.targets)[row];
          target = x >= 0 && x < p.vocab ? (int)x : -1;
        } else {
          target = p.target[p.first + row];
        }
      }
      const int cols = KIND == P_SUMS ? p.tile_n / 2 : kSumColumns;          // of this warp
      const int col0 = w.n0 + side * cols;
      float acc[kSumColumns];
      const int piece = piece_of(p, w);
      // of few rows most warps have none: they only hand the accumulators back
      const bool idle = KIND != P_DW && row0 >= live;
#pragma unroll 1
      for (int kb0 = w.kb0; kb0 < w.kb1; kb0 += piece) {
        const uint32_t set = (uint32_t)j & 1u, aphase = ((uint32_t)j >> 1) & 1u;
        ++j;
        ok = __all_sync(0xffffffffu, mbar_wait<PAIR>(smem_u32(&acc_full[set]), aphase, wc, 4u));
        if (!ok) break;
        tc_fence_after();
        const uint32_t t0 = tmem_base + ((uint32_t)(quarter * 32) << 16) + set * (uint32_t)kTile + (uint32_t)(side * cols);
        if (kb0 == w.kb0) {
          // the first piece goes where the sum is to be
          if (!idle) {
#pragma unroll
            for (int c = 0; c < kSumColumns; c += 32) tmem_ld32_floats(t0 + (uint32_t)c, acc + c);
          }
          tmem_ld_wait();
        } else if (!idle) {
#pragma unroll
          for (int c = 0; c < kSumColumns; c += 32) {
            uint32_t r[32];
            tmem_ld32_issue(t0 + (uint32_t)c, r);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[c + i] += __uint_as_float(r[i]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (rank != 0) mbar_arrive_cluster(map_to_cta(smem_u32(&acc_empty[set]), 0u));
          else mbar_arrive(smem_u32(&acc_empty[set]));
        }
      }
      if (!ok) break;
      if (idle) continue;
      if (w.kb0 >= w.kb1) {
#pragma unroll
        for (int i = 0; i < kSumColumns; ++i) acc[i] = 0.f;
      }
      if (KIND == P_SUMS || KIND == P_EXP) {
        factor = scaled_by(mantissa, exponent - own);
        if (factor == 0.f) factor = rises ? 1e-30f : -1e-30f;           // (a sign, for what takes a term out of the sum)
        // columns of the vocabulary among them (the registers beyond hold another warp's, or nothing)
        const int left = p.vocab - col0, valid = left < cols ? left : cols;
        const bool on = row < live;
        if (valid > 0) {
          // the largest logit: of a negative factor the least sum's
          const bool whole = valid == kSumColumns;
          float m = -INFINITY;
          if (whole && rises) {
#pragma unroll
            for (int i = 0; i < kSumColumns; ++i) m = fmaxf(m, acc[i]);
            m *= factor;
          } else {
#pragma unroll
            for (int i = 0; i < kSumColumns; ++i) m = fmaxf(m, i < valid ? acc[i] * factor : -INFINITY);
          }
          const int t = target - col0;
          const bool here = on && t >= 0 && t < valid;
          const float power = power_of(m);
          const bool far = on && fabsf(power) >= 4194304.f;
          float shift = 15.f - power;
          if (__any_sync(0xffffffffu, here || far)) {
            float below = -power;
            // Exponentials reach 2^15, near the end of half precision. Logits beyond 2^22 are rounded by half of one
            // and more, as their power was: a lane that has some goes on with the rounded ones' differences to it.
            if (__any_sync(0xffffffffu, far)) {
              const float way = rises ? 1.f : -1.f;
#pragma unroll
              for (int i = 0; i < kSumColumns; ++i) acc[i] = far ? __fadd_rn(__fmul_rn(acc[i], factor), -power) * way : acc[i];
              if (far) { factor = way; shift = 15.f; below = 0.f; }
            }
            // the target's term stays out of the sum, and its logit is kept relative to the power: the loss of a row
            // that is sure of it is what the others' terms add to one, with no difference of two logits in it
            float zt = 0.f;
            const float gone = rises ? -INFINITY : INFINITY;
#pragma unroll
            for (int i = 0; i < kSumColumns; ++i) {
              zt = i == t ? acc[i] : zt;
              acc[i] = i == t ? gone : acc[i];
            }
            if (here) p.target_z[p.first + row] = fmaf(zt, factor, below);
          }
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < kSumColumns; ++i) acc[i] = exp2_fast(fmaf(acc[i], factor, shift));
          if (!whole) {
#pragma unroll
            for (int i = 0; i < kSumColumns; ++i) acc[i] = i < valid ? acc[i] : 0.f;
          }
#pragma unroll
          for (int i = 0; i < kSumColumns; ++i) sum += acc[i];
          if (on) p.sums[(size_t)row * p.sum_blocks + col0 / cols] = make_float2(power, sum);
          if (KIND == P_EXP) {
            // (up to the end of the padded row)
            const int most = (valid + kBK - 1) / kBK * kBK;
            if constexpr (kFloats) store_all(acc, lay_floats, Narrow{}, &p.out, col0, row0, most);
            else store_all(acc, [&](const float* v, uint32_t at) { lay_pairs(v, at, halves); }, Wide{}, &p.out, col0, row0, most);
          }
        }
      } else if (KIND == P_DH || w.share >= 0) {
        if (w.share < 0) store_all(acc, lay_floats, Narrow{}, &p.out, col0, row0, p.dim - col0);
        else store_all(acc, lay_floats, Narrow{}, &p.acc, col0 - w.n0, w.share * kTile + row0 - w.m0, p.dim - col0);
      } else {
        // sums over earlier pieces come from, and unless this is the last go back to, a float array of their own
        const bool add = p.first > 0, last = p.first + p.piece >= p.info->live;
#pragma unroll
        for (int c = 0; c < kSumColumns; c += 32) {
          if (col0 + c < p.dim) {
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[c + i] *= factor;
            if (add && row < p.vocab) {
              const float4* from = reinterpret_cast<const float4*>(p.partial + (size_t)row * p.ld_partial + col0 + c);
#pragma unroll
              for (int q = 0; q < 8; ++q) {
                const float4 v = from[q];
                acc[c + 4 * q] += v.x; acc[c + 4 * q + 1] += v.y; acc[c + 4 * q + 2] += v.z; acc[c + 4 * q + 3] += v.w;
              }
            }
          }
        }
        if (row0 >= p.vocab) continue;
        const int left = p.dim - col0;
        if (!last) {
          store_all(acc, lay_floats, Narrow{}, &p.acc, col0, row0, left);
        } else if (p.dw_engine) {
          if (p.dw_bf16) store_all(acc, [&](const float* v, uint32_t at) { lay_pairs(v, at, bf16s); }, Wide{}, &p.out, col0, row0, left);
          else store_all(acc, lay_floats, Narrow{}, &p.out, col0, row0, left);
        } else if (p.dw_bf16) {
#pragma unroll
          for (int c = 0; c < kSumColumns; c += 64) {
            if (c < left) {
              __syncwarp();
              lay_pairs(acc + c, sbuf, bf16s);
              __syncwarp();
              store_rows<unsigned short, 2>(sbuf, static_cast<unsigned short*>(p.dw) + (size_t)row0 * p.ld_dw + col0 + c, p.ld_dw, p.vocab - row0, left - c, lane);
            }
          }
        } else {
#pragma unroll
          for (int c = 0; c < kSumColumns; c += 32) {
            if (c < left) {
              __syncwarp();
              lay_floats(acc + c, sbuf);
              __syncwarp();
              store_rows<uint32_t, 1>(sbuf, static_cast<uint32_t*>(p.dw) + (size_t)row0 * p.ld_dw + col0 + c, p.ld_dw, p.vocab - row0, left - c, lane);
            }
          }
        }
      }
    }
    if (lane == 0) bulk_wait_all();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0 && lane == 0 && abort_flag) {
    // a wait ran out: copies still in flight get 4 ms to land before the CTA retires
    for (const uint64_t t0 = global_timer_ns(); global_timer_ns() - t0 < 4000000ull;) __nanosleep(1000);
    if (p.total) *p.total = __int_as_float(0x7fffffff);       // (the kernels that follow see the status)
  }
  if (KIND == P_DW && abort_flag && p.shares == 1 && p.first + p.piece >= p.info->live) {
    // no kernel follows that could: what this CTA has not written of dW, and what it has
    for (int u = pair; u < units; u += pairs) {
      const Unit w = unit_at<KIND>(p, u, live, plan);
      for (int i = threadIdx.x; i < kHalf * kTile; i += kLossThreads) {
        const int v = w.m0 + (int)rank * kHalf + i / kTile, c = w.n0 + i % kTile;
        if (v >= p.vocab || c >= p.dim) continue;
        if (p.dw_bf16) static_cast<__nv_bfloat16*>(p.dw)[(int64_t)v * p.ld_dw + c] = __float2bfloat16_rn(__int_as_float(0x7fffffff));
        else static_cast<float*>(p.dw)[(int64_t)v * p.ld_dw + c] = __int_as_float(0x7fffffff);
      }
    }
  }
  if (PAIR) cluster_sync_all();
  tc_fence_after();
  if (warp == 1) {
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

// ---- rows -------------------------------------------------------------------------------------
template <typename I>
__device__ __forceinline__ int target_of(const I* targets, const float* weight, int64_t i, int vocab) {
  const I t = targets[i];
  const bool in = t >= 0 && t < (I)vocab && (weight == nullptr || weight[i] != 0.f);
  return in ? (int)t : -1;
}

template <typename I>
__global__ void __launch_bounds__(kIndexRows) count_live_kernel(const I* targets, const float* weight, int64_t rows, int vocab, int* counts) {
  after_previous();
  const int64_t i = (int64_t)blockIdx.x * kIndexRows + threadIdx.x;
  const int n = __syncthreads_count(i < rows && target_of(targets, weight, i, vocab) >= 0);
  if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

// rows with a target to the front of `row`, in order, the others to its end, and their losses are zero
template <typename I>
__global__ void __launch_bounds__(kIndexRows)
index_live_kernel(const I* targets, const float* weight, int64_t rows, int vocab, const int* counts, int blocks, int* row, int* target,
                  float* g, float* loss, LossInfo* info) {
  after_previous();
  __shared__ int warp_sum[32];
  __shared__ int sums[2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x < 2) sums[threadIdx.x] = 0;
  // a block that is alone counts for itself and clears what the call's kernels share
  const bool alone = counts == nullptr;
  if (alone && threadIdx.x < sizeof(LossInfo) / 4) reinterpret_cast<unsigned*>(info)[threadIdx.x] = 0;
  __syncthreads();
  int mine[2] = {0, 0};
  for (int b = threadIdx.x; !alone && b < blocks; b += kIndexRows) {
    mine[0] += counts[b];
    if (b < (int)blockIdx.x) mine[1] += counts[b];
  }
  if (mine[0]) atomicAdd(&sums[0], mine[0]);
  if (mine[1]) atomicAdd(&sums[1], mine[1]);
  const int64_t i = (int64_t)blockIdx.x * kIndexRows + threadIdx.x;
  const int t = i < rows ? target_of(targets, weight, i, vocab) : -1;
  const unsigned on = __ballot_sync(0xffffffffu, t >= 0);
  if (lane == 0) warp_sum[warp] = __popc(on);
  __syncthreads();
  int live = sums[0];
  if (alone)
    for (int w = 0; w < 32; ++w) live += warp_sum[w];
  int at = sums[1] + __popc(on & ((1u << lane) - 1u));
  for (int w = 0; w < warp; ++w) at += warp_sum[w];
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    info->live = live;
    if (!weight && live > 0) {
      info->g_max = __float_as_uint(1.f / (float)live);
      info->g_far = 0x7fffffffu - info->g_max;
    }
  }
  if (i >= rows) return;
  if (t >= 0) {
    row[at] = (int)i;
    target[at] = t;
    g[at] = weight ? weight[i] : 1.f / (float)live;
    const unsigned bits = __float_as_uint(fabsf(g[at]));
    if (weight && bits < 0x7f800000u) {
      atomicMax(&info->g_max, bits);
      atomicMax(&info->g_far, 0x7fffffffu - bits);
    }
  } else {
    row[rows - 1 - (i - at)] = (int)i;
    loss[i] = 0.f;
  }
}


// bits of a finite |v|, zero of another: the largest of them bounds the operands' range
__device__ __forceinline__ unsigned finite_bits(float v) {
  const unsigned b = __float_as_uint(fabsf(v));
  return b < 0x7f800000u ? b : 0u;
}

// The terms of v; beside an infinity or a NaN the second is zero.
__device__ __forceinline__ void split_half(float v, unsigned short& hi, unsigned short& lo) {
  const __half h = __float2half_rn(v);
  const float back = __half2float(h);
  const __half l = __float2half_rn(isfinite(back) ? v - back : 0.f);
  hi = __half_as_ushort(h);
  lo = __half_as_ushort(l);
}

// the largest of a block's values into *most
__device__ __forceinline__ void block_largest(unsigned m, unsigned* most) {
  __shared__ unsigned warp_m[8];
  m = __reduce_max_sync(0xffffffffu, m);
  if ((threadIdx.x & 31) == 0) warp_m[threadIdx.x >> 5] = m;
  __syncthreads();
  if (threadIdx.x < 32) {
    m = __reduce_max_sync(0xffffffffu, threadIdx.x < 8 ? warp_m[threadIdx.x] : 0u);
    if (threadIdx.x == 0 && m) atomicMax(most, m);
  }
}

__device__ __forceinline__ void split_bf16(float v, unsigned short& hi, unsigned short& lo) {
  const __nv_bfloat16 h = __float2bfloat16_rn(v);
  const float back = __bfloat162float(h);
  hi = __bfloat16_as_ushort(h);
  lo = __bfloat16_as_ushort(__float2bfloat16_rn(isfinite(back) ? v - back : 0.f));
}

// h (rows with a target, by their index) and W as operands: [terms][staged rows][padded columns], zero beyond a row's
// end, and of h beyond the last row to a multiple of a tile
template <typename T>
struct Operands {
  const T *w, *h;
  int64_t ld_w, ld_h;
  unsigned short *w_out, *h_out;
  unsigned short* common_out;     // h as dW wants it where the rows are not of one size (null: not wanted)
  const int* row;
  const float* g;
  int* row_exponent;
  int vocab, dim, padded;
  int rows, staged_rows;          // of h
  T* dead;                        // rows of dh that get zeros
  int64_t ld_dead;
  LossInfo* info;
  int row_threads;                // of a row of h
  int64_t w_blocks;               // the first blocks are W's
};

// What a thread has of a row at a time: eight columns, on their way (WIDE) before the first is used
template <typename T, bool WIDE>
struct Eights {
  static constexpr int kAhead = WIDE ? (sizeof(T) == 2 ? 4 : 2) : 1, kLoads = sizeof(T) == 2 ? 1 : 2;
  uint4 raw[kAhead][kLoads];
  // from: a row's start, or null
  __device__ __forceinline__ void load(int a, const T* from, int c, int dim) {
#pragma unroll
    for (int q = 0; q < kLoads; ++q)
      raw[a][q] = WIDE && from && c + q * 4 < dim ? reinterpret_cast<const uint4*>(from + c)[q] : make_uint4(0u, 0u, 0u, 0u);
  }
  // their terms under f1 f2, and the largest finite of them (bits; not where it is not LARGEST)
  template <int TERMS, bool SCALED, bool LARGEST>
  __device__ __forceinline__ unsigned write(int a, const T* from, int c, int dim, float f1, float f2, unsigned short* out, int64_t next_term) const {
    const uint32_t b[4] = {raw[a][0].x, raw[a][0].y, raw[a][0].z, raw[a][0].w};
    unsigned short hi[8], lo[8];
    unsigned m = 0;
    if (SCALED && WIDE && sizeof(T) == 2) {
      // eight bf16 numbers: two conversions an instruction, and the largest of them two at a time (beside an infinity
      // or a NaN one by one)
      uint32_t pair = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t h = half2_bits(__uint_as_float(b[k] << 16) * f1 * f2, __uint_as_float(b[k] & 0xffff0000u) * f1 * f2);
        hi[2 * k] = (unsigned short)h;
        hi[2 * k + 1] = (unsigned short)(h >> 16);
        if (LARGEST) pair = __vmaxu2(pair, b[k] & 0x7fff7fffu);
      }
      if (LARGEST) {
        const unsigned top = max(pair & 0xffffu, pair >> 16);
        if (top < 0x7f80u) {
          m = top << 16;
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) m = max(m, max(finite_bits(__uint_as_float(b[k] << 16)), finite_bits(__uint_as_float(b[k] & 0xffff0000u))));
        }
      }
    } else if (SCALED) {
      float v[8];
      if (WIDE) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint4& w = raw[a][k / 4 % kLoads];
          v[k] = __uint_as_float(k % 4 == 0 ? w.x : (k % 4 == 1 ? w.y : (k % 4 == 2 ? w.z : w.w)));
        }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = from && c + k < dim ? to_f32(from[c + k]) : 0.f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (LARGEST) m = max(m, finite_bits(v[k]));
        split_half(v[k] * f1 * f2, hi[k], lo[k]);
      }
    } else {
      const unsigned short* x = reinterpret_cast<const unsigned short*>(from);
#pragma unroll
      for (int k = 0; k < 8; ++k) hi[k] = WIDE ? (unsigned short)(b[k / 2] >> (k % 2 * 16)) : (from && c + k < dim ? x[c + k] : (unsigned short)0);
    }
    auto pack = [](const unsigned short (&x)[8]) {
      return make_uint4(x[0] | (uint32_t)x[1] << 16, x[2] | (uint32_t)x[3] << 16, x[4] | (uint32_t)x[5] << 16, x[6] | (uint32_t)x[7] << 16);
    };
    *reinterpret_cast<uint4*>(out + c) = pack(hi);
    if (TERMS == 2) *reinterpret_cast<uint4*>(out + c + next_term) = pack(lo);
    return m;
  }
};

// W under one power of two, in pieces of eight columns whatever the rows.  AGAIN: only where it is of an unusual size.
template <typename T, int TERMS, bool SCALED, bool WIDE, bool AGAIN>
__device__ __forceinline__ void stage_weight(const Operands<T>& o) {
  int e = 0;
  if (SCALED) {
    e = usual_exponent(TERMS);
    if (AGAIN) {
      if (!unusual(o.info->w_max, TERMS, kLeastOfWeight)) return;
      e = range_exponent(o.info->w_max);
    }
  }
  const float f = power_of_two(e);
  const uint32_t per = (uint32_t)o.padded / 8;
  const int64_t items = (int64_t)o.vocab * per;
  const bool small = items < 0x7fffffff;
  unsigned m = 0;
  using Pieces = Eights<T, WIDE>;
  constexpr int kAhead = Pieces::kAhead;
  for (int64_t i0 = (int64_t)blockIdx.x * (256 * kAhead) + threadIdx.x; i0 < items; i0 += o.w_blocks * (256 * kAhead)) {
    Pieces x;
    int rr[kAhead], cc[kAhead];            // (rows are 2^24 at the most)
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int64_t i = i0 + a * 256;
      rr[a] = i < items ? (int)(small ? (uint32_t)i / per : i / per) : -1;
      cc[a] = i < items ? (int)((uint32_t)i - (uint32_t)rr[a] * per) * 8 : 0;
      x.load(a, rr[a] >= 0 ? o.w + (int64_t)rr[a] * o.ld_w : nullptr, cc[a], o.dim);
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a)
      if (rr[a] >= 0)
        m = max(m, x.template write<TERMS, SCALED, !AGAIN>(a, o.w + (int64_t)rr[a] * o.ld_w, cc[a], o.dim, f, 1.f, o.w_out + (int64_t)rr[a] * o.padded,
                                                            (int64_t)o.vocab * o.padded));
  }
  if (SCALED && !AGAIN) block_largest(m, &o.info->w_max);
}

// The rows of h, `row_threads` each (8, 32 or 256), under a power of two each. AGAIN: for dW, where they are not of one
// size.
template <typename T, int TERMS, bool SCALED, bool WIDE, bool AGAIN>
__device__ __forceinline__ void stage_rows(const Operands<T>& o) {
  __shared__ unsigned warp_m[2][8];
  if (AGAIN && (!o.common_out || of_one_size(o.info))) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, threads = o.row_threads, thread = (int)threadIdx.x % threads, at_once = 256 / threads;
  const int64_t blocks = gridDim.x - o.w_blocks, block = blockIdx.x - o.w_blocks;
  const int n = o.info->live, whole = (n + kTile - 1) / kTile * kTile, upto = whole < o.staged_rows ? whole : o.staged_rows;
  const int last = o.dead && upto < o.rows ? o.rows : upto;
  const int64_t next_term = (int64_t)o.staged_rows * o.padded;
  unsigned short* to = AGAIN ? o.common_out : o.h_out;
  using Pieces = Eights<T, WIDE>;
  constexpr int kStep = 8 * Pieces::kAhead;
  unsigned reach = 0, uneven = 0;
  int turn = 0;
  // (the lanes of a warp together, whatever rows they have)
  for (int64_t r0 = block * at_once; r0 < last; r0 += blocks * at_once, turn ^= 1) {
    const int64_t r = r0 + threadIdx.x / threads;
    unsigned short* out = to + r * o.padded;
    if (r >= n && r < last) {
      if (r < upto)
        for (int c = thread * 8; c < o.padded; c += threads * 8) {
          *reinterpret_cast<uint4*>(out + c) = make_uint4(0u, 0u, 0u, 0u);
          if (TERMS == 2) *reinterpret_cast<uint4*>(out + c + next_term) = make_uint4(0u, 0u, 0u, 0u);
        }
      if (!AGAIN && o.dead && r < o.rows)
        for (int c = thread; c < o.dim; c += threads) o.dead[(int64_t)o.row[r] * o.ld_dead + c] = from_f64<T>(0.0);
    }
    if (r0 >= n) continue;
    const bool on = r < n;
    const T* from = on ? o.h + (int64_t)o.row[r] * o.ld_h : nullptr;
    auto pass = [&](auto largest, int e) {
      constexpr bool kLargest = decltype(largest)::value;
      unsigned m = 0;
      const float f1 = power_of_two(e / 2), f2 = power_of_two(e - e / 2);
      for (int c0 = thread * 8; on && c0 < o.padded; c0 += threads * kStep) {
        Pieces x;
#pragma unroll
        for (int a = 0; a < Pieces::kAhead; ++a) x.load(a, from, c0 + a * threads * 8, o.dim);
#pragma unroll
        for (int a = 0; a < Pieces::kAhead; ++a)
          if (c0 + a * threads * 8 < o.padded)
            m = max(m, x.template write<TERMS, SCALED, kLargest>(a, from, c0 + a * threads * 8, o.dim, f1, f2, out, next_term));
      }
      return m;
    };
    if (AGAIN) {
      const int e = common_exponent(o.info) - (on ? weight_exponent(o.g[r]) : 0);
      pass(std::false_type{}, e < -250 ? -250 : (e > 250 ? 250 : e));
    } else if (!SCALED) {
      pass(std::false_type{}, 0);
    } else {
      unsigned m = pass(std::true_type{}, usual_exponent(TERMS));
      if (threads < 32) {
#pragma unroll
        for (int d = 4; d; d >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, d));
      } else {
        m = __reduce_max_sync(0xffffffffu, m);
      }
      if (threads > 32) {
        if (lane == 0) warp_m[turn][warp] = m;
        __syncthreads();
        m = __reduce_max_sync(0xffffffffu, warp_m[turn][lane & 7]);
      }
      const bool other = unusual(m, TERMS, kLeastOfRow);
      if (other) pass(std::false_type{}, range_exponent(m));
      if (on && thread == 0) o.row_exponent[r] = operand_exponent(m, TERMS, kLeastOfRow);
      if (m && fabsf(o.g[r]) < INFINITY) reach = max(reach, (unsigned)(1024 + (int)(m >> 23) - 127 - weight_exponent(o.g[r])));
      uneven |= other;
    }
  }
  if (SCALED && !AGAIN) {
    block_largest(reach, &o.info->reach);
    if (uneven && thread == 0) o.info->uneven = 1;
  }
}

template <typename T, int TERMS, bool SCALED, bool WIDE, bool AGAIN>
__global__ void __launch_bounds__(256, WIDE ? 4 : 6) stage_kernel(const Operands<T> o) {
  after_previous();
  if (blockIdx.x < o.w_blocks) stage_weight<T, TERMS, SCALED, WIDE, AGAIN>(o);
  else stage_rows<T, TERMS, SCALED, WIDE, AGAIN>(o);
}

// joins the sums of a row's blocks: log2 of the whole sum
struct RowSum { float k, sum; };
__device__ __forceinline__ RowSum join(RowSum a, RowSum b) {
  const float k = fmaxf(a.k, b.k);
  return {k, a.sum * exp2_fast(a.k - k) + b.sum * exp2_fast(b.k - k)};
}
__device__ __forceinline__ RowSum warp_join(RowSum v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const RowSum o = {__shfl_xor_sync(0xffffffffu, v.k, d), __shfl_xor_sync(0xffffffffu, v.sum, d)};
    // (both lanes of a pair join in the same order, so all lanes have the same bits)
    v = (threadIdx.x & d) ? join(o, v) : join(v, o);
  }
  return v;
}
// What a row's sums say: `v` of all terms but the target's (times 2^15, relative to 2^v.k), the target's logit relative
// to its own block's power.  odds: log2 of the others' terms over the target's.
struct RowEnd {
  float loss, total, less;      // the loss, all terms as v.sum holds them, 1 - p of the target
};
__device__ __forceinline__ RowEnd row_end(const LossInfo* info, RowSum v, float target_z, float target_power) {
  RowEnd e;
  const float odds = (v.k - target_power) + log2f(v.sum * 0x1p-15f) - target_z, r = exp2f(odds);
  const bool far = odds > 24.f;
  e.loss = far ? 0.69314718055994531f * odds : log1pf(r);
  e.less = far ? 1.f : r / (1.f + r);
  e.total = v.sum + exp2f((target_power - v.k) + 15.f + target_z);
  // a wait ran out: nothing here is right; or the target's logit is infinite, and inf - inf no difference
  if (info->st.code != 0 || target_z == INFINITY) e.loss = e.total = e.less = __int_as_float(0x7fffffff);
  return e;
}

// The last block of the launch that brings the last losses adds them up, in an order that the rows' number alone sets.
__device__ __forceinline__ void total_by_last(LossInfo* info, int n, const double* part, float* total) {
  __shared__ double sums[8];
  __shared__ bool last;
  if (total == nullptr) return;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(&info->done, 1u) + 1u == gridDim.x;
    __threadfence();
  }
  __syncthreads();
  if (!last) return;
  double t = 0.0;
#pragma unroll 8
  for (int i = threadIdx.x; i < n; i += 256) t += __ldcg(part + i);
#pragma unroll
  for (int d = 16; d; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    t = 0.0;
    for (int i = 0; i < 8; ++i) t += sums[i];
    // (a wait that ran out where gradients of earlier rows are formed leaves these losses right, and the call wrong)
    *total = info->st.code != 0 ? __int_as_float(0x7fffffff) : (float)t;
  }
}

// losses of all live rows, a warp each
__global__ void __launch_bounds__(256)
loss_rows_kernel(LossInfo* info, const float2* sums, int sum_blocks, const float* target_z, const int* row, const int* target, const float* g,
                 float* loss, double* part, float* total) {
  after_previous();
  const int lane = threadIdx.x & 31;
  for (int64_t i = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); i < info->live; i += (int64_t)gridDim.x * 8) {
    RowSum v = {kNoPower, 0.f};
    for (int b0 = lane; b0 < sum_blocks; b0 += 32 * 8) {
      float2 x[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] = b0 + 32 * q < sum_blocks ? sums[i * sum_blocks + b0 + 32 * q] : make_float2(kNoPower, 0.f);
#pragma unroll
      for (int q = 0; q < 8; ++q) v = join(v, {x[q].x, x[q].y});
    }
    v = warp_join(v);
    if (lane == 0) {
      const float l = row_end(info, v, target_z[i], sums[i * sum_blocks + target[i] / kSumColumns].x).loss;
      loss[row[i]] = l;
      part[i] = (double)g[i] * (double)l;
    }
  }
  total_by_last(info, info->live, part, total);
}

// The same of at most 256 rows that were taken as they are: those left out are found here.
template <typename I>
__global__ void __launch_bounds__(256)
direct_rows_kernel(LossInfo* info, const float2* sums, int sum_blocks, int columns, const float* target_z, const I* targets, const float* weight, int rows,
                   int vocab, float* loss, double* part, float* total) {
  after_previous();
  const int lane = threadIdx.x & 31, mine = threadIdx.x;
  const int live = __syncthreads_count(mine < rows && target_of(targets, weight, mine, vocab) >= 0);
  const int i = (int)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (i < rows) {
    const bool on = target_of(targets, weight, i, vocab) >= 0;
    RowSum v = {kNoPower, 0.f};
    for (int b0 = lane; b0 < sum_blocks && on; b0 += 32 * 8) {
      float2 x[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] = b0 + 32 * q < sum_blocks ? sums[(size_t)i * sum_blocks + b0 + 32 * q] : make_float2(kNoPower, 0.f);
#pragma unroll
      for (int q = 0; q < 8; ++q) v = join(v, {x[q].x, x[q].y});
    }
    v = warp_join(v);
    if (lane == 0) {
      const float l = on ? row_end(info, v, target_z[i], sums[(size_t)i * sum_blocks + (int)targets[i] / columns].x).loss : 0.f;
      loss[i] = l;
      part[i] = on ? (double)(weight ? weight[i] : 1.f / (float)live) * (double)l : 0.0;
    }
  }
  total_by_last(info, rows, part, total);
}

// a row's exponentials -> dz times a power of two, in their place: WARPS warps of a block of eight a row, or `slices`
// blocks where rows are few and long (each joins the row's sums for itself)
template <int MODE, int WARPS>
__global__ void __launch_bounds__(256)
dz_kernel(LossInfo* info, int first, int piece, const float2* sums, int sum_blocks, const float* target_z, const int* row,
          const int* target, const float* g, float* loss, double* part, float* total, unsigned short* e, int padded, int slices) {
  after_previous();
  __shared__ RowSum warp_v[8];
  constexpr int kThreads = WARPS * 32, kRows = 8 / WARPS, TERMS = MODE == M_ONE ? 1 : 2;
  constexpr int kColumns = MODE == M_THIN ? kThinColumns : kSumColumns;
  int live = info->live - first;
  live = live < 0 ? 0 : (live < piece ? live : piece);
  int upto = (live + kBK - 1) / kBK * kBK;            // (behind the piece's rows the copy engine brings zeros)
  upto = MODE == M_THIN ? live : (upto < piece ? upto : piece);
  const int warp = WARPS == 1 ? 0 : (int)(threadIdx.x >> 5), lane = threadIdx.x & 31, thread = (int)threadIdx.x % kThreads;
  for (int b = (int)blockIdx.x; b * kRows < upto * slices; b += gridDim.x) {
    const int slice = b % slices, r = b / slices * kRows + (WARPS == 1 ? (int)(threadIdx.x >> 5) : 0);
    if (WARPS == 1 && r >= upto) break;
    unsigned short* at = e + (size_t)r * padded * TERMS;
    if (r >= live) {                                  // rows that fill up the last block of K
      for (int c = slice * kThreads + thread; c < padded * TERMS / 8; c += slices * kThreads) reinterpret_cast<uint4*>(at)[c] = make_uint4(0u, 0u, 0u, 0u);
      continue;
    }
    const float2* mine = sums + (size_t)r * sum_blocks;
    const int i = first + r, t = target[i];
    RowSum v = {kNoPower, 0.f};
    for (int b = thread; b < sum_blocks; b += kThreads) v = join(v, {mine[b].x, mine[b].y});
    v = warp_join(v);
    if (WARPS > 1) {
      __syncthreads();
      if (lane == 0) warp_v[warp] = v;
      __syncthreads();
      v = warp_v[0];
      for (int w = 1; w < WARPS; ++w) v = join(v, warp_v[w]);
    }
    const RowEnd end = row_end(info, v, target_z[i], mine[t / kColumns].x);
    if (thread == 0 && slice == 0) {
      loss[row[i]] = end.loss;
      part[i] = (double)g[i] * (double)end.loss;
    }
    const float gi = g[i] * (MODE == M_THIN ? 1.f : power_of_two(MODE == M_FEW ? weight_exponent(info->g_max) : weight_exponent(g[i]))), at_target = -gi * end.less, share = gi / end.total;
    // (four accesses of a thread under way)
    constexpr int kAhead = 4;
    if (TERMS == 1) {
      for (int c0 = (slice * kAhead * kThreads + thread) * 8; c0 < padded; c0 += slices * kThreads * 8 * kAhead) {
        uint4 raw[kAhead];
        float f[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int c = c0 + j * kThreads * 8;
          if (c < padded) {
            raw[j] = *reinterpret_cast<const uint4*>(at + c);
            f[j] = mine[c / kColumns].x;
          }
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int c = c0 + j * kThreads * 8;
          if (c < padded) {
            const float by = share * exp2_fast(f[j] - v.k);
            const uint32_t in[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
            uint32_t out[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&in[q]));
              out[q] = half2_bits(x.x * by, x.y * by);
            }
            if (t >= c && t < c + 8) {
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const uint32_t h = half2_bits(at_target, at_target);
                if (t - c == 2 * q) out[q] = (out[q] & 0xffff0000u) | (h & 0xffffu);
                if (t - c == 2 * q + 1) out[q] = (out[q] & 0xffffu) | (h & 0xffff0000u);
              }
            }
            *reinterpret_cast<uint4*>(at + c) = make_uint4(out[0], out[1], out[2], out[3]);
          }
        }
      }
    } else {
      // a group of 64 floats becomes 64 leading terms and 64 remainders: sixteen lanes, four of them each
      for (int c0 = (slice * kAhead * WARPS + warp) * 128 + lane * 4; c0 - lane * 4 < padded; c0 += slices * WARPS * 128 * kAhead) {          // (a warp together)
        float4 raw[kAhead];
        float f[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int c = c0 + j * WARPS * 128;
          if (c < padded) {
            raw[j] = *reinterpret_cast<const float4*>(at + 2 * c);
            f[j] = mine[c / kColumns].x;
          }
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int c = c0 + j * WARPS * 128;
          if (c < padded) {
            const float by = share * exp2_fast(f[j] - v.k);
            float x[4] = {raw[j].x * by, raw[j].y * by, raw[j].z * by, raw[j].w * by};
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = c + q == t ? at_target : x[q];
            if (MODE == M_THIN) {
              *reinterpret_cast<float4*>(at + 2 * c) = make_float4(x[0], x[1], x[2], x[3]);
              continue;
            }
            unsigned short hi[4], lo[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if (MODE == M_FEW) split_bf16(x[q], hi[q], lo[q]);
              else split_half(x[q], hi[q], lo[q]);
            }
            unsigned short* to = at + 2 * (c & ~63) + (c & 63);
            *reinterpret_cast<uint2*>(to) = make_uint2(hi[0] | (uint32_t)hi[1] << 16, hi[2] | (uint32_t)hi[3] << 16);
            *reinterpret_cast<uint2*>(to + 64) = make_uint2(lo[0] | (uint32_t)lo[1] << 16, lo[2] | (uint32_t)lo[3] << 16);
          }
        }
      }
    }
  }
  total_by_last(info, info->live, part, total);
}

__device__ __forceinline__ void put(float* at, float v) { *at = v; }
__device__ __forceinline__ void put(__nv_bfloat16* at, float v) { *at = __float2bfloat16_rn(v); }

// dh of the piece's rows: the sums over the shares of K, in order, to the rows they belong to, four columns a thread
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256)
dh_rows_kernel(LossArgs a, const float* slab, const float* shares, int padded, int tiles_n, int blocks_k, int workers, int room, int mode, int first,
               int piece, const int* row, const float* g, const LossInfo* info, T* dh) {
  after_previous();
  int live = info->live - first;
  live = live < 0 ? 0 : (live < piece ? live : piece);
  int exponent = 0;
  float mantissa = (float)frexp((double)a.scale, &exponent);
  if (a.scaled) exponent -= operand_exponent(info->w_max, terms_b(mode), kLeastOfWeight);
  if (info->st.code != 0) mantissa = __int_as_float(0x7fffffff);
  const DhPlan plan = dh_plan(live, tiles_n, blocks_k, workers, room, products_of(mode));
  const uint32_t per = (uint32_t)(a.dim + 3) / 4;
  const int64_t items = (int64_t)live * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per;
    const int c = (int)(i % per) * 4;
    float4 v = *reinterpret_cast<const float4*>(slab + (size_t)r * padded + c);
    const int tile = (int)(r / kTile) * tiles_n + c / kTile;
    if (tile >= plan.whole) {
      const float* from = shares + ((size_t)(tile - plan.whole) * (plan.shares - 1) * kTile + r % kTile) * kTile + c % kTile;
      for (int s = 1; s < plan.shares; ++s, from += kTile * kTile) {
        const float4 x = *reinterpret_cast<const float4*>(from);
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
      }
    }
    // (two factors: their product may lie below a float's range where dh does not)
    int x = exponent - (a.scaled ? weight_exponent(g[first + r]) : weight_exponent(info->g_max));
    x = x < -250 ? -250 : (x > 250 ? 250 : x);
    const float f1 = mantissa * power_of_two(x / 2), f2 = power_of_two(x - x / 2);
    v.x = v.x * f1 * f2; v.y = v.y * f1 * f2; v.z = v.z * f1 * f2; v.w = v.w * f1 * f2;
    T* to = dh + (int64_t)row[first + r] * a.ld_dh + c;
    if (WIDE) {
      if (sizeof(T) == 4) *reinterpret_cast<float4*>(to) = v;
      else *reinterpret_cast<uint2*>(to) = make_uint2(bf162_bits(v.x, v.y), bf162_bits(v.z, v.w));
    } else {
      const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k < a.dim) put(to + k, x[k]);
    }
  }
}

// dW of few tiles: the sums over the shares of K, in order, and over the pieces before, four columns a thread
template <typename G>
__global__ void __launch_bounds__(256)
dw_rows_kernel(LossArgs a, const float* blocks, int tiles_n, int shares, int mode, int first, int piece, const LossInfo* info, float* partial,
               int padded, G* dw) {
  after_previous();
  const int live = info->live;
  if (first > 0 && live <= first) return;
  const bool last = first + piece >= live;
  const float f = dweight_factor(info, a.scale, a.scaled, terms_b(mode));
  const uint32_t per = (uint32_t)(a.dim + 3) / 4;
  const int64_t items = (int64_t)a.vocab * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
    const int64_t v = i / per;
    const int c = (int)(i - v * per) * 4;
    const int tile = (int)(v / kTile) * tiles_n + c / kTile;
    const float* from = blocks + ((size_t)tile * shares * kTile + v % kTile) * kTile + c % kTile;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < shares; ++s, from += kTile * kTile) {
      const float4 y = *reinterpret_cast<const float4*>(from);
      x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
    }
    x.x *= f; x.y *= f; x.z *= f; x.w *= f;
    float4* held = reinterpret_cast<float4*>(partial + (size_t)v * padded + c);
    if (first > 0) {
      const float4 y = *held;
      x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
    }
    if (!last) {
      *held = x;
    } else {
      const float y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k < a.dim) put(dw + v * a.ld_dw + c + k, y[k]);
    }
  }
}

// ---- very few rows ----------------------------------------------------------------------------
// Up to 8 rows of fp32. As operands W passes memory three times for the loss and five for the gradient; here each
// kernel reads it once (or writes dW), in fp32 throughout, and the CUDA cores' multiplications stay below the time of
// that. Beside the products: loss of 32768x2048 59 us of 1 row, 81 of 8 (154), gradient 179 and 213 us (276); of
// 848x512 17 (33) and 32 (57); of 131072x100 gradient 108 and 165 (157). 16 rows took 155 and 325 us (154, 277), as
// bf16 rows off the copy engine's boundaries did (8 rows of 33620x1615 gradient 272 us, 199 as operands). Bound by
// memory: 8 rows' logits 3.4 TB/s (their h out of shared memory takes as long as the multiplications), 4 rows' 4.2; dh
// 6.0 and 4.4 TB/s, eight rows of W under way a thread; dW 5.6. (Tiles of 32 logits, which divide evenly among the
// blocks, were no faster: 62 us of 1 row.) A thread's four numbers of a group of 4 * STRIDE: together where rows allow
// 16 bytes at a time, else STRIDE apart.
template <bool WIDE, int STRIDE>
__device__ __forceinline__ int place(int i, int j) { return WIDE ? 4 * i + j : i + STRIDE * j; }
__device__ __forceinline__ void load_wide(const float* from, float (&x)[4]) {
  const float4 v = *reinterpret_cast<const float4*>(from);
  x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
// zeros from `left` on (WIDE: a multiple of four)
template <bool WIDE, int STRIDE>
__device__ __forceinline__ void load_four(const float* from, int i, int left, float (&x)[4]) {
  if (WIDE) {
    if (4 * i < left) load_wide(from + 4 * i, x);
    else x[0] = x[1] = x[2] = x[3] = 0.f;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = i + STRIDE * j < left ? from[i + STRIDE * j] : 0.f;
  }
}
// Sums over a warp's lanes of N numbers each: afterwards a lane has number (lane * N + i) / 32 in v[i], i < N / 32 or
// one
template <int N>
__device__ __forceinline__ void sum_lanes(float (&v)[N], int lane) {
  int m = N;
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    if (m > 1) {
      m /= 2;
      const bool upper = lane & d;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        if (i < m) {
          const float give = upper ? v[i] : v[i + m], keep = upper ? v[i + m] : v[i];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, give, d);
        }
      }
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], d);
    }
  }
}

// What P_SUMS (and, with `e`, P_EXP) leave, by blocks of 64 logits: a warp takes four rows of W at a time against all
// rows of h, which lie in shared memory, whole or `chunk` columns of them.
template <int R, bool WIDE>
__global__ void __launch_bounds__(512, 1)
thin_logits_kernel(const float* h, int64_t ld_h, const float* w, int64_t ld_w, int rows, int vocab, int dim, int chunk, float factor, LossInfo* info,
                   const int* row, const int* target, const void* targets, int index_bytes, float2* sums, int sum_blocks, float* target_z,
                   float* e, int padded) {
  extern __shared__ __align__(16) float hs[];          // [R][chunk]
  __shared__ float zs[2][R][kThinColumns];
  after_previous();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (!row && blockIdx.x == 0 && threadIdx.x < sizeof(LossInfo) / 4) reinterpret_cast<unsigned*>(info)[threadIdx.x] = 0;
  const int live = row ? info->live : rows;
  if (live == 0) return;
  int t = -1;
  if (warp < live) {
    if (row) {
      t = target[warp];
    } else {
      const int64_t x = index_bytes == 4 ? (int64_t) static_cast<const int32_t*>(targets)[warp] : static_cast<const int64_t*>(targets)[warp];
      t = x >= 0 && x < vocab ? (int)x : -1;
    }
  }
  bool there = false;
  int turn = 0;
  for (int tile = blockIdx.x; (int64_t)tile * kThinColumns < vocab; tile += gridDim.x, turn ^= 1) {
    const int v0 = tile * kThinColumns + warp * 4;
    float acc[4 * R];
#pragma unroll
    for (int i = 0; i < 4 * R; ++i) acc[i] = 0.f;
    const float* from[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) from[v] = w + (int64_t)(v0 + v < vocab ? v0 + v : vocab - 1) * ld_w;
    for (int k0 = 0; k0 < dim; k0 += chunk) {
      const int kc = dim - k0 < chunk ? dim - k0 : chunk;
      // (two groups of 128 columns under way while two are multiplied)
      float x[2][4][4], next[2][4][4];
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int v = 0; v < 4; ++v) load_four<WIDE, 32>(from[v] + k0 + 128 * g, lane, kc - 128 * g, x[g][v]);
      if (!there || chunk < dim) {
        __syncthreads();
        for (int i = threadIdx.x; i < R * chunk; i += 512) {
          const int r = i / chunk, c = k0 + i - r * chunk;
          hs[i] = r < live && c < dim ? h[(int64_t)(row ? row[r] : r) * ld_h + c] : 0.f;
        }
        there = true;
        __syncthreads();
      }
      for (int k = 0; k < kc; k += 256) {
        if (k + 256 < kc) {
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int v = 0; v < 4; ++v) load_four<WIDE, 32>(from[v] + k0 + k + 256 + 128 * g, lane, kc - k - 256 - 128 * g, next[g][v]);
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          if (k + 128 * g < kc) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float* at = hs + r * chunk + k + 128 * g;
              float y[4];
              if (WIDE) load_wide(at + 4 * lane, y);
              else {
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = at[lane + 32 * j];
              }
#pragma unroll
              for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[v * R + r] = fmaf(x[g][v][j], y[j], acc[v * R + r]);
            }
          }
        }
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[g][v][j] = next[g][v][j];
      }
    }
    sum_lanes<4 * R>(acc, lane);
    constexpr int kEach = 4 * R / 32 > 1 ? 4 * R / 32 : 1;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int n = lane * (4 * R) / 32 + i;
      zs[turn][n % R][warp * 4 + n / R] = acc[i] * factor;
    }
    __syncthreads();
    if (warp < live && warp < R) {
      const int col = tile * kThinColumns + lane;
      float z[2];
      float m = -INFINITY;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        z[q] = col + 32 * q < vocab ? zs[turn][warp][lane + 32 * q] : -INFINITY;
        m = fmaxf(m, z[q]);
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      const float power = power_of(m);
      float sum = 0.f;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        // (the target's term is kept apart)
        if (col + 32 * q == t) {
          target_z[warp] = z[q] - power;
          z[q] = -INFINITY;
        }
        const float x = exp2_fast(z[q] + (15.f - power));
        if (e) e[(int64_t)warp * padded + col + 32 * q] = x;
        sum += x;
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (lane == 0) sums[(int64_t)warp * sum_blocks + tile] = make_float2(power, sum);
    }
  }
}

// 64 rows of the vocabulary's dz, [row of W][row of h]
template <int R>
__device__ __forceinline__ void thin_rows(float (*d)[R], const float* e, int padded, int live, int v0, int v1) {
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * R; i += 256) {
    const int r = i / 64, j = i - r * 64;
    d[j][r] = r < live && v0 + j < v1 ? e[(int64_t)r * padded + v0 + j] : 0.f;
  }
  __syncthreads();
}
// dz W over `per` rows of W, 1024 columns a block, four a thread
template <int R, bool WIDE>
__global__ void __launch_bounds__(256)
thin_dh_kernel(const float* w, int64_t ld_w, int vocab, int dim, const LossInfo* info, const float* e, int padded, float* parts, int tiles, int per) {
  __shared__ __align__(16) float d[64][R];
  after_previous();
  const int live = info->live, tile = blockIdx.x % tiles, slice = blockIdx.x / tiles, left = dim - tile * 1024;
  if (live == 0) return;
  const int v0 = slice * per, v1 = v0 + per < vocab ? v0 + per : vocab;
  float acc[R][4];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[r][j] = 0.f;
  for (int vb = v0; vb < v1; vb += 64) {
    thin_rows<R>(d, e, padded, live, vb, v1);
    const int n = v1 - vb < 64 ? v1 - vb : 64;
    const float* from = w + (int64_t)vb * ld_w + tile * 1024;
    for (int v = 0; v < n; v += 8, from += 8 * ld_w) {
      float x[8][4];
#pragma unroll
      for (int u = 0; u < 8; ++u) load_four<WIDE, 256>(from + (v + u < n ? u : 0) * ld_w, threadIdx.x, left, x[u]);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        if (v + u < n) {
#pragma unroll
          for (int r = 0; r < R; r += 4) {
            float y[4];
            load_wide(&d[v + u][r], y);
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int j = 0; j < 4; ++j) acc[r + q][j] = fmaf(y[q], x[u][j], acc[r + q][j]);
          }
        }
      }
    }
  }
  float* to = parts + ((int64_t)slice * R * tiles + tile) * 1024;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) to[(int64_t)r * tiles * 1024 + place<WIDE, 256>(threadIdx.x, j)] = acc[r][j];
}
// ... of all slices, in order, to the rows they belong to, and zeros to those left out: a block 32 columns of a row
__global__ void __launch_bounds__(256)
thin_dh_rows_kernel(LossArgs a, const float* parts, int tiles, int padded_rows, int slices, const int* row, const LossInfo* info, float* dh) {
  __shared__ __align__(16) float4 some[32][8];
  after_previous();
  const int r = blockIdx.y, part = threadIdx.x >> 3, quad = threadIdx.x & 7, c = blockIdx.x * 32 + quad * 4;
  const bool on = r < info->live;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (on && c < a.dim) {
#pragma unroll 8
    for (int s = part; s < slices; s += 32) {
      const float4 x = *reinterpret_cast<const float4*>(parts + ((int64_t)s * padded_rows + r) * tiles * 1024 + c);
      v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    }
  }
  some[part][quad] = v;
  __syncthreads();
  if (part == 0) {
    for (int i = 1; i < 32; ++i) {
      const float4 x = some[i][quad];
      v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    }
    float* to = dh + (int64_t)row[r] * a.ld_dh + c;
    const float out[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (c + q < a.dim) to[q] = on ? out[q] * a.scale : 0.f;
  }
}
__device__ __forceinline__ void put_wide(float* to, const float (&x)[4]) { *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void put_wide(__nv_bfloat16* to, const float (&x)[4]) {
  *reinterpret_cast<uint2*>(to) = make_uint2(bf162_bits(x[0], x[1]), bf162_bits(x[2], x[3]));
}
// dW of `per` rows, 1024 columns a block: a thread has its four columns of all rows of h
template <typename U, int R, bool WIDE>
__global__ void __launch_bounds__(256)
thin_dw_kernel(const float* h, int64_t ld_h, const int* row, int vocab, int dim, float scale, const LossInfo* info, const float* e, int padded, U* dw,
               int64_t ld_dw, int tiles, int per) {
  __shared__ __align__(16) float d[64][R];
  after_previous();
  const int live = info->live, tile = blockIdx.x % tiles, slice = blockIdx.x / tiles, left = dim - tile * 1024;
  const int v0 = slice * per, v1 = v0 + per < vocab ? v0 + per : vocab;
  float y[R][4];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = place<WIDE, 256>(threadIdx.x, j);
      y[r][j] = r < live && c < left ? h[(int64_t)row[r] * ld_h + tile * 1024 + c] : 0.f;
    }
  for (int vb = v0; vb < v1; vb += 64) {
    thin_rows<R>(d, e, padded, live, vb, v1);
    const int n = v1 - vb < 64 ? v1 - vb : 64;
    U* to = dw + (int64_t)vb * ld_dw + tile * 1024;
#pragma unroll 2
    for (int v = 0; v < n; ++v, to += ld_dw) {
      float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int r = 0; r < R; r += 4) {
        float f[4];
        load_wide(&d[v][r], f);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = fmaf(f[q], y[r + q][j], x[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] *= scale;
      if (WIDE) {
        if (4 * (int)threadIdx.x < left) put_wide(to + 4 * threadIdx.x, x);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if ((int)threadIdx.x + 256 * j < left) put(to + threadIdx.x + 256 * j, x[j]);
      }
    }
  }
}

// ---- host -------------------------------------------------------------------------------------
struct LossWs {
  LossInfo* info;
  int *counts, *row, *target;
  int* row_exponent;
  float *g, *target_z;
  double* part;
  float2* sums;
  unsigned short *h, *h_common, *w, *e;
  float *slab, *shares, *dw;
  int blocks, piece, padded, vpadded, sum_blocks, staged_rows;
  int dh_room, share_blocks;        // blocks of 256 x 256 sums: that dh's plan may use, and of all
  bool few;               // M_FEW
  bool thin;              // M_THIN
  bool in_place;          // W is read where it lies
};

// Columns of a tile of few rows, whose time is the vocabulary's way through memory: as even a share for every pair as
// the instructions allow, 64 at least (16 rows of 32768x2048: 147 tiles of 224 columns on 148 CTAs).
int logits_tile(int vocab, int workers) {
  const int waves = ceil_div(ceil_div(vocab, kTile), workers);
  const int n = (int)align_up((size_t)ceil_div(vocab, waves * workers), 32);
  return n < 64 ? 64 : n;
}

// K shares of dW's tiles where these are for less than half of the pairs, of eight blocks at least
int dw_shares(int tiles, int blocks_k, int pairs) {
  return 2 * tiles <= pairs && blocks_k >= 16 ? std::min(pairs / tiles, blocks_k / 8) : 1;
}
// Slices of the vocabulary, for `blocks` blocks a multiprocessor, of very few rows: rows of each
int thin_slice(int vocab, int tiles, int blocks) {
  return ceil_div(vocab, std::max(1, std::min(blocks * sm_count() / tiles, ceil_div(vocab, 16))));
}
constexpr int kThinBlocks = 4;

// aligned: the weight starts on a 16-byte boundary
size_t loss_layout(const mw_token_loss_desc* d, bool gradient, bool aligned, char* base, LossWs* l) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* p = base + at;
    at += align_up(bytes, 1024);
    return p;
  };
  const int terms = d->dtype == MW_F32 ? 2 : 1;
  const size_t n = (size_t)d->rows, v = (size_t)d->vocab, dim = (size_t)d->dim;
  const int64_t ld_w = d->ld_weight ? d->ld_weight : d->dim;
  l->few = gradient && aligned && terms == 1 && d->rows > 0 && d->rows <= kFewRows && 8 * (int64_t)d->rows <= d->dim &&
           (int64_t)d->vocab * d->dim >= kFewNumbers && ld_w % 8 == 0 && d->dim % kBK == 0;
  l->in_place = l->few || (!gradient && terms == 1 && ld_w % 8 == 0);
  l->thin = terms == 2 && d->rows > 0 && d->rows <= kThinRows;
  const int held = l->few || l->thin ? 2 : terms;          // half-precision numbers that an exponential takes
  l->blocks = ceil_div(d->rows, kIndexRows);
  l->padded = (int)align_up(dim, kBK);
  l->vpadded = (int)align_up(v, kBK);
  l->sum_blocks = ceil_div(d->vocab, kSumColumns);
  l->staged_rows = (int)align_up(n ? n : 1, kTile);
  int64_t piece = d->rows ? d->rows : 1;
  if (gradient) {
    piece = d->piece_rows;
    if (!piece) {
      piece = kPieceBytes / (2 * held * (int64_t)l->vpadded);
      if (piece < 1024) piece = 1024;
    }
    if (piece < d->rows) piece = (int64_t)align_up((size_t)piece, kTile);
    if (piece > d->rows) piece = d->rows ? d->rows : 1;
  }
  l->piece = (int)piece;
  l->info = (LossInfo*)take(sizeof(LossInfo));
  l->counts = (int*)take((size_t)l->blocks * 4);
  l->row = (int*)take(n * 4);
  l->target = (int*)take(n * 4);
  l->g = (float*)take(n * 4);
  l->target_z = (float*)take(n * 4);
  l->part = (double*)take(n * 8);
  // (few rows have blocks of 32 columns and more)
  l->sums = (float2*)take((size_t)l->piece * (n <= kTile ? ceil_div(d->vocab, 32) : l->sum_blocks) * 8);
  l->h = (unsigned short*)take(l->thin ? 0 : (size_t)l->staged_rows * l->padded * 2 * terms);
  l->h_common = (unsigned short*)take(gradient && !l->thin && !l->few ? (size_t)l->staged_rows * l->padded * 2 * terms : 0);
  l->row_exponent = (int*)take(n * 4);
  l->w = (unsigned short*)take(l->in_place || l->thin ? 0 : v * l->padded * 2 * terms);
  l->e = (unsigned short*)take(gradient ? (size_t)l->piece * l->vpadded * 2 * held : 0);
  l->slab = (float*)take(gradient ? (size_t)l->piece * l->padded * 4 : 0);
  l->dh_room = l->share_blocks = 0;
  if (l->thin) {
    const int tiles = ceil_div(d->dim, 1024), slices = ceil_div(d->vocab, thin_slice(d->vocab, tiles, kThinBlocks));
    l->share_blocks = ceil_div((int64_t)slices * tiles * 1024 * (d->rows <= 4 ? 4 : kThinRows), kTile * kTile);
  } else if (gradient) {
    // the most that the plan of dh may want: tiles beside the whole waves, times shares of eight blocks of K and more
    const int pairs = sm_count() / 2, workers = d->rows <= kHalf ? sm_count() : pairs, across = ceil_div(d->dim, kTile);
    const int64_t rest = std::min((int64_t)ceil_div(l->piece, kTile) * across, (int64_t)workers - 1);
    const int most_shares = std::min(32, std::max(1, (l->vpadded / kBK - 1) / 7));
    l->dh_room = (int)std::min((int64_t)share_blocks(pairs), rest * most_shares);
    const int tiles = ceil_div(d->vocab, kTile) * across, shares = dw_shares(tiles, ceil_div(l->piece, kBK), pairs);
    const int held = (int)std::min((int64_t)l->dh_room, rest * (most_shares - 1));          // (a tile's first share has its own place)
    l->share_blocks = std::max(std::max(1, held), shares > 1 ? tiles * shares : 0);
  }
  l->shares = (float*)take(gradient ? (size_t)l->share_blocks * kTile * kTile * 4 : 0);
  l->dw = (float*)take(gradient && l->piece < d->rows ? v * l->padded * 4 : 0);
  return at;
}

mw_status check_loss(const mw_token_loss_desc* d) {
  if (!d || d->rows < 0 || d->vocab < 1 || d->dim < 1 || d->piece_rows < 0 || !isfinite((float)d->scale)) return MW_ERR_INVALID_ARG;
  if (d->index_bytes != 4 && d->index_bytes != 8) return MW_ERR_INVALID_ARG;
  if (d->rows > (1 << 24) || d->vocab > (1 << 24) || d->dim > (1 << 16) || d->dtype == MW_F64) return MW_ERR_UNSUPPORTED;
  if (d->dtype != MW_F32 && d->dtype != MW_BF16_F32ACC) return MW_ERR_INVALID_ARG;
  if (d->grad_dtype != 0 && d->grad_dtype != MW_F32 && d->grad_dtype != MW_BF16_F32ACC) return MW_ERR_INVALID_ARG;
  for (int64_t ld : {d->ld_h, d->ld_weight, d->ld_dh, d->ld_dweight})
    if (ld != 0 && ld < d->dim) return MW_ERR_INVALID_ARG;
  // (tiles are counted in 32 bits)
  if ((d->rows / kTile + 1) * (d->vocab / 64 + 1) > (1 << 30)) return MW_ERR_UNSUPPORTED;
  return MW_OK;
}

// a tensor map of `rank` dimensions; strides in bytes, of all but the first
mw_status make_map(CUtensorMap* out, CUtensorMapDataType type, int rank, const void* base, const int64_t* dims, const int64_t* strides,
                   const int* box) {
  auto fn = encode_fn();
  if (!fn) return MW_ERR_CUDA;
  cuuint64_t d[4], st[3];
  cuuint32_t b[4], one[4] = {1u, 1u, 1u, 1u};
  for (int i = 0; i < rank; ++i) {
    d[i] = (cuuint64_t)dims[i];
    b[i] = (cuuint32_t)box[i];
    if (i) st[i - 1] = (cuuint64_t)strides[i - 1];
  }
  return fn(out, type, (cuuint32_t)rank, const_cast<void*>(base), d, st, b, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? MW_OK : MW_ERR_CUDA;
}
// operand rows with K along them: boxes of 64 columns, 128 rows and all terms
mw_status row_map(CUtensorMap* out, bool bf16, const void* base, int64_t cols, int64_t rows, int64_t ld, int terms, int box_rows) {
  const int64_t dims[3] = {cols, rows, terms}, strides[2] = {ld * 2, rows * ld * 2};
  const int box[3] = {kBK, box_rows, terms};
  return make_map(out, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, base, dims, strides, box);
}
// operand rows in groups of 64 columns: boxes of `rows_box` rows and `groups` groups
mw_status group_map(CUtensorMap* out, const void* base, int64_t cols, int64_t rows, int64_t row_bytes, int64_t group_bytes,
                    int64_t term_bytes, int terms, int rows_box, int groups) {
  const int64_t dims[4] = {64, rows, cols / 64, terms}, strides[3] = {row_bytes, group_bytes, term_bytes};
  const int box[4] = {64, rows_box, groups, terms};
  return make_map(out, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, base, dims, strides, box);
}
// results: boxes of 32 rows of 128 bytes
mw_status out_map(CUtensorMap* out, CUtensorMapDataType type, int size, const void* base, int64_t cols, int64_t rows, int64_t ld) {
  const int64_t dims[2] = {cols, rows}, strides[1] = {ld * size};
  const int box[2] = {128 / size, 32};
  return make_map(out, type, 2, base, dims, strides, box);
}

template <int MODE, int KIND, bool PAIR>
mw_status run_product_in(ProductArgs& p, int64_t most_units, cudaStream_t s) {
  // (A of few rows is short; dW's rows are the vocabulary's)
  p.a_term = KIND == P_DW ? kPlaneBytes : (uint32_t)p.a_rows * (kBK * 2);
  p.a_stage = terms_a(MODE, KIND) * p.a_term;
  p.buffers = buffers_for(MODE, KIND, p.blocks_k);
  p.most_blocks = piece_blocks(MODE, KIND, p.piece);
  p.stages = stages_for(p.buffers, p.a_stage + terms_b(MODE) * plane_b(PAIR));
  p.wait_ns = unmet_ms ? unmet_ms * 1000000ull : kLossWaitNs;
  p.unmet = unmet_ms != 0 && unmet_product == (of_logits(KIND) ? 0 : (KIND == P_DH ? 1 : 2));
  static bool ready[kMaxDevices] = {};
  const int dev = current_device();
  auto kernel = loss_products_kernel<MODE, KIND, PAIR>;
  if (!ready[dev]) {
    MW_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost));
    ready[dev] = true;
  }
  const int64_t each = PAIR ? 2 : 1, workers = sm_count() / each;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(each * (most_units < workers ? (most_units < 1 ? 1 : most_units) : workers)));
  cfg.blockDim = dim3(kLossThreads);
  cfg.dynamicSmemBytes = kSmemMost;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = PAIR ? 2 : 1;
  ++g_launch_count;
  return cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess ? MW_OK : MW_ERR_CUDA;
}

template <int TERMS, int KIND>
mw_status run_product(bool few, bool single, ProductArgs& p, int64_t most_units, cudaStream_t s) {
  constexpr int kMode = TERMS == 2 ? M_TWO : M_ONE;
  if constexpr (KIND == P_DW) {
    if constexpr (TERMS == 1)
      if (few) return run_product_in<M_FEW, KIND, true>(p, most_units, s);
    return run_product_in<kMode, KIND, true>(p, most_units, s);
  } else {
    if constexpr (TERMS == 1 && KIND != P_SUMS)
      if (few) return run_product_in<M_FEW, KIND, false>(p, most_units, s);
    return single ? run_product_in<kMode, KIND, false>(p, most_units, s) : run_product_in<kMode, KIND, true>(p, most_units, s);
  }
}

// fp32 accumulator, the operands' type, K across the rows of A and of B, N / 8, M / 16
uint32_t instruction(bool bf16, bool turned_a, bool turned_b, int m = kTile, int n = kTile) {
  return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((turned_a ? 1u : 0u) << 15) | ((turned_b ? 1u : 0u) << 16) |
         ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// The calls of very few rows.  (dW before dh, which may take h's place.)
template <int R>
mw_status thin_run_of(const LossArgs& a, const LossWs& l, const float* h, const float* w, const void* targets, int index_bytes, float* loss, float* total, float* dh,
                      void* dw, bool dw_bf16, bool gradient, cudaStream_t s) {
  auto wide = [&](const void* p, int64_t ld, int size) { return ((uintptr_t)p & (uintptr_t)(4 * size - 1)) == 0 && ld % 4 == 0 && a.dim % 4 == 0; };
  const bool wide_w = wide(w, a.ld_w, 4);
  const int sums = ceil_div(a.vocab, kThinColumns), most = (int)(192 * 1024 / (4 * R)), chunk = std::min((int)align_up((size_t)a.dim, 128), most / 128 * 128);
  auto logits = wide_w ? thin_logits_kernel<R, true> : thin_logits_kernel<R, false>;
  const size_t smem = (size_t)R * chunk * 4;
  MW_CUDA_OK(cudaFuncSetAttribute(logits, cudaFuncAttributeMaxDynamicSharedMemorySize, 192 * 1024));
  MW_TRY(launch_after(logits, (unsigned)std::min(sums, sm_count()), 512, smem, s, h, a.ld_h, w, a.ld_w, (int)a.rows, a.vocab, a.dim, chunk,
                      (float)((double)a.scale * 1.4426950408889634), l.info, gradient ? l.row : nullptr, l.target, targets, index_bytes, l.sums, sums,
                      l.target_z, gradient ? (float*)l.e : nullptr, l.vpadded));
  if (!gradient) return MW_OK;
  const int slices = std::min(2 * sm_count() / (int)a.rows, ceil_div(l.vpadded, 4096));
  MW_TRY(launch_after(dz_kernel<M_THIN, 8>, (unsigned)(a.rows * slices), 256, 0, s, l.info, 0, (int)a.rows, l.sums, sums, l.target_z, l.row, l.target, l.g,
                      loss, l.part, total, l.e, l.vpadded, slices));
  // slices of the vocabulary for as many blocks as the device holds a few times over
  const int tiles = ceil_div(a.dim, 1024);
  if (dw) {
    const int per = thin_slice(a.vocab, tiles, kThinBlocks), n = ceil_div(a.vocab, per) * tiles;
    auto go = [&](auto kernel, auto* to) { return launch_after(kernel, (unsigned)n, 256, 0, s, h, a.ld_h, l.row, a.vocab, a.dim, a.scale, l.info, (const float*)l.e,
                                                               l.vpadded, to, a.ld_dw, tiles, per); };
    if (dw_bf16) MW_TRY(go(wide(dw, a.ld_dw, 2) ? thin_dw_kernel<__nv_bfloat16, R, true> : thin_dw_kernel<__nv_bfloat16, R, false>, (__nv_bfloat16*)dw));
    else MW_TRY(go(wide(dw, a.ld_dw, 4) ? thin_dw_kernel<float, R, true> : thin_dw_kernel<float, R, false>, (float*)dw));
  }
  if (dh) {
    const int per = thin_slice(a.vocab, tiles, kThinBlocks), n = ceil_div(a.vocab, per);
    MW_TRY(launch_after(wide_w ? thin_dh_kernel<R, true> : thin_dh_kernel<R, false>, (unsigned)(n * tiles), 256, 0, s, w, a.ld_w, a.vocab, a.dim, l.info,
                        (const float*)l.e, l.vpadded, l.shares, tiles, per));
    MW_TRY(launch_after(thin_dh_rows_kernel, dim3((unsigned)ceil_div(a.dim, 32), (unsigned)a.rows), 256, 0, s, a, l.shares, tiles, R, n, l.row, l.info, dh));
  }
  return MW_OK;
}

template <typename T, typename I>
mw_status loss_run(const mw_token_loss_desc* d, const T* h, const T* w, const I* targets, const float* weight, float* loss, float* total,
                   T* dh, void* dw, bool gradient, char* ws, cudaStream_t s) {
  constexpr int TERMS = sizeof(T) == 4 ? 2 : 1;
  LossArgs a;
  a.rows = d->rows; a.vocab = d->vocab; a.dim = d->dim;
  a.ld_h = d->ld_h ? d->ld_h : d->dim;
  a.ld_w = d->ld_weight ? d->ld_weight : d->dim;
  a.ld_dh = d->ld_dh ? d->ld_dh : d->dim;
  a.ld_dw = d->ld_dweight ? d->ld_dweight : d->dim;
  a.scale = (float)d->scale;
  LossWs l;
  loss_layout(d, gradient, ((uintptr_t)w & 15) == 0, ws, &l);
  // bf16 operands of the loss alone, and of few rows, are taken as they are
  const bool scaled = TERMS == 2 || (gradient && !l.few);
  const int mode = TERMS == 2 ? M_TWO : (l.few ? M_FEW : M_ONE);
  a.scaled = scaled;
  const unsigned wide = 148 * 8;
  // few rows of the loss alone: no row is moved where the copy engine can read h as it lies
  const bool direct = l.in_place && !gradient && a.rows > 0 && a.rows <= kTile && a.ld_h % 8 == 0 && ((uintptr_t)h & 15) == 0;
  if constexpr (TERMS == 2) {
    if (l.thin) {
      if (gradient) MW_TRY(launch_after(index_live_kernel<I>, 1, kIndexRows, 0, s, targets, weight, a.rows, a.vocab, (int*)nullptr, 1, l.row, l.target, l.g, loss, l.info));
      auto run = a.rows <= 4 ? thin_run_of<4> : thin_run_of<8>;
      const bool dw_bf16 = (d->grad_dtype ? d->grad_dtype : d->dtype) == MW_BF16_F32ACC;
      MW_TRY(run(a, l, h, w, targets, (int)sizeof(I), loss, total, dh, dw, dw_bf16, gradient, s));
      if (gradient) return MW_OK;
      return launch_after(direct_rows_kernel<I>, 1, 256, 0, s, l.info, l.sums, ceil_div(a.vocab, kThinColumns), kThinColumns, l.target_z, targets, weight, (int)a.rows,
                          a.vocab, loss, l.part, total);
    }
  }
  if (l.blocks != 1) MW_CUDA_OK(cudaMemsetAsync(ws, 0, sizeof(LossInfo), s));
  if (a.rows > 0 && !direct) {
    int* counts = l.blocks > 1 ? l.counts : nullptr;
    if (counts) MW_TRY(launch_after(count_live_kernel<I>, l.blocks, kIndexRows, 0, s, targets, weight, a.rows, a.vocab, counts));
    MW_TRY(launch_after(index_live_kernel<I>, l.blocks, kIndexRows, 0, s, targets, weight, a.rows, a.vocab, counts, l.blocks, l.row, l.target, l.g, loss, l.info));
    Operands<T> o = {w, h, a.ld_w, a.ld_h, l.w, l.h, scaled && dw ? l.h_common : nullptr, l.row, l.g, l.row_exponent, l.in_place ? 0 : a.vocab, a.dim, l.padded,
                     (int)a.rows, l.staged_rows, dh, a.ld_dh, l.info, 0, 0};
    auto aligned = [&](const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld * (int64_t)sizeof(T) % 16 == 0; };
    const bool rows16 = aligned(h, a.ld_h) && aligned(w, a.ld_w) && a.dim * (int64_t)sizeof(T) % 16 == 0;
    // a warp a row of h, a quarter of one a short row (16384 rows of 64: 5.2 us, by warps 12.4), a block a long one
    // (1003 rows of 515 fp32 are no faster by blocks: 10.9 us, by warps 9.3)
    o.row_threads = l.padded <= (rows16 ? 256 : 64) ? 8 : (l.padded <= 2048 ? 32 : 256);
    // blocks by the operands' shares of the work, eight a multiprocessor at the most of either
    const int64_t most = 8 * (int64_t)sm_count(), want_w = ((int64_t)o.vocab * (l.padded / 8) + 511) / 512, want_h = ceil_div(a.rows + kTile, 256 / o.row_threads);
    const int64_t bw = std::min(want_w, most), bh = std::min(want_h, most);
    auto stage = [&](auto kernel, int64_t nw, int64_t nh) {
      o.w_blocks = nw;
      return launch_after(kernel, (unsigned)(nw + nh), 256, 0, s, o);
    };
    if (scaled) {
      // (the second seldom has anything to do: two blocks a multiprocessor see to that sooner than eight)
      const int64_t few = 2 * (int64_t)sm_count();
      MW_TRY(stage(rows16 ? stage_kernel<T, TERMS, true, true, false> : stage_kernel<T, TERMS, true, false, false>, bw, bh));
      MW_TRY(stage(rows16 ? stage_kernel<T, TERMS, true, true, true> : stage_kernel<T, TERMS, true, false, true>, std::min(bw, few), std::min(bh, few)));
    } else {
      MW_TRY(stage(rows16 ? stage_kernel<T, 1, false, true, false> : stage_kernel<T, 1, false, false, false>, bw, bh));
    }
  }
  if (a.rows > 0 || dw) {
    const bool bf16 = !scaled;
    const int dw_bf16 = (d->grad_dtype ? d->grad_dtype : d->dtype) == MW_BF16_F32ACC;
    const int dw_size = dw_bf16 ? 2 : 4;
    ProductArgs p = {};
    p.info = l.info;
    p.st = &l.info->st;
    p.total = total;
    p.vocab = a.vocab; p.dim = a.dim;
    p.scale = a.scale; p.scaled = scaled;
    p.piece = l.piece;
    p.sum_blocks = l.sum_blocks;
    p.sums = l.sums; p.target_z = l.target_z; p.target = l.target;
    p.row_exponent = scaled ? l.row_exponent : nullptr;
    // (few rows: CTAs of their own)
    const bool single = a.rows <= kHalf;
    const int pairs = sm_count() / 2, tile_m = single ? kHalf : kTile;
    p.workers = single ? sm_count() : pairs;
    p.share_room = l.dh_room;
    p.shares = 1;
    p.tile_n = kTile;
    ProductArgs logits = p, by_h = p, by_w = p;
    logits.direct = direct;
    logits.clear = l.info;
    logits.targets = targets;
    logits.index_bytes = (int)sizeof(I);
    if (direct) logits.tile_n = logits_tile(a.vocab, p.workers);
    logits.tiles_n = ceil_div(a.vocab, logits.tile_n);
    logits.sum_blocks = ceil_div(a.vocab, logits.tile_n / 2);
    logits.blocks_k = l.padded / kBK;
    const int64_t held = kHeldBytes / ((int64_t)kTile * l.padded * 2 * TERMS);
    logits.group_rows = held < 8 ? 8 : (int)held;
    logits.idesc = instruction(bf16, false, false, tile_m, logits.tile_n);
    // Few rows: only theirs are copied, the others' products come out as whatever they are and are not read.
    logits.a_rows = by_h.a_rows = !single ? kHalf : (a.rows <= 16 ? 16 : (a.rows <= 32 ? 32 : (a.rows <= 64 ? 64 : kHalf)));
    const int share_b = single ? kTile : kHalf;          // of a tile's columns in a CTA
    MW_TRY(direct ? row_map(&logits.a, bf16, h, a.dim, a.rows, a.ld_h, 1, logits.a_rows) : row_map(&logits.a, bf16, l.h, l.padded, l.staged_rows, l.padded, TERMS, logits.a_rows));
    MW_TRY(l.in_place ? row_map(&logits.b, bf16, w, a.dim, a.vocab, a.ld_w, 1, logits.tile_n * share_b / kTile)
                      : row_map(&logits.b, bf16, l.w, l.padded, a.vocab, l.padded, TERMS, share_b));
    if (gradient) {
      // an exponential's place, and that of dz's terms: groups of 64, one term after the other
      const int held = l.few ? 2 : TERMS;
      const int64_t row_bytes = (int64_t)l.vpadded * 2 * held, group_bytes = 128 * held, hw_bytes = (int64_t)l.padded * 2;
      MW_TRY(out_map(&logits.out, held == 1 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2 * held, l.e, l.vpadded, l.piece, l.vpadded));
      // dh: K along the rows of dz and across those of W
      by_h.tiles_n = ceil_div(a.dim, kTile);
      by_h.blocks_k = l.vpadded / kBK;
      by_h.idesc = instruction(bf16, false, true, tile_m);
      MW_TRY(group_map(&by_h.a, l.e, l.vpadded, l.piece, row_bytes, group_bytes, 128, held, by_h.a_rows, 1));
      MW_TRY(l.few ? group_map(&by_h.b, w, a.dim, a.vocab, a.ld_w * 2, 128, 128, 1, kBK, share_b / 64)
                   : group_map(&by_h.b, l.w, l.padded, a.vocab, hw_bytes, 128, hw_bytes * a.vocab, TERMS, kBK, share_b / 64));
      MW_TRY(out_map(&by_h.out, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, l.slab, l.padded, l.piece, l.padded));
      MW_TRY(out_map(&by_h.acc, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, l.shares, kTile, (int64_t)l.share_blocks * kTile, kTile));
      // dW: K across the rows of both
      by_w.tiles_m = ceil_div(a.vocab, kTile);
      by_w.tiles_n = ceil_div(a.dim, kTile);
      by_w.blocks_k = ceil_div(l.piece, kBK);
      by_w.idesc = instruction(bf16, true, true);
      MW_TRY(group_map(&by_w.a, l.e, l.vpadded, l.piece, row_bytes, group_bytes, 128, held, kBK, 2));
      MW_TRY(group_map(&by_w.b, l.h, l.padded, l.staged_rows, hw_bytes, 128, hw_bytes * l.staged_rows, TERMS, kBK, 2));
      if (scaled) MW_TRY(group_map(&by_w.b_common, l.h_common, l.padded, l.staged_rows, hw_bytes, 128, hw_bytes * l.staged_rows, TERMS, kBK, 2));
      by_w.shares = dw_shares(by_w.tiles_m * by_w.tiles_n, by_w.blocks_k, pairs);
      if (by_w.shares > 1) by_w.out = by_w.acc = by_h.acc;
      by_w.dw = dw; by_w.ld_dw = a.ld_dw; by_w.dw_bf16 = dw_bf16;
      // (the copy engine ends a row at 16 bytes, which may lie beyond its last column)
      by_w.dw_engine = by_w.shares == 1 && ((uintptr_t)dw & 15) == 0 && (a.ld_dw * dw_size) % 16 == 0 && (int64_t)a.dim * dw_size % 16 == 0;
      if (by_w.dw_engine && dw)
        MW_TRY(out_map(&by_w.out, dw_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, dw_size, dw, a.dim, a.vocab, a.ld_dw));
      by_w.partial = l.dw; by_w.ld_partial = l.padded;
      if (l.piece < a.rows && by_w.shares == 1) MW_TRY(out_map(&by_w.acc, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, l.dw, l.padded, a.vocab, l.padded));
    }
    const int64_t tm = ceil_div(l.piece, kTile);
    for (int64_t first = 0; first < (a.rows > 0 ? a.rows : 1); first += l.piece) {
      logits.first = by_h.first = by_w.first = (int)first;
      if (a.rows > 0) {
        if (gradient) {
          MW_TRY((run_product<TERMS, P_EXP>(l.few, single, logits, tm * logits.tiles_n, s)));
          // A warp a row of up to 4096 logits, a block a longer one (9234 rows of 2882, a block each: 51 us, most of
          // them waits of one row after another), several where rows are few (1 of 66235: 24 us, 10 in 17)
          const bool short_rows = a.vocab <= 4096 && l.piece > 2 * sm_count();
          const int most = 2 * sm_count() / l.piece, parts = ceil_div(l.vpadded, TERMS == 2 || l.few ? 4096 : 8192);
          const int slices = short_rows || most < 2 ? 1 : (most < parts ? most : parts);
          const int dz_blocks = short_rows ? ceil_div(l.piece, 8) : l.piece * slices;
          constexpr int kMode = TERMS == 2 ? M_TWO : M_ONE, kOther = TERMS == 2 ? M_TWO : M_FEW;
          auto dz = l.few ? (short_rows ? dz_kernel<kOther, 1> : dz_kernel<kOther, 8>) : (short_rows ? dz_kernel<kMode, 1> : dz_kernel<kMode, 8>);
          MW_TRY(launch_after(dz, (unsigned)(dz_blocks < (int)wide ? dz_blocks : wide), 256, 0, s,
                              l.info, (int)first, l.piece, l.sums, l.sum_blocks, l.target_z, l.row, l.target, l.g, loss, l.part,
                              first + l.piece >= a.rows ? total : nullptr, l.e, l.vpadded, slices));
        } else {
          MW_TRY((run_product<TERMS, P_SUMS>(false, single, logits, tm * logits.tiles_n, s)));
          const unsigned blocks = (unsigned)(a.rows < wide * 8 ? ceil_div(a.rows, 8) : wide);          // (a warp a row)
          if (direct)
            MW_TRY(launch_after(direct_rows_kernel<I>, blocks, 256, 0, s, l.info, l.sums, logits.sum_blocks, logits.tile_n / 2, l.target_z, targets, weight, (int)a.rows,
                                a.vocab, loss, l.part, total));
          else
            MW_TRY(launch_after(loss_rows_kernel, blocks, 256, 0, s, l.info, l.sums, l.sum_blocks, l.target_z, l.row, l.target, l.g, loss, l.part,
                                total));
        }
        if (dh) {
          MW_TRY((run_product<TERMS, P_DH>(l.few, single, by_h, p.workers, s)));
          auto rows_kernel = ((uintptr_t)dh & 15) == 0 && a.ld_dh % 4 == 0 && a.dim % 4 == 0 ? dh_rows_kernel<T, true> : dh_rows_kernel<T, false>;
          MW_TRY(launch_after(rows_kernel, wide, 256, 0, s, a, l.slab, l.shares, l.padded, by_h.tiles_n, by_h.blocks_k, p.workers, p.share_room, mode, (int)first, l.piece,
                              l.row, l.g, l.info, dh));
        }
      }
      if (dw) {
        MW_TRY((run_product<TERMS, P_DW>(l.few, false, by_w, (int64_t)by_w.tiles_m * by_w.tiles_n * by_w.shares, s)));
        if (by_w.shares > 1) {
          if (dw_bf16)
            MW_TRY(launch_after(dw_rows_kernel<__nv_bfloat16>, wide, 256, 0, s, a, l.shares, by_w.tiles_n, by_w.shares, mode, (int)first, l.piece,
                                l.info, l.dw, l.padded, (__nv_bfloat16*)dw));
          else
            MW_TRY(launch_after(dw_rows_kernel<float>, wide, 256, 0, s, a, l.shares, by_w.tiles_n, by_w.shares, mode, (int)first, l.piece, l.info,
                                l.dw, l.padded, (float*)dw));
        }
      }
    }
  }
  if (total && a.rows == 0) MW_CUDA_OK(cudaMemsetAsync(total, 0, 4, s));
  return MW_OK;
}

mw_status loss_call(const mw_token_loss_desc* d, const void* h, const void* w, const void* targets, const float* weight, float* loss,
                    float* total, void* dh, void* dw, bool gradient, void* ws, size_t bytes, void* stream) {
  MW_TRY(check_loss(d));
  if (!w || (d->rows > 0 && (!h || !targets || !loss))) return MW_ERR_INVALID_ARG;
  const int64_t ld_h = d->ld_h ? d->ld_h : d->dim, ld_dh = d->ld_dh ? d->ld_dh : d->dim;
  if (dh == h && dh && ld_h != ld_dh) return MW_ERR_INVALID_ARG;
  // rows that the copy engine reads start on 16-byte boundaries (the gradient copies a weight that does not)
  const bool aligned = ((uintptr_t)w & 15) == 0;
  LossWs l;
  const size_t need = loss_layout(d, gradient, aligned, nullptr, &l);
  if (l.in_place && !aligned) return MW_ERR_INVALID_ARG;
  if (!ws || ((uintptr_t)ws & 255u) || bytes < need) return MW_ERR_WORKSPACE;
  // (dh is formed when h has been read, and either gradient may come first)
  if ((dw && (dw == w || dw == h || dw == dh)) || (dh && dh == w)) return MW_ERR_INVALID_ARG;
  cudaStream_t s = (cudaStream_t)stream;
  char* b = static_cast<char*>(ws);
  using bf = __nv_bfloat16;
  if (d->dtype == MW_F32) {
    if (d->index_bytes == 4) return loss_run<float, int32_t>(d, (const float*)h, (const float*)w, (const int32_t*)targets, weight, loss, total, (float*)dh, dw, gradient, b, s);
    return loss_run<float, int64_t>(d, (const float*)h, (const float*)w, (const int64_t*)targets, weight, loss, total, (float*)dh, dw, gradient, b, s);
  }
  if (d->index_bytes == 4) return loss_run<bf, int32_t>(d, (const bf*)h, (const bf*)w, (const int32_t*)targets, weight, loss, total, (bf*)dh, dw, gradient, b, s);
  return loss_run<bf, int64_t>(d, (const bf*)h, (const bf*)w, (const int64_t*)targets, weight, loss, total, (bf*)dh, dw, gradient, b, s);
}

}  // namespace
}  // namespace mw

extern "C" mw_status mw_token_loss_workspace_bytes(const mw_token_loss_desc* desc, int32_t gradient, size_t* bytes) {
  using namespace mw;
  if (!bytes || (gradient != 0 && gradient != 1)) return MW_ERR_INVALID_ARG;
  MW_TRY(check_loss(desc));
  LossWs l;
  *bytes = std::max(loss_layout(desc, gradient != 0, true, nullptr, &l), loss_layout(desc, gradient != 0, false, nullptr, &l));
  return MW_OK;
}

extern "C" mw_status mw_token_loss_forward(const mw_token_loss_desc* desc, const void* h, const void* weight, const void* targets,
                                           const float* row_weight, float* loss, float* total, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  return mw::loss_call(desc, h, weight, targets, row_weight, loss, total, nullptr, nullptr, false, workspace, workspace_bytes, stream);
}

extern "C" mw_status mw_token_loss_gradient(const mw_token_loss_desc* desc, const void* h, const void* weight, const void* targets,
                                            const float* row_weight, float* loss, float* total, void* dh, void* dweight,
                                            void* workspace, size_t workspace_bytes, void* stream) {
  return mw::loss_call(desc, h, weight, targets, row_weight, loss, total, dh, dweight, true, workspace, workspace_bytes, stream);
}

extern "C" mw_status mw_token_loss_status(const void* workspace, void* stream) {
  using namespace mw;
  if (!workspace) return MW_ERR_INVALID_ARG;
  DeviceStatus host;
  MW_CUDA_OK(cudaMemcpyAsync(&host, workspace, sizeof(host), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
  MW_CUDA_OK(cudaStreamSynchronize((cudaStream_t)stream));
  return (mw_status)host.code;
}

extern "C" mw_status mw_token_loss_selftest_unmet_wait(uint32_t limit_ms, int32_t product) {
  if (limit_ms > 1000 || product < 0 || product > 2) return MW_ERR_INVALID_ARG;
  mw::unmet_ms = limit_ms;
  mw::unmet_product = product;
  return MW_OK;
}
