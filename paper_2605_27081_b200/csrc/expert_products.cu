// The experts' products over rows sorted by expert, forward and backward, on the tensor cores.
//
// Every product is O[n, m] = sum_k M[m, k] N[n, k] over tiles of 256 x up to 256, computed by a pair of CTAs on two
// neighbouring SMs (tcgen05.mma with cta_group::2: each CTA stages 128 rows of M and half of the rows of N and keeps its 128 rows
// of the fp32 result in TMEM, a lane for each m).  The side that belongs to the weights is M, so that the ragged side, the rows of an
// expert, is N, whose width the instruction takes in steps of 32 columns:
//   kGateUp      m = channel (gate and up), n = row, k = hidden:              act = silu(g) u
//   kDown        m = hidden,  n = row, k = channel:                           ys = act W_down
//   kGradAct     m = channel, n = row, k = hidden:    d act = d_ys W_down^T;  d g, d u, act by the derivative of silu(g) u
//   kGradRows    m = hidden,  n = row, k = channel of d g, then of d u:       d_xs = d_g W_gate + d_u W_up
//   kGradBlocks  m = channel, n = hidden, k = row:    d W = (d g)^T xs, (d u)^T xs, act^T d_ys, one plane of a block each
// Operands come through tensor maps straight from where the caller keeps them: K-major tiles (k contiguous) are [128 rows x 64],
// MN-major ones two [64 x 64] boxes with k as the rows; both are the 128-byte-swizzled images the tensor cores read.
// Per CTA: warp 0 loads (TMA, a ring of stages of 64 k, 32 KB), warp 1 of the pair's even CTA issues the products, warps 4-7 and 8-11 read the
// results out of TMEM (two buffers of 256 columns, so that a tile's epilogue runs behind the next tile's products; every other group of columns
// for each four, so that a tile alone is out sooner).  With k = row (kGradBlocks) an expert's last rows end inside a stage; what follows them there (the next expert's rows, or memory that nobody has
// written) would enter the sums, so warp 2 stands between the copies of such a stage and the products and clears it in both operands, up to the
// sixteen rows of an instruction.
// The epilogue turns its 8 x 8 pieces over on the way through shared memory (TMEM in the layout of matrix fragments, stmatrix.trans) and
// leaves by TMA stores of 16 or 32 rows x 64 values; only the columns of an expert's last, incomplete group of rows leave by plain stores,
// since a copy would run over the next expert's first rows.  kGradBlocks has the rows of its output as lanes and copies boxes of 16 rows x 64
// columns, which the tensor map ends at the block's channels and columns, each warp on its own.  (Straight from the registers, 32 bytes of 32 rows a
// store, the gradient of 64 blocks of 1408 x 2048 from 24576 rows took 435 us instead of 403: as many requests as sectors.  128 bytes of eight rows a
// store, turned over by shuffles: 3 % slower for it, and 8 % for blocks of few rows.)  kGradAct's kept gates and ups come in the same way, by warps 2 and 3.
// Where a launch has few tiles of a long k (a shared expert, a few rows), up to four pairs, a cluster, take a part of a tile's k each.  When all have
// ended, each sends the others its sums of their columns, into the rings, which are idle by then, and finishes columns of its own: the order of the
// sums is the same in every run.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cstdlib>
#include <cstring>

#include "expert_host.h"
#include "tma_ring.cuh"

namespace remoe {
namespace {

using namespace ring;

enum Mode { kGateUp, kDown, kGradAct, kGradRows, kGradBlocks };

constexpr int kTile = 256;                               // rows of M and most rows of N of a pair's tile
constexpr int kK = 64;                                   // k of a stage: 128 bytes
constexpr int kOperandBytes = 128 * 128;                 // a CTA's half of an operand's stage
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kThreads = 384;
constexpr uint32_t kTmemCols = 512;
// Polls of a bounded wait, of 2900 clocks each (measured on a barrier that never completes: 1.5 us, so 0.4 s); and more of them for a wait that may last
// for whole tiles, by the pieces of 64 k in them: 24 us a piece, which takes 0.3 to 0.8.
constexpr unsigned kPolls = 1u << 18, kPiecePolls = 16;
constexpr int kBoxes = 5;
// Rows of N in one copy: 16, 32, 64, 96, 128.
__host__ __device__ constexpr int box_rows(int b) { return b == 0 ? 16 : b == 1 ? 32 : 32 * b; }

// Shared memory: ring, then the buffers of the two epilogues, each of kCols columns of the result.
template <int MODE>
struct Shape {
  static constexpr int kStages = MODE == kGradAct ? 5 : 6;
  static constexpr int kCols = MODE == kGradAct ? 16 : 32;
  static constexpr int kBuffer = MODE == kGradBlocks ? 4 * 2048 : MODE == kDown || MODE == kGradRows ? 8192 : 12288;  // the others: three outputs
  static constexpr int kKept = MODE == kGradAct ? 2 * 8192 : 0;        // kept gates and ups: two groups of columns
  static constexpr int kStaging = 2 * (kBuffer + kKept);
  static constexpr int kBarriers = 3 * kStages + 2 + 2 + 1 + 2 * 4;
  static constexpr size_t kFixed = 1024 + (size_t)kStages * kStageBytes + kStaging + 8 * kBarriers + 8;
  static constexpr size_t smem(int n_experts) { return kFixed + (size_t)(2 * n_experts + 2) * 4; }
  static_assert(smem(REMOE_SORT_MAX_EXPERTS) <= 227 * 1024, "shared memory of a CTA");
};

struct ProductArgs {
  CUtensorMap m;                                         // M: blocks; kGradBlocks: d g, d u, act
  CUtensorMap n[kBoxes];                                 // N: boxes of box_rows; kGradBlocks: xs, d_ys, boxes of 64
  const int* offsets;
  int n_experts, n_rows, H, I;
  CUtensorMap gate_up;                                   // kGradAct: [2, n_rows, I], boxes of 16 rows
  CUtensorMap o[2];                                      // outputs (kGateUp: act, the kept gates and ups), boxes of kCols rows
  uint16_t* out;                                         // rows or blocks; kGateUp, kGradAct: [.., n_rows, I]
  uint16_t* kept;                                        // kGateUp: [2, n_rows, I] or null
  int64_t out_stride, block_stride;                      // elements between rows, between blocks
  int parts;                                             // pairs that share a tile's k; more than one: a tile at most for a cluster
  unsigned polls;                                        // of a bounded wait
  int lose;                                              // failure-detection test aid (Lost): the first pair's waits are for a copy more than it issues
};
enum Lost { kNone, kOperand, kKeptValues };              // a piece of an operand; kGradAct: of kept gates and ups

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// One lane of a converged warp.  The roles that issue copies and products run with whole warps and take a lane only around the instructions
// themselves: their operands then lie in uniform registers, as the instructions want them.  (With the loop itself in one lane an
// MMA took 67 cycles to issue and a commit 150: for a stage of 128 k, as it was then, more than the 512 that its eight products run for.)
__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
}
// Products of one call follow one another by programmatic launch: the next kernel's CTAs come up, and load what does not depend on
// the kernel before, as soon as SMs are free; dependency_wait() returns when that kernel has completed.
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address of a CTA's copy of a shared variable.
__device__ __forceinline__ uint32_t in_cta(const void* p, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void send(uint32_t at, const float* v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void expect_tx_at(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Loads of this CTA's own shared memory; completion is counted on a barrier of either CTA of the pair.
__device__ __forceinline__ void load_5d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, int c4, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
      : "memory");
}
__device__ __forceinline__ void load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
// Shared-memory matrix descriptor, 128-byte swizzle (see ffn_batched_tc.cu).
// (An address within a cluster has the CTA's number in its upper bits, which are none of the descriptor's.)
__device__ __forceinline__ constexpr uint32_t desc_lo(uint32_t addr, uint32_t lbo_bytes) { return ((addr >> 4) & 0x3fffu) | (lbo_bytes >> 4 << 16); }
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);     // eight rows of 128 bytes apart
__device__ __forceinline__ void mma_pair(uint32_t tmem_d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc,
                                         uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tmov.b64 a, {%1, %2};\n\tmov.b64 b, {%3, %4};\n\tsetp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %5, p;\n\t}" ::"r"(tmem_d),
      "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Arrives on the barrier of both CTAs (of the cluster's, as a mask) once every product issued so far by this thread has completed.
__device__ __forceinline__ void commit_pair(uint64_t* bar, uint32_t both) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
               "h"((uint16_t)both)
               : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Waits for the loads from TMEM under way, whose registers pass through so that nothing reads them before.
template <int N>
__device__ __forceinline__ void ld_wait(float (&v)[N]) {
  static_assert(N % 8 == 0, "eight registers a time");
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7])::"memory");
#pragma unroll
  for (int i = 8; i < N; i += 8)
    asm volatile("" : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]), "+f"(v[i + 6]), "+f"(v[i + 7])::"memory");
}
// 16 lanes x 16 fp32 columns of TMEM as 8 x 8 fragments: for the columns 8 i .. 8 i + 7 the thread holds, of lane T / 4, the columns 2 (T % 4) and
// the next in v[4 i], v[4 i + 1], and of lane T / 4 + 8 the same in v[4 i + 2], v[4 i + 3].  The caller waits.
__device__ __forceinline__ void tmem_fragments(uint32_t taddr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
// The same of 64 columns.
__device__ __forceinline__ void tmem_fragments_64(uint32_t taddr, float (&v)[32]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(taddr));
}
// Four 8 x 8 matrices of 16-bit values between fragments and shared memory, turned over: a lane gives the address of row
// (lane % 8) of matrix (lane / 8), a row being the fragment's column.
__device__ __forceinline__ void store_turned(uint32_t addr, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(r0), "r"(r1), "r"(r2), "r"(r3) : "memory");
}
// The same as they are: the rows are the fragment's.
__device__ __forceinline__ void store_fragments(uint32_t addr, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(r0), "r"(r1), "r"(r2), "r"(r3) : "memory");
}
__device__ __forceinline__ void load_turned(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// Stores of shared memory as boxes of rows; what lies outside the tensor is left out.
__device__ __forceinline__ void store_3d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void store_4d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2, int c3) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
               : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void epilogue_bar(int group) { asm volatile("bar.sync %0, 128;" ::"r"(1 + group) : "memory"); }

template <typename T> __device__ __forceinline__ uint32_t pack(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <> __device__ __forceinline__ uint32_t pack<__half>(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <typename T> __device__ __forceinline__ float2 unpack(uint32_t v);
template <> __device__ __forceinline__ float2 unpack<__nv_bfloat16>(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

// From exp(-|x|), so that the divisor stays between 1 and 2: the fast division gives 0 for one above 2^126, which silu(x) u of x < -87.3 is not for a large u.
__device__ __forceinline__ float sigmoid(float x) {
  const float e = __expf(-fabsf(x)), r = __fdividef(1.f, 1.f + e);
  return x < 0.f ? e * r : r;                            // (NaN: e and r are, too)
}

// One tile of a pair.
struct Tile {
  int e = 0, row = 0, n = 0;                             // expert; first row (kGradBlocks: column of hidden) and number of them
  int half = 0;                                          // rows of N in each CTA, a multiple of 16
  int m0 = 0;                                            // first row of M (kGateUp: channel)
  int plane = 0;                                         // kGradBlocks: plane of the block
  int first_row = 0, count = 0;                          // kGradBlocks: the expert's rows
  int pieces = 0;                                        // of k
};

// kGradBlocks: halves of a tile, 128 channels, of a plane.  Those of the gates and the ups lie in one row, so that an odd number of them leaves no half
// empty (64 blocks of 1408 x 2048: 17 tiles for 18).
__host__ __device__ constexpr int half_tiles(int channels) { return (channels + 127) / 128; }

// The tiles of a launch in the order of experts, dealt to the pairs in turn: a pair's next tile is as many further as there are pairs.  Each
// role of a CTA walks them by itself, a whole warp together, in steps of mixed digits (no division a tile), with the table of the experts
// (first [N + 1]: their rows, ascending; upto [N + 1]: tiles of N of lower experts) looked at through a window of 32 entries, one in each lane:
// shared memory, busy with operands, takes some hundred cycles to answer, and every tile would wait for it several times.
template <int MODE, bool SPLIT>
struct Walk {
  const ProductArgs& a;
  const int* first;
  const int* upto;
  int base, row_at, tiles_at;                            // window from expert `base` on: entries first[base + lane], upto[base + lane]
  int m_tiles, n_tiles, m, i, e, total;                  // tile of M, tile of N of all experts (of `total`), expert; kGradBlocks: of N, of M of the expert
  int step_m, step_i, step_e;
  __device__ __forceinline__ void look(int from) {
    base = from;
    const int x = min(from + ((int)threadIdx.x & 31), a.n_experts);
    row_at = first[x];
    tiles_at = upto[x];
  }
  __device__ Walk(const ProductArgs& args, const int* first_, const int* upto_) : a(args), first(first_), upto(upto_), e(0) {
    const int rows = MODE == kGateUp ? 2 * a.I : MODE == kGradAct ? a.I : a.H;
    const int parts = SPLIT ? a.parts : 1, pairs = (int)gridDim.x / (2 * parts), pair = (int)blockIdx.x / (2 * parts);          // (clusters, where pairs share a tile)
    m_tiles = (rows + kTile - 1) / kTile;
    const int halves = half_tiles(a.I);
    n_tiles = halves + (halves + 1) / 2;
    m = pair % m_tiles; i = pair / m_tiles;
    step_m = pairs % m_tiles; step_i = pairs / m_tiles;
    step_e = 0;
    if constexpr (MODE == kGradBlocks) {
      e = i / n_tiles; i %= n_tiles;
      step_e = step_i / n_tiles; step_i %= n_tiles;
    }
    total = upto[a.n_experts];
    look(MODE == kGradBlocks ? min(e, a.n_experts) : 0);
  }
  // Back to the first tile, or to none.
  __device__ __forceinline__ void again(bool none) {
    const int cluster = (int)blockIdx.x / (2 * a.parts);
    m = cluster % m_tiles;
    i = none ? total : cluster / m_tiles;
    look(0);
  }
  __device__ bool next(Tile& g) {
    if constexpr (MODE == kGradBlocks) {
      if (e >= a.n_experts) return false;
      if (e > base + 30) look(e);
      g.e = e;
      // half a tile of M for each CTA, of the gates and the ups (the rows of N are the same) or the downs
      const int halves = half_tiles(a.I), cta = (int)blockIdx.x & 1, at = 2 * (i < halves ? i : i - halves) + cta;
      g.plane = i >= halves ? 2 : at >= halves;
      g.m0 = (g.plane == 1 ? at - halves : at) * 128 - cta * 128;
      g.row = m * kTile;
      g.n = min(kTile, a.H - g.row);
      g.first_row = __shfl_sync(0xffffffffu, row_at, e - base);
      g.count = __shfl_sync(0xffffffffu, row_at, e - base + 1) - g.first_row;
      g.pieces = (g.count + kK - 1) / kK;
      m += step_m;
      i += step_i;
      if (m >= m_tiles) { m -= m_tiles; ++i; }
      e += step_e;
      if (i >= n_tiles) { i -= n_tiles; ++e; }
    } else {
      if (i >= total) return false;
      // the last expert with no more tiles in front of it than this one has: the one with this tile
      int behind;
      while ((behind = __popc(__ballot_sync(0xffffffffu, tiles_at <= i))) == 32) look(base + 31);
      const int at = behind - 1, row = __shfl_sync(0xffffffffu, row_at, at), count = __shfl_sync(0xffffffffu, row_at, at + 1) - row;
      const int before = __shfl_sync(0xffffffffu, tiles_at, at), tiles = __shfl_sync(0xffffffffu, tiles_at, at + 1) - before;
      const int size = ((tiles == 1 ? count : (count + tiles - 1) / tiles) + 31) / 32 * 32;       // its rows in equal tiles
      g.e = base + at;
      g.m0 = m * (MODE == kGateUp ? kTile / 2 : kTile);
      g.row = row + (i - before) * size;
      g.n = min(size, count - (i - before) * size);
      const int k = MODE == kDown || MODE == kGradRows ? a.I : a.H;
      g.pieces = (k + kK - 1) / kK * (MODE == kGradRows ? 2 : 1);
      m += step_m;
      i += step_i;
      if (m >= m_tiles) { m -= m_tiles; ++i; }
    }
    g.half = (g.n + 31) / 32 * 16;
    return true;
  }
};

// Turns of sixteen columns that one of `units` groups of four epilogue warps takes for a tile of n columns, `cols` at a time; and the bytes of two groups' turn.
constexpr int kTurnBytes = 256 * 64;
__host__ __device__ constexpr int turns(int n, int cols, int units) { return ((n + cols - 1) / cols + units - 1) / units * (cols / 16); }

// A place in a ring and the parity of its present use.
template <int N>
struct Place {
  int s = 0;
  uint32_t turn = 0;
  __device__ __forceinline__ void next() {
    if (++s == N) { s = 0; turn ^= 1; }
  }
};

template <int MODE, bool SPLIT, typename T>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ ProductArgs a) {
  using S = Shape<MODE>;
  constexpr int kStages = S::kStages, kCols = S::kCols;
  constexpr bool kRagged = MODE == kGradBlocks;          // k ends inside a stage
  constexpr bool kMMajor = MODE == kDown || MODE == kGradRows || MODE == kGradBlocks, kNMajor = MODE == kGradBlocks;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  unsigned char* staging = smem + (size_t)kStages * kStageBytes;
  uint64_t* full = reinterpret_cast<uint64_t*>(staging + S::kStaging);   // even CTA: both halves of a stage are there
  uint64_t* landed = full + kStages;                     // kRagged: this CTA's copies of a stage that needs clearing have landed
  uint64_t* empty = landed + kStages;                    // a stage has been read
  uint64_t* acc_full = empty + kStages;                  // [2] a result is complete
  uint64_t* acc_empty = acc_full + 2;                    // [2] even CTA: it has been read out by both
  uint64_t* drain = acc_empty + 2;
  uint64_t* kept_full = drain + 1;                       // [4] kGradAct: kept gates and ups are there
  uint64_t* kept_empty = kept_full + 4;                  // [4] they have been read by four warps
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(kept_empty + 4);
  int* first = reinterpret_cast<int*>(tmem_slot + 1);    // [N + 1]
  int* upto = first + a.n_experts + 1;                   // [N + 1]

  launch_dependents();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = (int)cluster_rank(), cta = rank & 1, part = SPLIT ? rank >> 1 : 0, parts = SPLIT ? a.parts : 1;
  const uint32_t both = 3u << (2 * part);
  auto in_even_cta = [&](const void* p) { return in_cta(p, 2 * part); };
  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + s, kRagged ? 2 : 1);
      mbar_init(landed + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int b = 0; b < 2; ++b) { mbar_init(acc_full + b, 1); mbar_init(acc_empty + b, 16); }
    mbar_init(drain, 1);
    for (int b = 0; b < 4; ++b) { mbar_init(kept_full + b, 1); mbar_init(kept_empty + b, 4); }
    mbar_fence_init();
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  // Rows of the experts, held to the range and an ascending order, and their tiles of N, summed up.
  bool ascending = true;
  for (int e = tid; e <= a.n_experts; e += kThreads) {
    const int v = min(max(__ldg(a.offsets + e), 0), a.n_rows), before = e ? min(max(__ldg(a.offsets + e - 1), 0), a.n_rows) : 0;
    first[e] = v;
    upto[e] = e ? (v - before + kTile - 1) / kTile : 0;
    ascending &= v >= before;
  }
  if (!__syncthreads_and(ascending)) {
    if (tid == 0)
      for (int e = 1; e <= a.n_experts; ++e) {
        first[e] = max(first[e], first[e - 1]);
        upto[e] = (first[e] - first[e - 1] + kTile - 1) / kTile;
      }
    __syncthreads();
  }
  if (warp == 0) {
    // a piece of the list for each lane
    const int per = (a.n_experts + 32) / 32, e0 = min(lane * per, a.n_experts + 1), e1 = min(e0 + per, a.n_experts + 1);
    int sum = 0;
    for (int e = e0; e < e1; ++e) sum += upto[e];
    int before = sum;
    for (int d = 1; d < 32; d <<= 1) {
      const int w = __shfl_up_sync(0xffffffffu, before, d);
      if (lane >= d) before += w;
    }
    before -= sum;
    for (int e = e0; e < e1; ++e) upto[e] = before += upto[e];
  }
  fence_before();
  __syncthreads();
  cluster_sync_all();
  fence_after();
  const uint32_t tmem = *tmem_slot;
  Walk<MODE, SPLIT> walk(a, first, upto);
  Tile g;
  // A wait by a whole warp.  After one that ran out its role stops, whatever waits for that role runs out in its turn, and the results stay NaN.
  // (The first poll before anything looks at the limit: the roles that copy and multiply find most barriers complete.  Without it the backward pass of
  // 4096 x 6 rows of 64 experts of 2048 x 1408 bf16 took 1003 us instead of 974.)
  auto warp_wait = [&](uint64_t* bar, uint32_t parity, unsigned polls = 0) {
    return __all_sync(0xffffffffu, mbar_try_wait(bar, parity) || mbar_wait(bar, parity, polls ? polls : a.polls)) != 0;
  };
  // the part of a tile's stages that this pair takes
  auto stages_of = [&](int& begin, int& end) {
    const int per = SPLIT ? (g.pieces + parts - 1) / parts : g.pieces;
    begin = min(part * per, g.pieces);
    end = min(begin + per, g.pieces);
  };
  auto polls_for = [&](unsigned pieces) { return a.polls + min(pieces, 1u << 27) * kPiecePolls; };
  auto long_wait = [&]() { return polls_for(g.pieces); };                       // of one tile

  auto missing = [&](Lost what) { return blockIdx.x < 2 && a.lose == what ? 16u : 0u; };        // bytes that are waited for and never come
  if (warp != 0) dependency_wait();                      // (the kernel in front may run for longer than a bounded wait)
  if (warp == 0) {
    // ------------------------------------------------------------------------------------------------ copies
    Place<kStages> at;
    int64_t stages = 0;                                  // issued
    uint32_t cleared = 0, landing = 0;                   // kRagged, a bit for each stage: its copies count on `landed`; parity of its next landing
    bool ok = true;
    const uint32_t ring = uniform((int)smem_u32(smem)), bars = uniform((int)in_even_cta(full)), own_bars = uniform((int)smem_u32(landed));
    while (ok && walk.next(g)) {
      int box = 0;
      if constexpr (kRagged) box = g.half > 64 ? 2 : 1;  // copies of 64 columns
      else while (box_rows(box) < g.half) ++box;
      const uint32_t bytes = kOperandBytes + (kRagged ? box * 8192u : box_rows(box) * 128u) + missing(kOperand);
      const CUtensorMap* n_map = kRagged ? &a.n[g.plane == 2] : &a.n[box];
      const int n_row = g.row + cta * g.half;
      // the operands of stage p; M comes from the blocks (but for kGradBlocks) and so can be on its way before the kernel in front has ended
      auto load_m = [&](int p, uint32_t m_dst, uint32_t bar) {
        if constexpr (MODE == kGateUp) {
          load_5d(m_dst, &a.m, p * kK, 0, 0, (g.m0 + cta * 64) / 8, g.e, bar);
        } else if constexpr (MODE == kGradAct) {
          load_4d(m_dst, &a.m, p * kK, 2, g.m0 + cta * 128, g.e, bar);
        } else if constexpr (MODE == kDown || MODE == kGradRows) {
          const int per = MODE == kDown ? g.pieces : g.pieces / 2;
          const int j = p >= per, k0 = (p - j * per) * kK, plane = MODE == kDown ? 2 : j;
          load_4d(m_dst, &a.m, g.m0 + cta * 128, plane, k0, g.e, bar);
          load_4d(m_dst + 8192, &a.m, g.m0 + cta * 128 + 64, plane, k0, g.e, bar);
        } else {
          const int row = g.first_row + p * kK;
          load_3d(m_dst, &a.m, g.m0 + cta * 128, row, g.plane, bar);
          load_3d(m_dst + 8192, &a.m, g.m0 + cta * 128 + 64, row, g.plane, bar);
        }
      };
      auto load_n = [&](int p, uint32_t n_dst, uint32_t bar) {
        if constexpr (MODE == kGateUp || MODE == kGradAct) {
          load_3d(n_dst, n_map, p * kK, n_row, 0, bar);
        } else if constexpr (MODE == kDown || MODE == kGradRows) {
          const int per = MODE == kDown ? g.pieces : g.pieces / 2;
          const int j = p >= per;
          load_3d(n_dst, n_map, (p - j * per) * kK, n_row, j, bar);
        } else {
          const int row = g.first_row + p * kK;
          load_3d(n_dst, n_map, n_row, row, 0, bar);
          if (box == 2) load_3d(n_dst + 8192, n_map, n_row + 64, row, 0, bar);
        }
      };
      int begin, end;
      stages_of(begin, end);
      int early = begin;                                 // stages of the CTA's first tile before this one have their M on its way already
      if (stages == 0) {
        if constexpr (MODE == kDown || MODE == kGradRows) {
          early = min(end, begin + kStages);
          if (elect_one())
            for (int p = begin; p < early; ++p) {
              if (cta == 0) mbar_expect_tx(full + p - begin, 2 * bytes);
              load_m(p, ring + (p - begin) * kStageBytes, bars + (p - begin) * 8);
            }
          __syncwarp();
        }
        dependency_wait();
      }
      for (int p = begin; p < end; ++p) {
        if (stages >= kStages) {
          ok = warp_wait(empty + at.s, at.turn ^ 1);
          if (!ok) break;
        }
        // kRagged: each CTA's copies or, where it has to clear what follows the rows, its warp 2 arrive for its half
        const bool clear = kRagged && p + 1 == g.pieces && g.count % 16;
        if constexpr (kRagged) {
          cleared = clear ? cleared | 1u << at.s : cleared & ~(1u << at.s);
          landing ^= (uint32_t)clear << at.s;
        }
        if (elect_one()) {
          const uint32_t m_dst = ring + at.s * kStageBytes, bar = (clear ? own_bars : bars) + at.s * 8;
          if (p >= early) {
            if constexpr (kRagged) {
              if (clear) mbar_expect_tx(landed + at.s, bytes);
              else expect_tx_at(bars + at.s * 8, bytes);
            } else if (cta == 0) {
              mbar_expect_tx(full + at.s, 2 * bytes);
            }
            load_m(p, m_dst, bar);
          }
          load_n(p, m_dst + kOperandBytes, bar);
        }
        __syncwarp();
        at.next();
        ++stages;
      }
    }
    // The last products have read their stages and their arrivals have come in before the CTA leaves.
    const int64_t last = stages > kStages ? stages - kStages : 0;
    for (int64_t i = last; ok && i < stages; ++i) ok = warp_wait(empty + (int)(i % kStages), (uint32_t)(i / kStages) & 1);
    if (!ok) {
      // A wait ran out, here or in another role (then these stages were not read).  All copies were issued before it began; they are waited for where
      // their bytes count: `landed` of a stage to be cleared, else the even CTA's `full`, for both CTAs, whose cluster barrier at the end is behind this.
      // (A stage that one of them alone has brought never fills: that wait runs out, too.)  Then the arrivals of the products issued before they stopped.
      for (int64_t i = last; i < stages; ++i) {
        const int s = (int)(i % kStages);
        if (kRagged && (cleared >> s & 1)) warp_wait(landed + s, ((landing >> s) & 1) ^ 1);
        else if (cta == 0) warp_wait(full + s, (uint32_t)(i / kStages) & 1);
      }
      warp_wait(drain, 0);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------------------------------------ products
    if (cta == 0) {
      constexpr uint32_t kType = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
      // fp32 result, both operands of type T, M = 256; bit 15: M is MN-major, bit 16: N is
      constexpr uint32_t kIdesc = (1u << 4) | (kType << 7) | (kType << 10) | ((256u >> 4) << 24) | (kMMajor ? 1u << 15 : 0u) | (kNMajor ? 1u << 16 : 0u);
      // of the ring's first stage; a step of 16 k further: 32 bytes (K-major) or 16 rows of 128
      const uint32_t ring = uniform((int)smem_u32(smem)), d0 = uniform((int)tmem);
      const uint32_t m_desc = desc_lo(ring, kMMajor ? 8192 : 16), n_desc = desc_lo(ring + kOperandBytes, kNMajor ? 8192 : 16);
      constexpr uint32_t kMStep = (kMMajor ? 2048 : 32) >> 4, kNStep = (kNMajor ? 2048 : 32) >> 4;
      Place<kStages> at;
      int acc = 0;
      bool ok = true;
      while (walk.next(g)) {
        if (acc >= 2) ok = warp_wait(acc_empty + (acc & 1), ((acc >> 1) - 1) & 1);
        if (!ok) break;
        fence_after();
        const uint32_t d = d0 + (uint32_t)(acc & 1) * kTile, idesc = kIdesc | ((uint32_t)(2 * g.half) >> 3 << 17);
        int begin, end;
        stages_of(begin, end);
        for (int p = begin; p < end; ++p) {
          ok = warp_wait(full + at.s, at.turn);
          if (!ok) break;
          fence_after();
          if (elect_one()) {
            const uint32_t stage = (uint32_t)(at.s * kStageBytes) >> 4;
#pragma unroll
            for (int k = 0; k < kK / 16; ++k)
              if (!kRagged || p * kK + k * 16 < g.count)           // (sixteen rows that are not the expert's add nothing)
                mma_pair(d, m_desc + stage + k * kMStep, kDescHi, n_desc + stage + k * kNStep, kDescHi, idesc, p > begin || k ? 1u : 0u);
            commit_pair(empty + at.s, both);
          }
          __syncwarp();
          at.next();
        }
        if (!ok) break;
        if (elect_one()) commit_pair(acc_full + (acc & 1), both);
        __syncwarp();
        ++acc;
      }
      if (!ok) {
        if (elect_one()) commit_pair(drain, both);       // let the tensor cores finish before TMEM is freed
        warp_wait(drain, 0);
      }
    }
  } else if (warp < 4) {
    if constexpr (kRagged) {
      // ----------------------------------------------------------------------------- rows behind an expert's last
      if (warp == 2) {
        int at = 0;                                      // stage of a tile's first piece
        uint32_t turns = 0;                              // parity of each stage's next landing
        unsigned passed = 0;                             // pieces of the tiles so far: those with nothing to clear are passed over, and the next wait is for all of them
        bool ok = true;
        while (ok && walk.next(g)) {
          const int s = (at + max(g.pieces, 1) - 1) % kStages, left = g.count - (g.pieces - 1) * kK;
          at = (at + g.pieces) % kStages;
          passed = min(passed + g.pieces + 1, 1u << 27);
          if (left % 16 == 0) continue;
          ok = warp_wait(landed + s, (turns >> s) & 1, polls_for(passed));
          if (!ok) break;
          turns ^= 1u << s;
          // a row of the blocks of 64 rows a time, two of M and those of N
          unsigned char* mine = smem + (size_t)s * kStageBytes + (lane >> 3) * 8192 + (lane & 7) * 16;
          if ((lane >> 3) < (g.half > 64 ? 4 : 3)) {
#pragma unroll 4
            for (int r = left; r < (left + 15) / 16 * 16; ++r) *reinterpret_cast<uint4*>(mine + r * 128) = make_uint4(0, 0, 0, 0);
          }
          // The zeros are read by the tensor cores alone (the async proxy), from the shared memory they were written to: the proxy fence
          // of every lane, then the arrival, puts them before the products.  (Fences at cluster scope on both sides cost 1500 and 1700
          // cycles a tile of 7000.)
          async_fence();
          __syncwarp();
          if (lane == 0) arrive_at(in_even_cta(full + s));
        }
      }
    } else if constexpr (MODE == kGradAct) {
      // ---------------------------------------------------------- kept gates and ups, 16 rows a time, a warp for each epilogue
      const int group = warp - 2;
      const uint32_t bytes = 8192 + missing(kKeptValues);
      Place<2> at;
      int64_t groups = 0;
      bool ok = true;
      if constexpr (SPLIT) {                             // the two meetings of the epilogues, which take nothing from here before them
        cluster_sync_all();
        cluster_sync_all();
      }
      while (ok && walk.next(g)) {
        const int ch = g.m0 + cta * 128;
        for (int c0 = (part + parts * group) * kCols; c0 < g.n; c0 += 2 * parts * kCols) {
          if (groups >= 2) {
            ok = warp_wait(kept_empty + 2 * group + at.s, at.turn ^ 1, long_wait());
            if (!ok) break;
          }
          if (elect_one()) {
            const uint32_t to = smem_u32(staging) + 2 * S::kBuffer + (2 * group + at.s) * 8192, bar = smem_u32(kept_full + 2 * group + at.s);
            mbar_expect_tx(kept_full + 2 * group + at.s, bytes);
            load_3d(to, &a.gate_up, ch, g.row + c0, 0, bar);
            load_3d(to + 4096, &a.gate_up, ch + 64, g.row + c0, 0, bar);
          }
          __syncwarp();
          at.next();
          ++groups;
        }
      }
      // copies under way land before the CTA leaves, whoever still waits for them
      for (int64_t i = groups > 2 ? groups - 2 : 0; i < groups; ++i) warp_wait(kept_full + 2 * group + (int)(i & 1), (uint32_t)(i / 2) & 1);
    }
  } else {
    // ------------------------------------------------------------------------------------------------ results
    const int quad = warp & 3, t = tid & 127, group = (warp - 4) >> 2;
    const bool issuer = quad == 0;                       // one lane of it issues the stores
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    Place<2> at;                                         // kGradAct: of the kept gates and ups
    int third = 0;                                       // kGateUp without kept gates: act alone goes through each third of the buffer in turn
    bool ok = true, kept_ok = true;                      // no wait has run out; none for kept gates and ups
    const bool keep = MODE == kGateUp && a.kept;
    // Groups of kCols columns go round the units: the pairs that share the tile, with their first epilogue group and then with their second.  Each pair
    // sends the others what it has of their columns: 16 columns of a thread as four float4, a place for each of the 256 threads, a slot for each sender.
    const int unit = part + parts * group, units = 2 * parts;
    int slot_bytes = 0;
    if constexpr (SPLIT) {
      const bool here = walk.next(g);
      if (here) {
        slot_bytes = turns(g.n, kCols, units) * kTurnBytes;
        ok = warp_wait(acc_full, 0, long_wait());
        fence_after();
      }
      cluster_sync_all();                                // all products have ended, no ring is in use
      for (int d = 1; here && d < parts; ++d) {
        const int q = part + d < parts ? part + d : part + d - parts;
        uint32_t to = in_cta(smem, 2 * q + cta) + (parts - 1 - d) * slot_bytes + (tid - 128) * 16;
        for (int c0 = (q + parts * group) * kCols; c0 < g.n; c0 += units * kCols)
#pragma unroll 1
          for (int c = c0; c < min(c0 + kCols, g.n); c += 16, to += kTurnBytes) {
            float f[16];
            tmem_fragments(tmem + lanes + c, f);
            tmem_fragments(tmem + lanes + c + (16u << 16), f + 8);
            ld_wait(f);
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] = ok ? f[i] : __uint_as_float(0x7fc00000u);
#pragma unroll
            for (int i = 0; i < 4; ++i) send(to + i * 4096, f + 4 * i);
          }
      }
      cluster_sync_all();                                // they have arrived
      walk.again(!here);
    }
    for (int tile = 0; walk.next(g); ++tile) {
      const float4* theirs = reinterpret_cast<const float4*>(smem) + (tid - 128);
      // columns: kCols each from `from` on, every other such group (kGradBlocks: all, of half of the rows)
      const int acc = tile & 1, from = unit * kCols, by = units * kCols;
      const uint32_t col = tmem + lanes + (uint32_t)acc * kTile;
      if (ok) {
        ok = warp_wait(acc_full + acc, (tile >> 1) & 1, long_wait());
        fence_after();
      }
      // The buffer is free for the products, as far as this warp goes.  After a wait that ran out it stays taken, so that the products stop: this warp no
      // longer follows them, and a buffer given back for it could be written while another warp of the pair still reads.
      auto read_out = [&]() {
        fence_before();
        __syncwarp();
        if (ok && lane == 0) arrive_at(in_even_cta(acc_empty + acc));
      };
      if (MODE != kGradBlocks && from >= g.n) {
        read_out();
        continue;
      }
      if constexpr (MODE == kGradBlocks) {
        const int ch0 = g.m0 + cta * 128 + quad * 32;
        if (g.pieces == 0 && ok) {                       // an expert without rows: zeros, a row's columns of the tile with each access
          read_out();
          const int rows = min(32, a.I - ch0);
          uint16_t* block = a.out + (size_t)g.e * a.block_stride + (size_t)g.plane * a.H + g.row;
          uint16_t* out = block + (size_t)(ch0 + group) * 3 * a.H;
          // Rows start on any 16 bytes, and an access of part of a 32-byte sector costs as much as a whole one: where a row starts in the middle of a
          // sector, its piece begins and ends 8 columns later.
#pragma unroll 4
          for (int r = group; r < rows; r += 2, out += 6 * (size_t)a.H) {
            const int late = reinterpret_cast<uintptr_t>(out) & 16 ? 8 : 0;
            const int c = (g.row ? late : 0) + lane * 8, stop = g.row + g.n < a.H ? g.n + late : g.n;
            if (c < stop) *reinterpret_cast<uint4*>(out + c) = make_uint4(0, 0, 0, 0);
            if (g.row == 0 && lane == 0 && stop > kTile) *reinterpret_cast<uint4*>(out + kTile) = make_uint4(0, 0, 0, 0);
          }
          continue;
        }
        // sixteen rows of a quarter for each group, 64 columns a time
        const int row0 = ch0 + 16 * group;
        if (row0 >= a.I) {
          read_out();
          continue;
        }
        const uint32_t from16 = col + ((uint32_t)group << 20), buffer = smem_u32(staging) + (warp - 4) * 2048;
        float v[32];
        if (ok) tmem_fragments_64(from16, v);
#pragma unroll 1
        for (int c0 = 0; c0 < g.n; c0 += 64) {
          uint32_t packed[16];                           // of rows T / 4 and T / 4 + 8 in turn
          if (ok) {
            ld_wait(v);
#pragma unroll
            for (int j = 0; j < 16; ++j) packed[j] = pack<T>(v[2 * j], v[2 * j + 1]);
            if (c0 + 64 < g.n) tmem_fragments_64(from16 + c0 + 64, v);
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) packed[j] = 0x7fff7fffu;                // NaN in either type
          }
          if (c0 + 64 >= g.n) read_out();
          if (lane == 0) stores_read<0>();
          __syncwarp();
          const int row = ((lane >> 3) & 1) * 8 + (lane & 7);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            store_fragments(buffer + row * 128 + (((2 * j + (lane >> 4)) ^ (row & 7)) << 4), packed[4 * j], packed[4 * j + 1], packed[4 * j + 2],
                            packed[4 * j + 3]);
          async_fence();
          __syncwarp();
          if (lane == 0) {
            store_4d(&a.o[0], buffer, g.row + c0, g.plane, row0, g.e);
            store_commit();
          }
        }
        continue;
      }
      // Sixteen columns a time, in a loop that is not unrolled (a tile of few rows runs its code once, from cold instruction caches: unrolled over
      // 32 columns this took 4.5 us of one token's 18), the next sixteen on their way meanwhile; kCols of them leave together.
      const bool some = ok;
      float f[16];                                       // fragments of lanes 0-15 and 16-31 of the warp's quarter
      auto fetch = [&](int c) {
        if (some) {
          tmem_fragments(col + c, f);
          tmem_fragments(col + c + (16u << 16), f + 8);
        }
      };
      fetch(from);
#pragma unroll 1
      for (int c0 = from; c0 < g.n; c0 += by) {
        const bool whole = c0 + kCols <= g.n;
        unsigned char* buffer = staging + group * S::kBuffer;
        if (MODE == kGateUp && !keep) {
          buffer += third * 4096;
          third = third == 2 ? 0 : third + 1;
        }
        const uint32_t buffer_at = smem_u32(buffer);
        // (Waited for as long as they come, whatever has become of the products: a place given back too early would be brought twice at once.)
        if (MODE == kGradAct && kept_ok) {
          kept_ok = warp_wait(kept_full + 2 * group + at.s, at.turn);
          ok = ok && kept_ok;
        }
#pragma unroll 1
        for (int c = c0; c < min(c0 + kCols, g.n); c += 16) {
          float v[16];
          if (some) ld_wait(f);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = some ? f[i] : __uint_as_float(0x7fc00000u);
          for (int q = 0; q < parts - 1; ++q) {
            const float4* from_q = theirs + q * (slot_bytes / 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float4 w = from_q[i * 256];
              v[4 * i] += w.x; v[4 * i + 1] += w.y; v[4 * i + 2] += w.z; v[4 * i + 3] += w.w;
            }
          }
          theirs += kTurnBytes / 16;
          const int next = c + 16 < c0 + kCols ? c + 16 : c0 + by;
          if (next < g.n) fetch(next);
          else read_out();
          auto free_buffer = [&]() {                     // before the first columns are written
            if (c != c0) return;
            if (issuer && elect_one()) {
              if (MODE == kGateUp && !keep) stores_read<2>();
              else stores_read<0>();
            }
            __syncwarp();
            epilogue_bar(group);
          };
          if constexpr (MODE == kGateUp) {
            // rows of M are eight gates, then the ups of the same channels: a thread holds both.  Output rows of 64 channels, 128 bytes.  act is rounded
            // to 16 bits here, since the next product takes such operands (as d g, d u and a are below): one rounding more than the formula's own.
            uint32_t act[4];                             // two groups of columns x two of channels
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float* w = v + (j & 1) * 8 + (j >> 1) * 4;
              act[j] = pack<T>(w[0] * sigmoid(w[0]) * w[2], w[1] * sigmoid(w[1]) * w[3]);
            }
            free_buffer();
            const int row = c - c0 + (lane >> 4) * 8 + (lane & 7), chunk = quad * 2 + ((lane >> 3) & 1);       // that this lane addresses
            const uint32_t to = buffer_at + row * 128 + ((chunk ^ (row & 7)) << 4);
            store_turned(to, act[0], act[1], act[2], act[3]);
            if (keep) {
              store_turned(to + 4096, pack<T>(v[0], v[1]), pack<T>(v[8], v[9]), pack<T>(v[4], v[5]), pack<T>(v[12], v[13]));
              store_turned(to + 8192, pack<T>(v[2], v[3]), pack<T>(v[10], v[11]), pack<T>(v[6], v[7]), pack<T>(v[14], v[15]));
            }
          } else if constexpr (MODE == kGradAct) {
            // two halves of 64 channels: [2 planes x 16 rows x 128 bytes] of gates and ups, [3 planes x ...] of what leaves
            const uint32_t in_row = (lane & 7) * 128 + ((((quad & 1) * 4 + (lane >> 3)) ^ (lane & 7)) << 4);
            const uint32_t kept_at = smem_u32(staging) + 2 * S::kBuffer + (2 * group + at.s) * 8192 + (quad >> 1) * 4096 + in_row;
            uint32_t gates[2][4], ups[2][4], acts[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              load_turned(kept_at + i * 1024, gates[i]);
              load_turned(kept_at + i * 1024 + 2048, ups[i]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float* w = v + (j >> 1) * 8 + i * 4 + (j & 1) * 2;
                float2 gate = unpack<T>(gates[i][j]);
                const float2 up = unpack<T>(ups[i][j]);
                if (!ok) gate.x = gate.y = __uint_as_float(0x7fc00000u);
                const float s0 = sigmoid(gate.x), s1 = sigmoid(gate.y);
                gates[i][j] = pack<T>(w[0] * up.x * s0 * (1.f + gate.x * (1.f - s0)), w[1] * up.y * s1 * (1.f + gate.y * (1.f - s1)));
                ups[i][j] = pack<T>(w[0] * gate.x * s0, w[1] * gate.y * s1);
                acts[i][j] = pack<T>(gate.x * s0 * up.x, gate.y * s1 * up.y);
              }
            free_buffer();
            const uint32_t to = buffer_at + (quad >> 1) * 6144 + in_row;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              store_turned(to + i * 1024, gates[i][0], gates[i][1], gates[i][2], gates[i][3]);
              store_turned(to + i * 1024 + 2048, ups[i][0], ups[i][1], ups[i][2], ups[i][3]);
              store_turned(to + i * 1024 + 4096, acts[i][0], acts[i][1], acts[i][2], acts[i][3]);
            }
          } else {
            // output rows of 128 values in two halves of [32 rows x 128 bytes]
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = pack<T>(v[2 * j], v[2 * j + 1]);
            free_buffer();
            const int chunk = (quad & 1) * 4 + (lane >> 3);
            const uint32_t to = buffer_at + (quad >> 1) * 4096 + (c - c0 + (lane & 7)) * 128 + ((chunk ^ (lane & 7)) << 4);
            store_turned(to, w[0], w[1], w[4], w[5]);
            store_turned(to + 1024, w[2], w[3], w[6], w[7]);
          }
        }
        if constexpr (MODE == kGradAct) {
          __syncwarp();
          if (kept_ok && lane == 0) mbar_arrive(kept_empty + 2 * group + at.s);
        }
        async_fence();
        epilogue_bar(group);
        if constexpr (MODE == kGateUp) {
          const int ch = g.m0 + cta * 64;
          if (whole) {
            if (issuer && ch < a.I && elect_one()) {
              store_3d(&a.o[0], buffer_at, ch, g.row + c0, 0);
              if (keep) store_3d(&a.o[1], buffer_at + 4096, ch, g.row + c0, 0);
            }
          } else {
#pragma unroll 1
            for (int o = 0; o < (keep ? 3 : 1); ++o) {
              uint16_t* out = o == 0 ? a.out : a.kept + (size_t)(o - 1) * a.n_rows * a.I;
#pragma unroll 1
              for (int row = t >> 3, chunk = t & 7; row < kCols; row += 16)
                if (c0 + row < g.n && ch + chunk * 8 < a.I)
                  *reinterpret_cast<uint4*>(out + (size_t)(g.row + c0 + row) * a.I + ch + chunk * 8) =
                      *reinterpret_cast<const uint4*>(buffer + o * 4096 + row * 128 + ((chunk ^ (row & 7)) << 4));
            }
          }
        } else if constexpr (MODE == kGradAct) {
          const int ch = g.m0 + cta * 128;
          if (whole) {
            if (issuer && elect_one()) {
              if (ch < a.I) store_3d(&a.o[0], buffer_at, ch, g.row + c0, 0);
              if (ch + 64 < a.I) store_3d(&a.o[0], buffer_at + 6144, ch + 64, g.row + c0, 0);
            }
          } else {
#pragma unroll 1
            for (int i = 0; i < 6; ++i) {
              const int row = t >> 3, chunk = t & 7, c = ch + (i / 3) * 64 + chunk * 8;
              if (c0 + row < g.n && c < a.I)
                *reinterpret_cast<uint4*>(a.out + ((size_t)(i % 3) * a.n_rows + g.row + c0 + row) * a.I + c) =
                    *reinterpret_cast<const uint4*>(buffer + i * 2048 + row * 128 + ((chunk ^ (row & 7)) << 4));
            }
          }
        } else {
          const int m = g.m0 + cta * 128;
          if (whole) {
            if (issuer && elect_one()) {
#pragma unroll
              for (int i = 0; i < 2; ++i)
                if (m + i * 64 < a.H) store_3d(&a.o[0], buffer_at + i * 4096, m + i * 64, g.row + c0, 0);
            }
          } else {
            const int half = (t >> 3) & 1, chunk = t & 7, at_m = m + half * 64 + chunk * 8;
            if (at_m < a.H) {
#pragma unroll 1
              for (int row = t >> 4; row < kCols && c0 + row < g.n; row += 8)
                *reinterpret_cast<uint4*>(a.out + (size_t)(g.row + c0 + row) * a.out_stride + at_m) =
                    *reinterpret_cast<const uint4*>(buffer + half * 4096 + row * 128 + ((chunk ^ (row & 7)) << 4));
            }
          }
        }
        if (issuer && elect_one()) store_commit();
        __syncwarp();
        at.next();
      }
    }
    if (MODE == kGradBlocks ? lane == 0 : issuer && elect_one()) stores_done();
    if (!ok) warp_wait(drain, 0);                        // (the arrivals of the last products are for this CTA, too)
  }
  dependency_wait();                                     // no CTA, tiles or not, ends before the kernel in front
  __syncwarp();
  if (SPLIT && warp < (MODE == kGradAct ? 2 : 4)) {      // the two meetings of the epilogues
    cluster_sync_all();
    cluster_sync_all();
  }
  fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 2) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// ---------------------------------------------------------------------------------------------------------- host side

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

cudaError_t encoder(EncodeTiledFn* out) {
  static std::atomic<void*> known{nullptr};
  return sorted::driver_entry("cuTensorMapEncodeTiled", &known, out);
}

struct FfnCall {
  int32_t n_rows, n_experts, hidden, inter, dtype;
  const void* offsets;
  const void* blocks;
  int64_t block_stride;
};

// Failure-detection test aid, with REMOE_FAULT_INJECT=lost_product_copy in the environment when the library is first called for products: of every four
// calls the first waits for a copy of an operand that does not come, in each of its launches, the third for one of kept gates and ups, both under a short limit.
int copy_to_lose() {
  static const bool asked = [] {
    const char* v = std::getenv("REMOE_FAULT_INJECT");
    return v && std::strcmp(v, "lost_product_copy") == 0;
  }();
  if (!asked) return kNone;
  static std::atomic<unsigned> calls{0};
  const unsigned turn = calls.fetch_add(1) % 4;
  return turn == 0 ? kOperand : turn == 2 ? kKeptValues : kNone;
}
constexpr unsigned kFewPolls = 64;                       // 0.1 ms: far above what a copy takes

ProductArgs product_args(const FfnCall& c) {
  ProductArgs a{};
  a.offsets = static_cast<const int*>(c.offsets);
  a.n_experts = c.n_experts; a.n_rows = c.n_rows; a.H = c.hidden; a.I = c.inter;
  a.lose = copy_to_lose();
  a.polls = a.lose ? kFewPolls : kPolls;
  return a;
}

struct Encoder {
  EncodeTiledFn fn;
  CUtensorMapDataType type;
  bool ok;
  void encode(CUtensorMap* m, const void* p, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    const cuuint32_t step[5] = {1, 1, 1, 1, 1};
    auto encoded = [&] {
      return fn(m, type, rank, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    // A thread that has made no call of the runtime's that needs a context has none, and the driver then refuses the first map.
    int device;
    ok = ok && (encoded() || (cudaGetDevice(&device) == cudaSuccess && cudaSetDevice(device) == cudaSuccess && encoded()));
  }
  // `planes` matrices of n rows, `stride` elements apart; boxes of 64 columns and `box_rows` rows of `box_planes` of them
  void matrix(CUtensorMap* m, const void* p, int64_t n, int64_t columns, int64_t stride, int planes, unsigned box_rows, unsigned box_planes = 1) {
    const cuuint64_t dims[3] = {(cuuint64_t)columns, (cuuint64_t)n, (cuuint64_t)planes};
    const cuuint64_t strides[2] = {(cuuint64_t)stride * 2, (cuuint64_t)(planes > 1 ? n * stride : stride) * 2};       // (of one plane any that a map takes)
    const cuuint32_t box[3] = {64, box_rows, box_planes};
    encode(m, p, 3, dims, strides, box);
  }
  // expert blocks; boxes of 64 columns of one plane of `channels` channels
  void blocks(CUtensorMap* m, const FfnCall& c, const void* p, int64_t block_stride, unsigned channels) {
    const cuuint64_t dims[4] = {(cuuint64_t)c.hidden, 3, (cuuint64_t)c.inter, (cuuint64_t)c.n_experts};
    const cuuint64_t strides[3] = {(cuuint64_t)c.hidden * 2, (cuuint64_t)c.hidden * 6, (cuuint64_t)block_stride * 2};
    const cuuint32_t box[4] = {64, 1, channels, 1};
    encode(m, p, 4, dims, strides, box);
  }
  // the same with eight channels of a plane, then those of the next, as neighbours: boxes of 64 columns of gate and up of 64 channels
  void blocks_by_eight(CUtensorMap* m, const FfnCall& c) {
    const cuuint64_t dims[5] = {(cuuint64_t)c.hidden, 8, 3, (cuuint64_t)c.inter / 8, (cuuint64_t)c.n_experts};
    const cuuint64_t strides[4] = {(cuuint64_t)c.hidden * 6, (cuuint64_t)c.hidden * 2, (cuuint64_t)c.hidden * 48, (cuuint64_t)c.block_stride * 2};
    const cuuint32_t box[5] = {64, 8, 2, 8, 1};
    encode(m, c.blocks, 5, dims, strides, box);
  }
  // the rows of N
  void n_rows(ProductArgs* a, const void* p, int64_t n, int64_t columns, int64_t stride, int planes) {
    for (int b = 0; b < kBoxes; ++b) matrix(&a->n[b], p, n, columns, stride, planes, box_rows(b));
  }
};

// `clusters` of `parts` pairs each.
template <int MODE, bool SPLIT, typename T>
cudaError_t launch_pairs(const ProductArgs& a, int clusters, bool follows, cudaStream_t stream) {
  static std::atomic<bool> ready[kMaxDevices];
  const cudaError_t e = allow_dynamic_smem(product_kernel<MODE, SPLIT, T>, Shape<MODE>::smem(REMOE_SORT_MAX_EXPERTS), ready);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(clusters * a.parts * 2));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Shape<MODE>::smem(a.n_experts);
  cfg.stream = stream;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)a.parts * 2;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = follows ? 2 : 1;                        // a product of this call is in front
  return cudaLaunchKernelEx(&cfg, product_kernel<MODE, SPLIT, T>, a);
}

template <int MODE, typename T>
cudaError_t launch_product(const ProductArgs& a, bool follows, cudaStream_t stream) {
  const int m = MODE == kGateUp ? 2 * a.I : MODE == kGradAct ? a.I : a.H;
  const int64_t m_tiles = (m + kTile - 1) / kTile, halves = half_tiles(a.I);
  const int64_t n_tiles = MODE == kGradBlocks ? a.n_experts * (halves + (halves + 1) / 2) : (a.n_rows + (kTile - 1) * (int64_t)std::min(a.n_experts, a.n_rows)) / kTile;
  const int64_t tiles = m_tiles * n_tiles;
  if (tiles == 0) return cudaSuccess;
  ProductArgs args = a;
  args.parts = 1;
  if constexpr (MODE != kGradBlocks) {
    using S = Shape<MODE>;
    // Four pairs for a tile up to 15 tiles, two up to 33: as many clusters as this GPU holds at once, fewer where k is short.  With one, two and four pairs a forward pass of a few
    // rows took (us, the product's pieces of 64 k and its tiles; the rest of the time is the other product's):
    //   16 pieces,  8 tiles 13.1 13.2 12.9   32 pieces,  8 tiles 16.2 14.9 13.8   88 pieces,  8 tiles 31.1 23.9 21.7
    //               16 tiles 13.0 13.5                   15 tiles 25.1 23.6 24.9               15 tiles 41.6 36.5 34.3
    //               30 tiles 22.0 24.5                   30 tiles 19.2 19.9                    30 tiles 61.6 58.4
    // With 256 rows a tile the sharing costs more and a piece takes longer: 16 pieces of 8 tiles 22.4, 21.6, 32 pieces 26.9, 24.2.  Both products
    // shared, 32 rows of one expert of 2048 x 5632 bf16 take 22.9 us instead of 31.4, the gradient of those rows 28.0 instead of 55.2.
    // A slot for each of the other pairs' results, where the ring was
    static_assert(turns(kTile, S::kCols, 4) * kTurnBytes <= S::kStages * kStageBytes && 3 * turns(kTile, S::kCols, 8) * kTurnBytes <= S::kStages * kStageBytes);
    const int k = MODE == kDown || MODE == kGradRows ? a.I : a.H, pieces = (k + kK - 1) / kK * (MODE == kGradRows ? 2 : 1);
    for (int parts : {4, 2})
      if (pieces >= 24 && tiles <= (parts == 4 ? std::min(15, pieces * 3 / 8) : std::min(33, pieces * 11 / 16))) {
        args.parts = parts;
        return launch_pairs<MODE, true, T>(args, (int)tiles, follows, stream);
      }
  }
  // one pair for each pair of SMs, fewer where there are fewer tiles
  return launch_pairs<MODE, false, T>(args, (int)std::min<int64_t>(74, tiles), follows, stream);
}

int check_ffn(const FfnCall& c) {
  if (c.n_rows < 0 || c.n_experts < 1 || c.hidden < 1 || c.inter < 1) return REMOE_E_ARG;
  if (c.dtype == REMOE_F32 || c.dtype == REMOE_FP8_E4M3 || c.dtype == REMOE_INT4_G32) return REMOE_E_UNSUPPORTED;
  if (c.dtype != REMOE_BF16 && c.dtype != REMOE_F16) return REMOE_E_ARG;
  if (c.hidden % 8 || c.inter % 8 || c.hidden > REMOE_FFN_MAX_WIDTH || c.inter > REMOE_FFN_MAX_WIDTH ||
      c.n_experts > REMOE_SORT_MAX_EXPERTS || c.n_rows > (1 << 30) || (int64_t)c.n_rows * c.inter >= (1LL << 38))
    return REMOE_E_UNSUPPORTED;
  if (!c.offsets || rows::misaligned(c.offsets, 4) || !c.blocks || rows::misaligned(c.blocks, 16)) return REMOE_E_ARG;
  if (c.n_experts > 1 && (c.block_stride < (int64_t)3 * c.inter * c.hidden || c.block_stride % 8)) return REMOE_E_ARG;
  if (c.block_stride >= (1LL << 38)) return REMOE_E_UNSUPPORTED;
  return REMOE_OK;
}
// Rows that the copies can take: 16-byte aligned.
bool bad_rows(const void* p, int64_t stride, int64_t n, int64_t columns) {
  return sorted::bad_matrix(p, stride, n, columns, 16) || (n > 1 && (stride % 8 || stride >= (1LL << 38)));
}

template <typename T>
cudaError_t forward(const FfnCall& c, Encoder& enc, const void* xs, int64_t xs_stride, void* gate_up, void* act, void* ys, int64_t ys_stride,
                    cudaStream_t stream) {
  ProductArgs a = product_args(c);
  enc.blocks_by_eight(&a.m, c);
  enc.n_rows(&a, xs, c.n_rows, c.hidden, xs_stride, 1);
  enc.matrix(&a.o[0], act, c.n_rows, c.inter, c.inter, 1, Shape<kGateUp>::kCols);
  if (gate_up) enc.matrix(&a.o[1], gate_up, c.n_rows, c.inter, c.inter, 2, Shape<kGateUp>::kCols, 2);
  a.out = static_cast<uint16_t*>(act);
  a.kept = static_cast<uint16_t*>(gate_up);
  if (!enc.ok) return cudaErrorInvalidValue;
  cudaError_t e = launch_product<kGateUp, T>(a, false, stream);
  if (e != cudaSuccess) return e;
  enc.blocks(&a.m, c, c.blocks, c.block_stride, 64);
  enc.n_rows(&a, act, c.n_rows, c.inter, c.inter, 1);
  enc.matrix(&a.o[0], ys, c.n_rows, c.hidden, ys_stride, 1, Shape<kDown>::kCols);
  a.out = static_cast<uint16_t*>(ys);
  a.out_stride = ys_stride;
  if (!enc.ok) return cudaErrorInvalidValue;
  return launch_product<kDown, T>(a, true, stream);
}

template <typename T>
cudaError_t backward(const FfnCall& c, Encoder& enc, const void* xs, int64_t xs_stride, const void* gate_up, const void* d_ys, int64_t d_ys_stride,
                     void* work, void* d_xs, int64_t d_xs_stride, void* d_blocks, int64_t d_block_stride, cudaStream_t stream) {
  ProductArgs a = product_args(c);
  cudaError_t e = cudaSuccess;
  if (c.n_rows > 0) {
    enc.blocks(&a.m, c, c.blocks, c.block_stride, 128);
    enc.n_rows(&a, d_ys, c.n_rows, c.hidden, d_ys_stride, 1);
    enc.matrix(&a.gate_up, gate_up, c.n_rows, c.inter, c.inter, 2, Shape<kGradAct>::kCols, 2);
    enc.matrix(&a.o[0], work, c.n_rows, c.inter, c.inter, 3, Shape<kGradAct>::kCols, 3);
    a.out = static_cast<uint16_t*>(work);
    if (!enc.ok) return cudaErrorInvalidValue;
    e = launch_product<kGradAct, T>(a, false, stream);
    if (e != cudaSuccess) return e;
  }
  if (d_xs && c.n_rows > 0) {
    enc.blocks(&a.m, c, c.blocks, c.block_stride, 64);
    enc.n_rows(&a, work, c.n_rows, c.inter, c.inter, 2);
    enc.matrix(&a.o[0], d_xs, c.n_rows, c.hidden, d_xs_stride, 1, Shape<kGradRows>::kCols);
    a.out = static_cast<uint16_t*>(d_xs);
    a.out_stride = d_xs_stride;
    if (!enc.ok) return cudaErrorInvalidValue;
    e = launch_product<kGradRows, T>(a, true, stream);
    if (e != cudaSuccess) return e;
  }
  if (d_blocks) {
    if (c.n_rows > 0) {                                  // (without rows no map is looked at)
      enc.matrix(&a.m, work, c.n_rows, c.inter, c.inter, 3, 64);
      enc.matrix(&a.n[0], xs, c.n_rows, c.hidden, xs_stride, 1, 64);
      enc.matrix(&a.n[1], d_ys, c.n_rows, c.hidden, d_ys_stride, 1, 64);
    }
    enc.blocks(&a.o[0], c, d_blocks, d_block_stride, 16);
    a.out = static_cast<uint16_t*>(d_blocks);
    a.block_stride = d_block_stride;
    if (!enc.ok) return cudaErrorInvalidValue;
    e = launch_product<kGradBlocks, T>(a, c.n_rows > 0, stream);
  }
  return e;
}

}  // namespace
}  // namespace remoe

using namespace remoe;

extern "C" int remoe_expert_ffn(int32_t n_rows, int32_t n_experts, int32_t hidden, int32_t inter, int32_t dtype, const void* xs_dev,
                                int64_t xs_stride, const int32_t* offsets_dev, const void* blocks_dev, int64_t block_stride,
                                void* gate_up_dev, void* act_dev, void* ys_dev, int64_t ys_stride, void* cuda_stream) {
  FfnCall c{n_rows, n_experts, hidden, inter, dtype, offsets_dev, blocks_dev, block_stride};
  const int bad = check_ffn(c);
  if (bad) return bad;
  if (bad_rows(xs_dev, xs_stride, n_rows, hidden) || bad_rows(ys_dev, ys_stride, n_rows, hidden) || bad_rows(act_dev, inter, n_rows, inter) ||
      rows::misaligned(gate_up_dev, 16))
    return REMOE_E_ARG;
  if (n_rows == 0) return REMOE_OK;
  if (n_experts == 1) c.block_stride = (int64_t)3 * inter * hidden;
  if (n_rows == 1) xs_stride = ys_stride = hidden;
  rows::PointerDevice device(blocks_dev);
  if (device.err_code()) return device.err_code();
  if (const int host = sorted::check_device_memory({xs_dev, offsets_dev, gate_up_dev, act_dev, ys_dev})) return host;
  Encoder enc{nullptr, dtype == REMOE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, true};
  if (encoder(&enc.fn) != cudaSuccess) return REMOE_E_CUDA;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return rows::status(dtype == REMOE_BF16 ? forward<__nv_bfloat16>(c, enc, xs_dev, xs_stride, gate_up_dev, act_dev, ys_dev, ys_stride, stream)
                                          : forward<__half>(c, enc, xs_dev, xs_stride, gate_up_dev, act_dev, ys_dev, ys_stride, stream));
}

extern "C" int remoe_expert_ffn_backward(int32_t n_rows, int32_t n_experts, int32_t hidden, int32_t inter, int32_t dtype, const void* xs_dev,
                                         int64_t xs_stride, const int32_t* offsets_dev, const void* blocks_dev, int64_t block_stride,
                                         const void* gate_up_dev, const void* d_ys_dev, int64_t d_ys_stride, void* work_dev, void* d_xs_dev,
                                         int64_t d_xs_stride, void* d_blocks_dev, int64_t d_block_stride, void* cuda_stream) {
  FfnCall c{n_rows, n_experts, hidden, inter, dtype, offsets_dev, blocks_dev, block_stride};
  const int bad = check_ffn(c);
  if (bad) return bad;
  if (!d_xs_dev && !d_blocks_dev && n_rows > 0) return REMOE_E_ARG;
  if (bad_rows(d_ys_dev, d_ys_stride, n_rows, hidden) || bad_rows(work_dev, inter, n_rows, inter) || bad_rows(gate_up_dev, inter, n_rows, inter))
    return REMOE_E_ARG;
  if (d_xs_dev && bad_rows(d_xs_dev, d_xs_stride, n_rows, hidden)) return REMOE_E_ARG;
  if (d_xs_dev && d_xs_dev == d_ys_dev && (d_blocks_dev || (d_xs_stride != d_ys_stride && n_rows > 1))) return REMOE_E_ARG;
  if (d_blocks_dev && (bad_rows(xs_dev, xs_stride, n_rows, hidden) || rows::misaligned(d_blocks_dev, 16) ||
                       (n_experts > 1 && (d_block_stride < (int64_t)3 * inter * hidden || d_block_stride % 8))))
    return REMOE_E_ARG;
  if (d_blocks_dev && n_experts > 1 && d_block_stride >= (1LL << 38)) return REMOE_E_UNSUPPORTED;
  if (n_rows == 0 && !d_blocks_dev) return REMOE_OK;
  if (n_experts == 1) c.block_stride = d_block_stride = (int64_t)3 * inter * hidden;
  if (n_rows == 1) xs_stride = d_ys_stride = d_xs_stride = hidden;
  rows::PointerDevice device(blocks_dev);
  if (device.err_code()) return device.err_code();
  if (const int host = n_rows > 0 ? sorted::check_device_memory({offsets_dev, d_blocks_dev, d_blocks_dev ? xs_dev : nullptr, gate_up_dev, d_ys_dev, work_dev, d_xs_dev})
                                  : sorted::check_device_memory({offsets_dev, d_blocks_dev}))
    return host;
  Encoder enc{nullptr, dtype == REMOE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, true};
  if (encoder(&enc.fn) != cudaSuccess) return REMOE_E_CUDA;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return rows::status(dtype == REMOE_BF16 ? backward<__nv_bfloat16>(c, enc, xs_dev, xs_stride, gate_up_dev, d_ys_dev, d_ys_stride, work_dev, d_xs_dev,
                                                                    d_xs_stride, d_blocks_dev, d_block_stride, stream)
                                          : backward<__half>(c, enc, xs_dev, xs_stride, gate_up_dev, d_ys_dev, d_ys_stride, work_dev, d_xs_dev,
                                                             d_xs_stride, d_blocks_dev, d_block_stride, stream));
}
