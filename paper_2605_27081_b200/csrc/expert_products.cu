// The experts' products over rows sorted by expert, forward and backward, on the tensor cores.
//
// Every product is O[n, m] = sum_k M[m, k] N[n, k] over tiles of 256 x up to 256, computed by a pair of CTAs on two
// neighbouring SMs (tcgen05.mma with cta_group::2: each CTA stages 128 rows of M and half of the rows of N and keeps its 128 rows
// of the fp32 result in TMEM, a lane for each m).  The side that belongs to the weights is M, so that the ragged side, the rows of an
// expert, is N, whose width the instruction takes in steps of 32 columns:
//   kGateUp      m = channel (gate and up rows in neighbouring lanes), n = row, k = hidden:   act = silu(g) u
//   kDown        m = hidden,  n = row, k = channel:                                             ys = act W_down
//   kGradAct     m = channel, n = row, k = hidden:    d act = d_ys W_down^T;   d g, d u, act by the derivative of silu(g) u
//   kGradRows    m = hidden,  n = row, k = channel of d g, then of d u:        d_xs = d_g W_gate + d_u W_up
//   kGradBlocks  m = hidden,  n = channel, k = row:   d W = (d g)^T xs, (d u)^T xs, act^T d_ys, one plane of a block each
// Operands come through tensor maps straight from where the caller keeps them: K-major tiles (k contiguous) are [128 rows x 64],
// MN-major ones two [64 x 64] boxes with k as the rows; both are the 128-byte-swizzled images the tensor cores read.
// Per CTA: warp 0 loads (TMA, a ring of six 32 KB stages), warp 1 of the pair's even CTA issues the products, warps 4-7 read the results out of
// TMEM (two buffers of 256 columns, so that a tile's epilogue runs behind the next tile's products).  With k = row (kGradBlocks) an expert's
// last rows end inside a stage; what follows them there (the next expert's rows, or memory that nobody has written) would
// enter the sums, so warp 2 stands between the copies and the products and clears it in both operands.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "expert_host.h"
#include "tma_ring.cuh"

namespace remoe {
namespace {

using namespace ring;

enum Mode { kGateUp, kDown, kGradAct, kGradRows, kGradBlocks };

constexpr int kTile = 256;                               // rows of M and most rows of N of a pair's tile
constexpr int kK = 64;                                   // k of a stage: 128 bytes
constexpr int kOperandBytes = 128 * 128;                 // a CTA's half of an operand
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kStages = 6;
constexpr int kThreads = 256;
constexpr uint32_t kTmemCols = 512;
constexpr unsigned kPolls = 1u << 18;                    // of a bounded wait

struct ProductArgs {
  CUtensorMap m[2];                                      // M: blocks; kGradBlocks: xs, d_ys
  CUtensorMap n[3];                                      // N: boxes of 16, 64 and 128 rows; kGradBlocks: n[0], boxes of 64
  const int* offsets;
  int n_experts, n_rows, H, I;
  const uint16_t* gate_up;                               // kGradAct: [2, n_rows, I]
  uint16_t* out;                                         // rows or blocks; kGateUp, kGradAct: [.., n_rows, I]
  uint16_t* kept;                                        // kGateUp: [2, n_rows, I] or null
  int64_t out_stride;                                    // elements between rows (blocks)
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address of the even CTA's copy of a shared variable.
__device__ __forceinline__ uint32_t in_even_cta(const void* p) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(p)));
  return r;
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Bounded wait that also sees what the other CTA has released.
__device__ __forceinline__ bool wait_cluster(uint64_t* bar, uint32_t parity) {
  for (unsigned it = 0; it < kPolls; ++it) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    if (ok) return true;
  }
  return false;
}
// Loads of this CTA's own shared memory; completion is counted on a barrier of either CTA of the pair.
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
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
  return (uint64_t)((addr >> 4) & 0x3fffu) | ((uint64_t)((lbo_bytes >> 4) & 0x3fffu) << 16) |
         ((uint64_t)((sbo_bytes >> 4) & 0x3fffu) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void mma_pair(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
      "l"(da), "l"(db), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Arrives on the barrier of both CTAs once every product issued so far by this thread has completed.
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
               "h"((uint16_t)3)
               : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 consecutive fp32 columns of this thread's TMEM lane.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

template <typename T> __device__ __forceinline__ uint16_t bits(float v);
template <> __device__ __forceinline__ uint16_t bits<__nv_bfloat16>(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
template <> __device__ __forceinline__ uint16_t bits<__half>(float v) { return __half_as_ushort(__float2half_rn(v)); }
template <typename T> __device__ __forceinline__ float value(uint16_t b);
template <> __device__ __forceinline__ float value<__nv_bfloat16>(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
template <> __device__ __forceinline__ float value<__half>(uint16_t b) { return __half2float(__ushort_as_half(b)); }

__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }

// One tile of a pair.
struct Tile {
  int e, row, n;                                         // expert; first row (kGradBlocks: channel) and number of them
  int half;                                              // rows of N in each CTA, a multiple of 16
  int m0;                                                // first row of M (kGateUp: channel)
  int plane;                                             // kGradBlocks: plane of the block
  int first_row, count;                                  // kGradBlocks: the expert's rows
  int steps;                                             // stages of k
};

// The tiles of a launch in the order of experts, dealt to the pairs in turn.  Each role of a CTA walks them by itself.
template <int MODE>
struct Walk {
  const ProductArgs& a;
  const int *first, *upto;                               // shared memory: [N] first row, [N + 1] tiles of N of lower experts
  const int* count;
  int m_tiles, n_tiles, t, e;
  __device__ Walk(const ProductArgs& args, const int* first_, const int* count_, const int* upto_)
      : a(args), first(first_), upto(upto_), count(count_), t((int)blockIdx.x >> 1), e(0) {
    const int m = MODE == kGateUp ? 2 * a.I : MODE == kGradAct ? a.I : a.H;
    m_tiles = (m + kTile - 1) / kTile;
    n_tiles = (a.I + kTile - 1) / kTile;
  }
  __device__ bool next(Tile& g) {
    if constexpr (MODE == kGradBlocks) {
      const int per = 3 * m_tiles * n_tiles;
      if ((int64_t)t >= (int64_t)a.n_experts * per) return false;
      g.e = t / per;
      int r = t - g.e * per;
      g.plane = r / (m_tiles * n_tiles);
      r -= g.plane * m_tiles * n_tiles;
      const int i = r / m_tiles;
      g.m0 = (r - i * m_tiles) * kTile;
      g.row = i * kTile;
      g.n = min(kTile, a.I - g.row);
      g.first_row = first[g.e];
      g.count = count[g.e];
      g.steps = (g.count + kK - 1) / kK;
    } else {
      while (e < a.n_experts && t >= upto[e + 1] * m_tiles) ++e;
      if (e >= a.n_experts) return false;
      const int local = t - upto[e] * m_tiles, tiles = upto[e + 1] - upto[e];
      const int i = local / m_tiles;
      const int size = ((count[e] + tiles - 1) / tiles + 31) / 32 * 32;
      g.e = e;
      g.m0 = (local - i * m_tiles) * (MODE == kGateUp ? kTile / 2 : kTile);
      g.row = first[e] + i * size;
      g.n = min(size, count[e] - i * size);
      const int k = MODE == kDown || MODE == kGradRows ? a.I : a.H;
      g.steps = (k + kK - 1) / kK * (MODE == kGradRows ? 2 : 1);
    }
    g.half = (g.n + 31) / 32 * 16;
    t += (int)gridDim.x >> 1;
    return true;
  }
};

template <int MODE, typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ ProductArgs a) {
  constexpr bool kRagged = MODE == kGradBlocks;          // k ends inside a stage
  constexpr bool kMMajor = MODE == kDown || MODE == kGradRows || MODE == kGradBlocks, kNMajor = MODE == kGradBlocks;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + (size_t)kStages * kStageBytes);   // even CTA: both halves of a stage are there
  uint64_t* landed = full + kStages;                     // kRagged: this CTA's copies of a stage have landed
  uint64_t* empty = landed + kStages;                    // a stage has been read
  uint64_t* acc_full = empty + kStages;                  // [2] a result is complete
  uint64_t* acc_empty = acc_full + 2;                    // [2] even CTA: it has been read out by both
  uint64_t* drain = acc_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  int* abort_flag = reinterpret_cast<int*>(tmem_slot + 1);
  int* first = abort_flag + 1;                           // [N]
  int* count = first + a.n_experts;                      // [N]
  int* upto = count + a.n_experts;                       // [N + 1]

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int cta = (int)cluster_rank();
  if (tid == 0) {
    *abort_flag = 0;
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + s, kRagged ? 2 : 1);
      mbar_init(landed + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int b = 0; b < 2; ++b) { mbar_init(acc_full + b, 1); mbar_init(acc_empty + b, 8); }
    mbar_init(drain, 1);
    mbar_fence_init();
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  for (int e = tid; e < a.n_experts; e += kThreads) {
    const int lo = min(max(__ldg(a.offsets + e), 0), a.n_rows), hi = min(max(__ldg(a.offsets + e + 1), 0), a.n_rows);
    first[e] = lo;
    count[e] = max(0, hi - lo);
  }
  __syncthreads();
  if (warp == 0) {
    int sum = 0;
    for (int e0 = 0; e0 < a.n_experts; e0 += 32) {
      int v = e0 + lane < a.n_experts ? (count[e0 + lane] + kTile - 1) / kTile : 0;
      for (int d = 1; d < 32; d <<= 1) {
        const int w = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += w;
      }
      if (e0 + lane < a.n_experts) upto[e0 + lane + 1] = sum + v;
      sum += __shfl_sync(0xffffffffu, v, 31);
    }
    if (lane == 0) upto[0] = 0;
  }
  fence_before();
  __syncthreads();
  cluster_sync_all();
  fence_after();
  const uint32_t tmem = *tmem_slot;
  auto aborted = [&]() { return *(volatile int*)abort_flag != 0; };
  auto give_up = [&]() { *(volatile int*)abort_flag = 1; return false; };

  Walk<MODE> walk(a, first, count, upto);
  Tile g;
  if (warp == 0) {
    // ------------------------------------------------------------------------------------------------ copies
    if (lane == 0) {
      int n = 0;
      bool ok = true;
      while (ok && walk.next(g)) {
        const int box = kRagged ? (g.half > 64 ? 2 : 1) : g.half <= 16 ? 0 : g.half <= 64 ? 1 : 2;
        const uint32_t n_bytes = kRagged ? box * 8192u : box == 0 ? 2048u : box == 1 ? 8192u : 16384u;
        for (int kb = 0; kb < g.steps && ok; ++kb, ++n) {
          const int s = n % kStages;
          if (n >= kStages) {
            ok = !aborted() && mbar_wait(empty + s, ((n / kStages) - 1) & 1, kPolls);
            if (!ok) { give_up(); break; }
          }
          const uint32_t m_dst = smem_u32(smem + (size_t)s * kStageBytes), n_dst = m_dst + kOperandBytes;
          uint32_t bar;
          if constexpr (kRagged) {
            mbar_expect_tx(landed + s, kOperandBytes + n_bytes);
            bar = smem_u32(landed + s);
          } else {
            if (cta == 0) mbar_expect_tx(full + s, 2 * (kOperandBytes + n_bytes));
            bar = in_even_cta(full + s);
          }
          const int n_row = g.row + cta * g.half;
          if constexpr (MODE == kGateUp) {
            load_4d(m_dst, &a.m[0], kb * kK, 0, g.m0 + cta * 64, g.e, bar);
            load_3d(n_dst, &a.n[box], kb * kK, n_row, 0, bar);
          } else if constexpr (MODE == kGradAct) {
            load_4d(m_dst, &a.m[0], kb * kK, 2, g.m0 + cta * 128, g.e, bar);
            load_3d(n_dst, &a.n[box], kb * kK, n_row, 0, bar);
          } else if constexpr (MODE == kDown || MODE == kGradRows) {
            const int per = MODE == kDown ? g.steps : g.steps / 2;
            const int j = kb >= per, k0 = (kb - j * per) * kK;
            const int plane = MODE == kDown ? 2 : j;
            load_4d(m_dst, &a.m[0], g.m0 + cta * 128, plane, k0, g.e, bar);
            load_4d(m_dst + 8192, &a.m[0], g.m0 + cta * 128 + 64, plane, k0, g.e, bar);
            load_3d(n_dst, &a.n[box], k0, n_row, j, bar);
          } else {
            const int row = g.first_row + kb * kK;
            const CUtensorMap* m = &a.m[g.plane == 2];
            load_3d(m_dst, m, g.m0 + cta * 128, row, 0, bar);
            load_3d(m_dst + 8192, m, g.m0 + cta * 128 + 64, row, 0, bar);
            load_3d(n_dst, &a.n[0], n_row, row, g.plane, bar);
            if (box == 2) load_3d(n_dst + 8192, &a.n[0], n_row + 64, row, g.plane, bar);
          }
        }
      }
      // The last products have read their stages and their arrivals have come in before the CTA leaves; after a wait that ran out, the
      // copies under way are waited for instead.
      for (int i = n > kStages ? n - kStages : 0; i < n; ++i) {
        if (ok) mbar_wait(empty + i % kStages, (i / kStages) & 1, kPolls);
        else mbar_wait((kRagged ? landed : full) + i % kStages, (i / kStages) & 1, kPolls);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------------------------------------ products
    if (lane == 0 && cta == 0) {
      constexpr uint32_t kType = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
      // fp32 result, both operands of type T, M = 256; bit 15: M is MN-major, bit 16: N is
      constexpr uint32_t kIdesc = (1u << 4) | (kType << 7) | (kType << 10) | ((256u >> 4) << 24) | (kMMajor ? 1u << 15 : 0u) | (kNMajor ? 1u << 16 : 0u);
      int n = 0, acc = 0;
      bool ok = true;
      while (ok && walk.next(g)) {
        if (g.steps == 0) continue;
        if (acc >= 2) ok = !aborted() && wait_cluster(acc_empty + (acc & 1), ((acc >> 1) - 1) & 1);
        if (!ok) break;
        fence_after();
        const uint32_t d = tmem + (uint32_t)(acc & 1) * kTile, idesc = kIdesc | ((uint32_t)(2 * g.half) >> 3 << 17);
        for (int kb = 0; kb < g.steps; ++kb, ++n) {
          const int s = n % kStages;
          ok = !aborted() && wait_cluster(full + s, (n / kStages) & 1);
          if (!ok) break;
          fence_after();
          const uint32_t m_at = smem_u32(smem + (size_t)s * kStageBytes), n_at = m_at + kOperandBytes;
#pragma unroll
          for (int k = 0; k < kK / 16; ++k)
            mma_pair(d, kMMajor ? operand_desc(m_at + k * 2048, 8192, 1024) : operand_desc(m_at + k * 32, 16, 1024),
                     kNMajor ? operand_desc(n_at + k * 2048, 8192, 1024) : operand_desc(n_at + k * 32, 16, 1024), idesc, (kb | k) ? 1u : 0u);
          commit_pair(empty + s);
        }
        if (!ok) break;
        commit_pair(acc_full + (acc & 1));
        ++acc;
      }
      if (!ok) {
        give_up();
        commit_pair(drain);                              // let the tensor cores finish before TMEM is freed
        mbar_wait(drain, 0, kPolls);
      }
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------------------------- rows behind an expert's last
    if constexpr (kRagged) {
      int n = 0;
      bool ok = true;
      while (ok && walk.next(g)) {
        const int chunks = g.half > 64 ? 4 : 3;
        for (int kb = 0; kb < g.steps; ++kb, ++n) {
          const int s = n % kStages;
          ok = !aborted() && mbar_wait(landed + s, (n / kStages) & 1, kPolls);
          if (!ok) break;
          const int left = g.count - kb * kK;
          if (left < kK) {
            unsigned char* st = smem + (size_t)s * kStageBytes;
            for (int i = lane; i < chunks * (kK - left) * 8; i += 32) {
              const int line = i >> 3, c = line / (kK - left), r = left + line % (kK - left);
              *reinterpret_cast<uint4*>(st + c * 8192 + r * 128 + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
          __syncwarp();
          if (lane == 0) arrive_cluster(in_even_cta(full + s));
        }
      }
      if (!ok) give_up();
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------------------------------------------ results
    const int quad = warp & 3;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    int acc = 0;
    bool ok = true;
    while (walk.next(g)) {
      if (g.steps && ok) {
        // a whole tile long: more polls for more stages
        ok = !aborted() && mbar_wait(acc_full + (acc & 1), (acc >> 1) & 1, kPolls + (unsigned)min(g.steps, 1 << 20) * 1024u);
        if (!ok) give_up();
        fence_after();
      }
      const uint32_t col = tmem + lanes + (uint32_t)(acc & 1) * kTile;
      for (int c0 = 0; c0 < g.n; c0 += 32) {
        float v[32];
        if (g.steps && ok) {
          tmem_ld32(col + c0, v);
        } else {
#pragma unroll
          for (int c = 0; c < 32; ++c) v[c] = ok ? 0.f : __uint_as_float(0x7fc00000u);
        }
        if constexpr (MODE == kGateUp) {
          // even lanes hold gates, odd lanes ups of the same channel: one exchange gives each of them both of every other row
          const int ch = g.m0 + cta * 64 + quad * 16 + (lane >> 1), odd = lane & 1;
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            const float got = __shfl_xor_sync(0xffffffffu, odd ? v[c] : v[c + 1], 1);
            const float gate = odd ? got : v[c], up = odd ? v[c + 1] : got;
            const int r = c0 + c + odd;
            if (r < g.n && ch < a.I) {
              const size_t at = (size_t)(g.row + r) * a.I + ch;
              a.out[at] = bits<T>(gate * sigmoid(gate) * up);
              if (a.kept) {
                a.kept[at] = bits<T>(gate);
                a.kept[at + (size_t)a.n_rows * a.I] = bits<T>(up);
              }
            }
          }
        } else {
          const int m = g.m0 + cta * 128 + quad * 32 + lane;
          if (m < (MODE == kGradAct ? a.I : a.H)) {
            if constexpr (MODE == kGradAct) {
              const size_t plane = (size_t)a.n_rows * a.I;
#pragma unroll
              for (int c = 0; c < 32; ++c)
                if (c0 + c < g.n) {
                  const size_t at = (size_t)(g.row + c0 + c) * a.I + m;
                  const float gate = value<T>(__ldg(a.gate_up + at)), up = value<T>(__ldg(a.gate_up + at + plane)), s = sigmoid(gate);
                  a.out[at] = bits<T>(v[c] * up * s * (1.f + gate * (1.f - s)));
                  a.out[at + plane] = bits<T>(v[c] * gate * s);
                  a.out[at + 2 * plane] = bits<T>(gate * s * up);
                }
            } else if constexpr (MODE == kGradBlocks) {
              uint16_t* out = a.out + (size_t)g.e * a.out_stride + (size_t)g.plane * a.H + m;
#pragma unroll
              for (int c = 0; c < 32; ++c)
                if (c0 + c < g.n) out[(size_t)(g.row + c0 + c) * 3 * a.H] = bits<T>(v[c]);
            } else {
#pragma unroll
              for (int c = 0; c < 32; ++c)
                if (c0 + c < g.n) a.out[(size_t)(g.row + c0 + c) * a.out_stride + m] = bits<T>(v[c]);
            }
          }
        }
      }
      if (g.steps) {
        fence_before();
        __syncwarp();
        if (lane == 0) arrive_cluster(in_even_cta(acc_empty + (acc & 1)));
        ++acc;
      }
    }
  }
  __syncwarp();
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
  void* fn = known.load(std::memory_order_acquire);
  if (!fn) {
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found);
    if (e != cudaSuccess) return e;
    if (!fn) return cudaErrorNotSupported;
    known.store(fn, std::memory_order_release);
  }
  *out = reinterpret_cast<EncodeTiledFn>(fn);
  return cudaSuccess;
}

struct Encoder {
  EncodeTiledFn fn;
  CUtensorMapDataType type;
  bool ok;
  void encode(CUtensorMap* m, const void* p, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    const cuuint32_t step[4] = {1, 1, 1, 1};
    ok = ok && fn(m, type, rank, const_cast<void*>(p), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  }
  // `planes` matrices of n rows, `stride` elements apart; boxes of 64 columns and `box_rows` rows
  void matrix(CUtensorMap* m, const void* p, int64_t n, int64_t columns, int64_t stride, int planes, unsigned box_rows) {
    const cuuint64_t dims[3] = {(cuuint64_t)columns, (cuuint64_t)n, (cuuint64_t)planes};
    const cuuint64_t strides[2] = {(cuuint64_t)stride * 2, (cuuint64_t)(n * stride) * 2};
    const cuuint32_t box[3] = {64, box_rows, 1};
    encode(m, p, 3, dims, strides, box);
  }
  // expert blocks; boxes of 64 columns of `kinds` planes of `channels` channels
  void blocks(CUtensorMap* m, const void* p, int n_experts, int H, int I, int64_t block_stride, unsigned kinds, unsigned channels) {
    const cuuint64_t dims[4] = {(cuuint64_t)H, 3, (cuuint64_t)I, (cuuint64_t)n_experts};
    const cuuint64_t strides[3] = {(cuuint64_t)H * 2, (cuuint64_t)H * 6, (cuuint64_t)block_stride * 2};
    const cuuint32_t box[4] = {64, kinds, channels, 1};
    encode(m, p, 4, dims, strides, box);
  }
};

template <int MODE, typename T>
cudaError_t launch_product(const ProductArgs& a, cudaStream_t stream) {
  const size_t smem = 1024 + (size_t)kStages * kStageBytes + 256 + (size_t)(3 * a.n_experts + 1) * 4;
  constexpr size_t kMost = 1024 + (size_t)kStages * kStageBytes + 256 + (size_t)(3 * REMOE_SORT_MAX_EXPERTS + 1) * 4;
  static_assert(kMost <= 227 * 1024, "shared memory of a CTA");
  static std::atomic<bool> ready[kMaxDevices];
  const cudaError_t e = allow_dynamic_smem(product_kernel<MODE, T>, kMost, ready);
  if (e != cudaSuccess) return e;
  // one pair for each pair of SMs, fewer where there are fewer tiles
  const int m = MODE == kGateUp ? 2 * a.I : MODE == kGradAct ? a.I : a.H;
  const int64_t m_tiles = (m + kTile - 1) / kTile, i_tiles = (a.I + kTile - 1) / kTile;
  const int64_t n_tiles = MODE == kGradBlocks ? a.n_experts * 3 * i_tiles : a.n_rows / kTile + std::min(a.n_experts, a.n_rows);
  const int64_t pairs = std::min<int64_t>(74, m_tiles * n_tiles);
  if (pairs == 0) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)pairs * 2);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  return cudaLaunchKernelEx(&cfg, product_kernel<MODE, T>, a);
}

struct FfnCall {
  int32_t n_rows, n_experts, hidden, inter, dtype;
  const void* offsets;
  const void* blocks;
  int64_t block_stride;
};

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
  ProductArgs a{};
  a.offsets = static_cast<const int*>(c.offsets);
  a.n_experts = c.n_experts; a.n_rows = c.n_rows; a.H = c.hidden; a.I = c.inter;
  constexpr unsigned kBox[3] = {16, 64, 128};
  enc.blocks(&a.m[0], c.blocks, c.n_experts, c.hidden, c.inter, c.block_stride, 2, 64);
  for (int b = 0; b < 3; ++b) enc.matrix(&a.n[b], xs, c.n_rows, c.hidden, xs_stride, 1, kBox[b]);
  a.out = static_cast<uint16_t*>(act);
  a.kept = static_cast<uint16_t*>(gate_up);
  if (!enc.ok) return cudaErrorInvalidValue;
  cudaError_t e = launch_product<kGateUp, T>(a, stream);
  if (e != cudaSuccess) return e;
  enc.blocks(&a.m[0], c.blocks, c.n_experts, c.hidden, c.inter, c.block_stride, 1, 64);
  for (int b = 0; b < 3; ++b) enc.matrix(&a.n[b], act, c.n_rows, c.inter, c.inter, 1, kBox[b]);
  a.out = static_cast<uint16_t*>(ys);
  a.out_stride = ys_stride;
  if (!enc.ok) return cudaErrorInvalidValue;
  return launch_product<kDown, T>(a, stream);
}

template <typename T>
cudaError_t backward(const FfnCall& c, Encoder& enc, const void* xs, int64_t xs_stride, const void* gate_up, const void* d_ys, int64_t d_ys_stride,
                     void* work, void* d_xs, int64_t d_xs_stride, void* d_blocks, int64_t d_block_stride, cudaStream_t stream) {
  ProductArgs a{};
  a.offsets = static_cast<const int*>(c.offsets);
  a.n_experts = c.n_experts; a.n_rows = c.n_rows; a.H = c.hidden; a.I = c.inter;
  constexpr unsigned kBox[3] = {16, 64, 128};
  cudaError_t e = cudaSuccess;
  if (c.n_rows > 0) {
    enc.blocks(&a.m[0], c.blocks, c.n_experts, c.hidden, c.inter, c.block_stride, 1, 128);
    for (int b = 0; b < 3; ++b) enc.matrix(&a.n[b], d_ys, c.n_rows, c.hidden, d_ys_stride, 1, kBox[b]);
    a.gate_up = static_cast<const uint16_t*>(gate_up);
    a.out = static_cast<uint16_t*>(work);
    if (!enc.ok) return cudaErrorInvalidValue;
    e = launch_product<kGradAct, T>(a, stream);
    if (e != cudaSuccess) return e;
  }
  if (d_xs && c.n_rows > 0) {
    enc.blocks(&a.m[0], c.blocks, c.n_experts, c.hidden, c.inter, c.block_stride, 1, 64);
    for (int b = 0; b < 3; ++b) enc.matrix(&a.n[b], work, c.n_rows, c.inter, c.inter, 2, kBox[b]);
    a.out = static_cast<uint16_t*>(d_xs);
    a.out_stride = d_xs_stride;
    if (!enc.ok) return cudaErrorInvalidValue;
    e = launch_product<kGradRows, T>(a, stream);
    if (e != cudaSuccess) return e;
  }
  if (d_blocks) {
    if (c.n_rows > 0) {                                  // (without rows no map is looked at)
      enc.matrix(&a.m[0], xs, c.n_rows, c.hidden, xs_stride, 1, 64);
      enc.matrix(&a.m[1], d_ys, c.n_rows, c.hidden, d_ys_stride, 1, 64);
      enc.matrix(&a.n[0], work, c.n_rows, c.inter, c.inter, 3, 64);
    }
    a.out = static_cast<uint16_t*>(d_blocks);
    a.out_stride = d_block_stride;
    if (!enc.ok) return cudaErrorInvalidValue;
    e = launch_product<kGradBlocks, T>(a, stream);
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
  if (n_rows == 0 && !d_blocks_dev) return REMOE_OK;
  if (n_experts == 1) c.block_stride = d_block_stride = (int64_t)3 * inter * hidden;
  if (n_rows == 1) xs_stride = d_ys_stride = d_xs_stride = hidden;
  rows::PointerDevice device(blocks_dev);
  if (device.err_code()) return device.err_code();
  Encoder enc{nullptr, dtype == REMOE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, true};
  if (encoder(&enc.fn) != cudaSuccess) return REMOE_E_CUDA;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return rows::status(dtype == REMOE_BF16 ? backward<__nv_bfloat16>(c, enc, xs_dev, xs_stride, gate_up_dev, d_ys_dev, d_ys_stride, work_dev, d_xs_dev,
                                                                    d_xs_stride, d_blocks_dev, d_block_stride, stream)
                                          : backward<__half>(c, enc, xs_dev, xs_stride, gate_up_dev, d_ys_dev, d_ys_stride, work_dev, d_xs_dev,
                                                             d_xs_stride, d_blocks_dev, d_block_stride, stream));
}
