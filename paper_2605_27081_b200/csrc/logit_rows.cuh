// Shared parts of the operators on rows of logits (token_logprobs.cu, distill.cu): how a row is cut into units, the
// one-pass softmax sums of a row, and their joins within a block and across a cluster.
//
// Units.  A row of V elements starts `pad` elements behind a 16-byte boundary.  It is cut into units of eight
// elements that start on such boundaries; position p = id + pad of an element gives its unit p / 8.  All units but the
// first (pad > 0) and the last (ragged) are loaded and stored with 16-byte instructions; those two go element by
// element, so nothing outside the row is touched whatever its length, address and stride.
//
// Sums.  With m the largest logit and c = log2(e) / temperature, a row's state is
//   m,  R = sum of 2^((x - m) c) over all elements but one that equals m,  U = sum of (x - m) c 2^((x - m) c),
// so Z = 1 + R, ln Z = log1p(R) and the entropy is ln Z - ln 2 U / Z.  Leaving the largest element out of R keeps
// ln Z exact where one token has nearly all of the mass (R = 1e-7 would be lost in a sum that starts at one).
// A thread keeps its largest element M apart: every element meets M in a max/min pair, the larger stays M and the
// smaller goes into the sum.  The sum is taken relative to a reference, an earlier M, that moves only when M has
// risen 2^40 above it; a running maximum would cost a branch in nearly every step of a warp.
// Differences are taken before the scaling: rows of the type's lowest value stay uniform, none becomes inf - inf.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "remoe.h"
#include "tma_ring.cuh"

namespace remoe {
namespace rows {

constexpr float kInf = HUGE_VALF;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float nan_value() { return __int_as_float(0x7fffffff); }
constexpr float kReferenceRise = 40.f;      // log2 of how far a thread's sum may grow above its reference's one

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// Two float32 in one 64-bit register for the packed instructions of sm_100.
typedef unsigned long long f2;
__device__ __forceinline__ f2 pack2(float lo, float hi) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(f2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// ---- element types -------------------------------------------------------------------------------------------
// Four words of two elements each; float32 words are the packed pairs above.
template <typename T>
struct Elem;

template <>
struct Elem<float> {
  typedef f2 Word;
  static constexpr int kUnusedBits = 0;       // low bits of the value as a float32 that are always zero
  static __device__ __forceinline__ Word lowest() { return pack2(-kInf, -kInf); }
  static __device__ __forceinline__ f2 widen(Word w) { return w; }
  static __device__ __forceinline__ Word narrow(f2 v) { return v; }
  static __device__ __forceinline__ void order(Word& hi, Word& lo) {   // hi, lo = max, min per half; NaN goes to both
    float a0, a1, b0, b1;
    unpack2(hi, a0, a1);
    unpack2(lo, b0, b1);
    hi = pack2(max_nan(a0, b0), max_nan(a1, b1));
    lo = pack2(min_nan(a0, b0), min_nan(a1, b1));
  }
  static constexpr bool kLifts = false;         // no packed maximum: the exponent is clamped instead
  static constexpr float kFloor = -kInf;
  static __device__ __forceinline__ Word lift(Word w) { return w; }
  static __device__ __forceinline__ Word larger(Word a, Word b) {
    float a0, a1, b0, b1;
    unpack2(a, a0, a1);
    unpack2(b, b0, b1);
    return pack2(max_nan(a0, b0), max_nan(a1, b1));
  }
  static __device__ __forceinline__ float masked() { return -kInf; }
  static __device__ __forceinline__ float get(const float* p) { return *p; }
  static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
};

template <>
struct Elem<__nv_bfloat16> {
  typedef uint32_t Word;
  static constexpr int kUnusedBits = 16;
  static __device__ __forceinline__ Word lowest() { return 0xff80ff80u; }
  static __device__ __forceinline__ f2 widen(Word w) { return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
  static __device__ __forceinline__ Word narrow(f2 v) {
    float lo, hi;
    unpack2(v, lo, hi);
    Word w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
  }
  static __device__ __forceinline__ void order(Word& hi, Word& lo) {
    Word a;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(hi), "r"(lo));
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(lo) : "r"(hi), "r"(lo));
    hi = a;
  }
  static constexpr bool kLifts = true;
  static constexpr float kFloor = -1152921504606846976.f;
  static __device__ __forceinline__ Word larger(Word a, Word b) {
    Word r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ Word lift(Word w) { return larger(w, 0xdd80dd80u); }   // at least kFloor
  static __device__ __forceinline__ __nv_bfloat16 masked() { return __ushort_as_bfloat16((unsigned short)0xff80); }
  static __device__ __forceinline__ float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  static __device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
};

template <>
struct Elem<__half> {
  typedef uint32_t Word;
  static constexpr int kUnusedBits = 13;
  static __device__ __forceinline__ Word lowest() { return 0xfc00fc00u; }
  static __device__ __forceinline__ f2 widen(Word w) {
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
    return pack2(v.x, v.y);
  }
  static __device__ __forceinline__ Word narrow(f2 v) {
    float lo, hi;
    unpack2(v, lo, hi);
    Word w;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
  }
  static __device__ __forceinline__ void order(Word& hi, Word& lo) {
    Word a;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(a) : "r"(hi), "r"(lo));
    asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(hi), "r"(lo));
    hi = a;
  }
  static constexpr bool kLifts = true;
  static constexpr float kFloor = -65504.f;
  static __device__ __forceinline__ Word larger(Word a, Word b) {
    Word r;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ Word lift(Word w) { return larger(w, 0xfbfffbffu); }   // at least kFloor
  static __device__ __forceinline__ __half masked() { return __ushort_as_half((unsigned short)0xfc00); }
  static __device__ __forceinline__ float get(const __half* p) { return __half2float(*p); }
  static __device__ __forceinline__ void put(__half* p, float v) { *p = __float2half_rn(v); }
};

// ---- units ---------------------------------------------------------------------------------------------------

template <typename T>
struct Unit {
  typename Elem<T>::Word w[4];
  __device__ __forceinline__ void values(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(Elem<T>::widen(w[i]), v[2 * i], v[2 * i + 1]);
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {   // values that came from the type: no rounding
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = Elem<T>::narrow(pack2(v[2 * i], v[2 * i + 1]));
  }
};

// Elements between the 16-byte boundary at or before `row` and `row`.
template <typename T>
__host__ __device__ __forceinline__ int row_pad(const T* row) { return (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T)); }

// p: 16-byte aligned, eight elements of the row.  Loads bypass L1: a row is read once or twice, the second time
// long after the first.
__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void store16(void* p, const uint4& v) {
  asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
template <typename T>
__device__ __forceinline__ void load_unit(const T* p, Unit<T>& u) {
  const uint4 v = load16(p);
  u.w[0] = v.x; u.w[1] = v.y; u.w[2] = v.z; u.w[3] = v.w;
}
template <>
__device__ __forceinline__ void load_unit<float>(const float* p, Unit<float>& u) {
  const uint4 a = load16(p), b = load16(p + 4);
  u.w[0] = pack2(__uint_as_float(a.x), __uint_as_float(a.y));
  u.w[1] = pack2(__uint_as_float(a.z), __uint_as_float(a.w));
  u.w[2] = pack2(__uint_as_float(b.x), __uint_as_float(b.y));
  u.w[3] = pack2(__uint_as_float(b.z), __uint_as_float(b.w));
}
template <typename T>
__device__ __forceinline__ void store_unit(T* p, const Unit<T>& u) {
  store16(p, make_uint4(u.w[0], u.w[1], u.w[2], u.w[3]));
}
template <>
__device__ __forceinline__ void store_unit<float>(float* p, const Unit<float>& u) {
  float v[8];
  u.values(v);
  store16(p, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
  store16(p + 4, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])));
}

// Unit u of a row, element by element; what lies outside the row reads as -inf and is not stored.
template <typename T>
__device__ __forceinline__ void load_ragged(const T* row, int V, int pad, int u, Unit<T>& out) {
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int id = 8 * u + j - pad;
    v[j] = id >= 0 && id < V ? Elem<T>::get(row + id) : -kInf;
  }
  out.set(v);
}
template <typename T>
__device__ __forceinline__ void store_ragged(T* row, int V, int pad, int u, const Unit<T>& in) {
  float v[8];
  in.values(v);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int id = 8 * u + j - pad;
    if (id >= 0 && id < V) Elem<T>::put(row + id, v[j]);
  }
}

// The units [first, last) of a row that one block works on; [full0, full1) of them are whole and aligned.
struct Slice {
  int pad, first, last, full0, full1;
  __device__ __forceinline__ Slice(int V, int pad_, int part, int parts) : pad(pad_) {
    const int units = (V + pad + 7) >> 3, per = (units + parts - 1) / parts;
    first = min(part * per, units);
    last = min(first + per, units);
    full0 = max(first, pad > 0 ? 1 : 0);
    full1 = min(last, (V + pad) >> 3);
  }
  // The i-th ragged unit of the slice (at most two), or -1.
  __device__ __forceinline__ int ragged(int i) const {
    const int head = first < last && first < full0 ? first : -1;
    const int tail = last > first && last - 1 >= full1 && last - 1 != head ? last - 1 : -1;
    return i == 0 ? head : tail;
  }
  __device__ __forceinline__ int length(int V) const { return max(0, min(V, 8 * last - pad) - max(0, 8 * first - pad)); }   // elements
  __device__ __forceinline__ bool holds(int id) const { const int u = (id + pad) >> 3; return u >= first && u < last; }
};

// Bounded wait for a barrier's phase: false if it has not come after a second or so.  A failed try sleeps for up to ten
// microseconds or until the phase comes.
__device__ __forceinline__ bool wait_phase(uint64_t* bar, uint32_t parity) {
  for (unsigned it = 0; it < (1u << 17); ++it) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(ring::smem_u32(bar)), "r"(parity), "r"(10000u) : "memory");
    if (ok) return true;
  }
  return false;
}

// ---- a slice in shared memory ----------------------------------------------------------------------------------
// A block brings its slice of the row into shared memory with bulk copies and works on it there: the whole slice is in
// flight at once whatever the threads' registers hold, and what is looked at again (candidates of the top elements, the
// gradient's second pass) is not read from memory again.  Blocks are small enough for several to lie on an SM, so that
// one's loads overlap another's arithmetic and stores.

template <typename T>
__device__ __forceinline__ void load_shared_unit(const unsigned char* units, int i, Unit<T>& u) {
  const uint4 v = reinterpret_cast<const uint4*>(units)[i];
  u.w[0] = v.x; u.w[1] = v.y; u.w[2] = v.z; u.w[3] = v.w;
}
template <>
__device__ __forceinline__ void load_shared_unit<float>(const unsigned char* units, int i, Unit<float>& u) {
  const ulonglong2 a = reinterpret_cast<const ulonglong2*>(units)[2 * i], b = reinterpret_cast<const ulonglong2*>(units)[2 * i + 1];
  u.w[0] = a.x; u.w[1] = a.y; u.w[2] = b.x; u.w[3] = b.y;
}

constexpr uint32_t kCopyBytes = 32768;        // of one bulk copy at most

// Starts the copies (thread 0) and brings the ragged units element by element (the next sixteen threads), -inf around the
// row.  The caller synchronises the block, then every thread waits for `bar` with wait_slice.
template <typename T>
__device__ __forceinline__ void start_slice(const T* row, int V, const Slice& sl, unsigned char* units, uint64_t* bar) {
  constexpr uint32_t kUnit = 8 * sizeof(T);
  const int tid = threadIdx.x;
  if (tid == 0) {
    ring::mbar_init(bar, 1);
    ring::mbar_fence_init();
    const uint32_t bytes = sl.full1 > sl.full0 ? (uint32_t)(sl.full1 - sl.full0) * kUnit : 0u;
    ring::mbar_expect_tx(bar, bytes);
    const unsigned char* src = reinterpret_cast<const unsigned char*>(row - sl.pad + 8 * (int64_t)sl.full0);
    unsigned char* dst = units + (size_t)(sl.full0 - sl.first) * kUnit;
    for (uint32_t o = 0; o < bytes; o += kCopyBytes) ring::bulk_g2s(dst + o, src + o, min(kCopyBytes, bytes - o), bar);
  } else if (tid >= 32 && tid < 48) {
    const int u = sl.ragged((tid >> 3) & 1), id = 8 * u + (tid & 7) - sl.pad;
    if (u >= 0) reinterpret_cast<T*>(units)[8 * (u - sl.first) + (tid & 7)] = id >= 0 && id < V ? row[id] : Elem<T>::masked();
  }
}
// False if the copies have not arrived within the limit of a wait and of another one: the row is given up as NaN.
__device__ __forceinline__ bool wait_slice(uint64_t* bar) { return wait_phase(bar, 0) || wait_phase(bar, 0); }

// ---- many rows: a persistent block with a ring of chunks --------------------------------------------------------
// With at least a row for every SM, blocks stay and take row after row.  The whole units of the rows pass through a ring of
// NB chunks in shared memory, filled by bulk copies that run ahead over the ends of rows: while a row is joined, its
// top elements are selected or its list is prepared, the next row is already on its way.  No cluster, so no waiting for
// other blocks: two to five blocks an SM, each with its own rows.  One warp issues the copies; the others consume, each at
// its own pace (a warp that is done with a chunk says so on the slot's `empty` barrier).
template <int NB>
struct PipeShared {
  uint64_t full[NB], empty[NB];
};

template <typename T, int CHUNK>              // CHUNK: bytes
struct Chunks {
  static constexpr int kUnits = CHUNK / (8 * (int)sizeof(T));
  static __device__ __forceinline__ int count(const Slice& sl) { return sl.full1 > sl.full0 ? (sl.full1 - sl.full0 + kUnits - 1) / kUnits : 0; }
  static __device__ __forceinline__ int units(const Slice& sl, int c) { return min(kUnits, sl.full1 - sl.full0 - c * kUnits); }
};

// Thread 0, before the block's first barrier.
template <int NB>
__device__ __forceinline__ void init_pipe(PipeShared<NB>& ps, int consumer_warps) {
  for (int s = 0; s < NB; ++s) {
    ring::mbar_init(&ps.full[s], 1);
    ring::mbar_init(&ps.empty[s], (unsigned)consumer_warps);
  }
  ring::mbar_fence_init();
}

// Weights of a block's rows r0, r0 + step, ..., read 32 at a time, a lane each: a load waits behind the copies on their way.
struct RowWeights {
  const float* weight;                        // null: all 1
  int64_t r0, step, n_rows;
  float mine = 1.f;
  int have = -1;
  __device__ __forceinline__ RowWeights(const float* w, int64_t n, int64_t first, int64_t by) : weight(w), r0(first), step(by), n_rows(n) {}
  // Weight of the block's i-th row; whole warps.
  __device__ __forceinline__ float at(int i) {
    if (!weight) return 1.f;
    if (i >> 5 != have) {
      have = i >> 5;
      const int64_t r = r0 + (int64_t)((i & ~31) + (int)(threadIdx.x & 31)) * step;
      mine = r < n_rows ? weight[r] : 0.f;
    }
    return __shfl_sync(0xffffffffu, mine, i & 31);
  }
  __device__ __forceinline__ int64_t row(int i) const { return r0 + (int64_t)i * step; }
  // The first row from i on that counts; its row() is n_rows or more if there is none.
  __device__ __forceinline__ int next(int i) {
    while (row(i) < n_rows && at(i) == 0.f) ++i;
    return i;
  }
};

// One warp: all copies of the rows that the weights' owner takes, issued by its first lane.  Rows with weight 0 are passed over.
template <typename T, int NB, int CHUNK>
__device__ void produce(PipeShared<NB>& ps, unsigned char* buf, RowWeights weights, const T* logits, int64_t stride, int V) {
  typedef Chunks<T, CHUNK> C;
  int turn = 0, phase = 0;                    // slot of the next load, and how often its turn has come
  bool ok = true;
  for (int i = weights.next(0); weights.row(i) < weights.n_rows; i = weights.next(i + 1)) {
    if ((threadIdx.x & 31) != 0 || !ok) continue;
    const T* row = logits + weights.row(i) * stride;
    const Slice sl(V, row_pad(row), 0, 1);
    const int n = C::count(sl);
    const T* base = row - sl.pad + 8 * (int64_t)sl.full0;
    for (int c = 0; c < n; ++c) {
      if (phase > 0 && !wait_phase(&ps.empty[turn], (phase - 1) & 1)) { ok = false; break; }
      const uint32_t bytes = (uint32_t)C::units(sl, c) * (8 * (uint32_t)sizeof(T));
      ring::mbar_expect_tx(&ps.full[turn], bytes);
      ring::bulk_g2s(buf + (size_t)turn * CHUNK, base + 8 * (int64_t)c * C::kUnits, bytes, &ps.full[turn]);
      if (++turn == NB) { turn = 0; ++phase; }
    }
  }
  // no copy is on its way when the warp leaves: each slot's last load has arrived
  if ((threadIdx.x & 31) == 0)
    for (int s = 0; s < NB; ++s) {
      const int loads = phase + (s < turn ? 1 : 0);
      if (loads > 0) wait_phase(&ps.full[s], (loads - 1) & 1);
    }
}

// A reader's place in the ring: slots come in turn.
template <int NB>
struct RingPlace {
  int slot = 0, parity = 0;
  bool ok = true;                             // false once a wait has run out: what follows is NaN
  __device__ __forceinline__ void wait(uint64_t* bars) {
    if (ok) ok = wait_phase(&bars[slot], parity);
  }
  // The warp is done with the slot and says so on `bars`.  The next copy into the slot is not ordered behind loads out of it
  // that are still on their way to registers, so the arrival is made to depend on something that was computed from all
  // of them (`seen`, any value): it decides which lane arrives.
  __device__ __forceinline__ void pass(uint64_t* bars, bool seen) {
    const int lane = __any_sync(0xffffffffu, seen) ? 1 : 0;
    __syncwarp();
    if ((threadIdx.x & 31) == lane) ring::mbar_arrive(&bars[slot]);
    if (++slot == NB) { slot = 0; parity ^= 1; }
  }
};

// Named barriers of a block.  kBarGroup: over a group of NT threads; kBarFinish: over the finishers; kBarReady, kBarFree: between
// consumers and finishers, kBarIds, kBarList, kBarListFree: for the lists of distill.cu, two each, by the row's parity.
constexpr int kBarGroup = 1, kBarFinish = 2, kBarReady = 4, kBarFree = 6, kBarIds = 8, kBarList = 10, kBarListFree = 12;
template <int NT>
__device__ __forceinline__ void sync_threads() { asm volatile("bar.sync %0, %1;" ::"n"(kBarGroup), "n"(NT) : "memory"); }

// A group of threads of the block: its barrier.
template <int NT>
struct WholeGroup {                           // all consumers, or all threads of the block
  static constexpr int kThreads = NT;
  __device__ __forceinline__ void sync() const { sync_threads<NT>(); }
};

// One of two barriers, by the row's parity (their numbers are immediates: a register would claim all of the block's sixteen).
template <int ID, int NT>
__device__ __forceinline__ void bar_sync(int parity) {
  if (parity) asm volatile("bar.sync %0, %1;" ::"n"(ID + 1), "n"(NT) : "memory");
  else asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(NT) : "memory");
}
template <int NT>
struct FinishGroup {                          // the finishers
  static constexpr int kThreads = NT;
  __device__ __forceinline__ void sync() const { bar_sync<kBarFinish, NT>(0); }
};
template <int ID, int NT>
__device__ __forceinline__ void bar_arrive(int parity) {
  __threadfence_block();
  if (parity) asm volatile("bar.arrive %0, %1;" ::"n"(ID + 1), "n"(NT) : "memory");
  else asm volatile("bar.arrive %0, %1;" ::"n"(ID), "n"(NT) : "memory");
}

// ---- element-wise passes ---------------------------------------------------------------------------------------
// A block's piece [u0, u1) of a row's units, written to `out` through f(unit number, unit), 64 bytes a thread at a time; the first
// are loaded before it is known whether the row counts.  Stores are whole units of `out`; loads are where `row` lies alike.
constexpr int kPieceThreads = 256;
template <typename T>
struct Piece {
  static constexpr int kUnits = sizeof(T) == 2 ? 4 : 2;
  const T* row;
  T* out;
  int V, pad, full0, full1, u0, u1;
  bool alike;
  __device__ __forceinline__ Piece(const T* row_, T* out_, int V_, int part, int parts) : row(row_), out(out_), V(V_), pad(row_pad(out_)) {
    const int units = (V + pad + 7) >> 3, per = (units + parts - 1) / parts;
    alike = row_pad(row_) == pad;
    full0 = pad > 0 ? 1 : 0;
    full1 = (V + pad) >> 3;
    u0 = min(part * per, units);
    u1 = min(u0 + per, units);
  }
  __device__ __forceinline__ void load(int u, Unit<T>& q) const {
    if (alike && u >= full0 && u < full1) load_unit(row - pad + 8 * (int64_t)u, q);
    else load_ragged(row, V, pad, u, q);
  }
  __device__ __forceinline__ void store(int u, const Unit<T>& q) const {
    if (u >= full0 && u < full1) store_unit(out - pad + 8 * (int64_t)u, q);
    else store_ragged(out, V, pad, u, q);
  }
  __device__ __forceinline__ void load_batch(int u, Unit<T> (&q)[kUnits]) const {
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
      if (u + i * kPieceThreads < u1) load(u + i * kPieceThreads, q[i]);
  }
  template <typename F>
  __device__ __forceinline__ void run(Unit<T> (&q)[kUnits], F f) const {
    for (int u = u0 + threadIdx.x; u < u1;) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i)
        if (u + i * kPieceThreads < u1) f(u + i * kPieceThreads, q[i]);
#pragma unroll
      for (int i = 0; i < kUnits; ++i)
        if (u + i * kPieceThreads < u1) store(u + i * kPieceThreads, q[i]);
      u += kPieceThreads * kUnits;
      load_batch(u, q);
    }
  }
  // The same where the row is not looked at: every element is `value`.
  __device__ __forceinline__ void fill(float value) const {
    const float v[8] = {value, value, value, value, value, value, value, value};
    Unit<T> q;
    q.set(v);
    for (int u = u0 + threadIdx.x; u < u1; u += kPieceThreads) store(u, q);
  }
};

// ---- one-pass sums -------------------------------------------------------------------------------------------

struct State {
  float m, R, U;     // m = -inf: no live element; R = NaN: the row holds a NaN or +inf
};

__device__ __forceinline__ State merge(const State& a, const State& b, float c) {
  const bool swap = b.m > a.m;
  const State h = swap ? b : a, l = swap ? a : b;
  if (l.m == -kInf) return h;
  const float d = (l.m - h.m) * c, r = ex2(d);
  State s;
  s.m = h.m;
  s.R = h.R + (1.f + l.R) * r;
  s.U = h.U + r * l.U + (r == 0.f ? 0.f : r * d * (1.f + l.R));
  return s;
}

// One thread's running sums over the units it is given.
//   EXACT: R leaves the largest element out (otherwise 1 + R is the plain sum, good to a rounding); ENTROPY: U is kept.
// Two ways to the exponent.  Near: fma(x, c, -k) with k a whole number near m c, one packed instruction whose only error is
// the rounding of its result (k is exact, and so is any change of it).  Far, for values so large that x c has no
// fraction left or overflows (rows of the type's lowest value): (x - m) c.
// The near way takes -inf as a large negative number where U is kept, since 0 * inf is none; it is used only where
// that number is 2^-160 of the reference or less.
template <typename T, bool EXACT, bool ENTROPY>
struct Stream {
  typename Elem<T>::Word M;
  float ref, k, limit, c;
  bool far;
  f2 R, U;
  __device__ __forceinline__ explicit Stream(float c_) : M(Elem<T>::lowest()), ref(0.f), k(0.f), limit(-kInf), c(c_), far(false), R(0), U(0) {}

  __device__ __forceinline__ void move_reference(float m) {
    const float t = m * c;
    const bool go_far = !(fabsf(t) < 1048576.f && c < 1e15f && (m - Elem<T>::kFloor) * c >= 160.f);
    const float nk = rintf(t);
    if (limit > -kInf) {
      // from the reference that the sums are relative to (2^(ref c) far, 2^k near) to the new one (2^(m c) or 2^nk)
      const float d = far ? (go_far ? (ref - m) * c : fmaf(ref, c, -nk)) : go_far ? -fmaf(m, c, -k) : k - nk, r = ex2(d);
      const f2 r2 = pack2(r, r);
      if (ENTROPY) U = r > 0.f ? mul2(r2, fma2(R, pack2(d, d), U)) : 0ull;
      R = mul2(R, r2);
    } else {
      R = U = 0ull;                                    // masked elements only so far
    }
    far = go_far;
    k = nk;
    ref = m;
    limit = m + kReferenceRise / c;
  }

  template <int N>
  __device__ __forceinline__ void add(Unit<T> (&u)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (EXACT) Elem<T>::order(M, u[i].w[j]);
        else M = Elem<T>::larger(M, u[i].w[j]);
      }
    float m0, m1;
    unpack2(Elem<T>::widen(M), m0, m1);
    const float m = fmaxf(m0, m1);
    if (m > limit) move_reference(m);                  // the first live element, or far above the reference
    const f2 cc = pack2(c, c);
    if (far) {
      const f2 nref = pack2(-ref, -ref);
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) accumulate(mul2(add2(Elem<T>::widen(u[i].w[j]), nref), cc), true);
    } else {
      const f2 nk = pack2(-k, -k);
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (ENTROPY) u[i].w[j] = Elem<T>::lift(u[i].w[j]);
          accumulate(fma2(Elem<T>::widen(u[i].w[j]), cc, nk), !Elem<T>::kLifts);
        }
    }
  }

  __device__ __forceinline__ void accumulate(f2 d, bool clamp) {
    float d0, d1;
    unpack2(d, d0, d1);
    const f2 e = pack2(ex2(d0), ex2(d1));
    R = add2(R, e);
    if (ENTROPY) U = fma2(e, clamp ? pack2(max_nan(d0, -200.f), max_nan(d1, -200.f)) : d, U);   // 2^-200 is 0 in float32
  }

  // For callers that want the largest element of each of several segments: ends one (its largest is top() before the call), and
  // folds it into `all`, the largest element so far; finish() is called with M = all.
  __device__ __forceinline__ void close_segment(typename Elem<T>::Word& all) {
    typename Elem<T>::Word lo = M;
    Elem<T>::order(all, lo);
    if (far) {
      accumulate(mul2(add2(Elem<T>::widen(lo), pack2(-ref, -ref)), pack2(c, c)), true);
    } else {
      if (ENTROPY) lo = Elem<T>::lift(lo);
      accumulate(fma2(Elem<T>::widen(lo), pack2(c, c), pack2(-k, -k)), !Elem<T>::kLifts);
    }
    M = Elem<T>::lowest();
  }

  // Largest element seen (-inf if none; NaN if there was one).
  __device__ __forceinline__ float top() const {
    float a, b;
    unpack2(Elem<T>::widen(M), a, b);
    return max_nan(a, b);
  }

  __device__ __forceinline__ State finish() const {
    float a, b, r0, r1, u0, u1;
    unpack2(Elem<T>::widen(M), a, b);
    unpack2(R, r0, r1);
    unpack2(U, u0, u1);
    const float hi = max_nan(a, b), lo = min_nan(a, b);
    if (hi == -kInf) return State{hi, 0.f, 0.f};
    if (!(hi < kInf)) return State{0.f, nan_value(), nan_value()};
    const float d = far ? (ref - hi) * c : -fmaf(hi, c, -k), r = ex2(d);
    State s;
    s.m = hi;
    s.R = (r0 + r1) * r;
    s.U = ENTROPY ? r * (u0 + u1) + r * d * (r0 + r1) : 0.f;
    if (EXACT) {                                        // the smaller half's largest is an element of the sum like others
      const float dl = (lo - hi) * c, el = ex2(dl);
      s.R += el;
      if (ENTROPY && el > 0.f) s.U += el * dl;
    } else {
      s.R -= 1.f;
    }
    return s;
  }
};

__device__ __forceinline__ State shuffle_down(const State& s, int by, int width) {
  return State{__shfl_down_sync(0xffffffffu, s.m, by, width), __shfl_down_sync(0xffffffffu, s.R, by, width),
               __shfl_down_sync(0xffffffffu, s.U, by, width)};
}

// The same with one barrier, which the caller has: each warp's state before it, the block's in every lane of the calling
// warp behind it.
__device__ __forceinline__ void join_warp(State s, float c, State* per_warp) {
#pragma unroll
  for (int o = 16; o; o >>= 1) s = merge(s, shuffle_down(s, o, 32), c);
  if ((threadIdx.x & 31) == 0) per_warp[threadIdx.x >> 5] = s;
}
template <int NT>
__device__ __forceinline__ State join_warps(const State* per_warp, float c) {
  constexpr int W = NT / 32;
  const int lane = threadIdx.x & 31;
  State s = lane < W ? per_warp[lane] : State{-kInf, 0.f, 0.f};
#pragma unroll
  for (int o = 16; o; o >>= 1)
    if (o < W) s = merge(s, shuffle_down(s, o, 32), c);
  return State{__shfl_sync(0xffffffffu, s.m, 0), __shfl_sync(0xffffffffu, s.R, 0), __shfl_sync(0xffffffffu, s.U, 0)};
}

// Joins the threads' states in a fixed order; the result is in *out (shared memory) after a __syncthreads().
template <int NT>
__device__ __forceinline__ void join_block(State s, float c, State* per_warp, State* out) {
#pragma unroll
  for (int o = 16; o; o >>= 1) s = merge(s, shuffle_down(s, o, 32), c);
  if ((threadIdx.x & 31) == 0) per_warp[threadIdx.x >> 5] = s;
  sync_threads<NT>();
  if (threadIdx.x < 32) {
    constexpr int W = NT / 32;
    s = threadIdx.x < W ? per_warp[threadIdx.x] : State{-kInf, 0.f, 0.f};
#pragma unroll
    for (int o = 16; o; o >>= 1)
      if (o < W) s = merge(s, shuffle_down(s, o, 32), c);
    if (threadIdx.x == 0) *out = s;
  }
}

// ---- clusters --------------------------------------------------------------------------------------------------

__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}
// Address of this block's shared variable `p` as it is in block `rank` of the cluster.
__device__ __forceinline__ uint32_t remote_shared(const void* p, unsigned rank) {
  uint32_t a = (uint32_t)__cvta_generic_to_shared(p), r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  return r;
}
__device__ __forceinline__ float load_remote(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ unsigned long long load_remote64(uint32_t a) {
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
  return v;
}
// State of all blocks of the cluster (`parts`: a power of two up to eight), the same in every thread of every block.  Whole
// warps, behind cluster_sync().
__device__ __forceinline__ State join_cluster(const State* mine, int parts, float c) {
  const int lane = threadIdx.x & 31;
  State s{-kInf, 0.f, 0.f};
  if (lane < parts)
    s = State{load_remote(remote_shared(&mine->m, lane)), load_remote(remote_shared(&mine->R, lane)), load_remote(remote_shared(&mine->U, lane))};
  for (int o = parts >> 1; o; o >>= 1) s = merge(s, shuffle_down(s, o, 32), c);
  return State{__shfl_sync(0xffffffffu, s.m, 0), __shfl_sync(0xffffffffu, s.R, 0), __shfl_sync(0xffffffffu, s.U, 0)};
}

// ln z of a positive float64, to the precision of a float32's logarithm of what is left of the nearest power of two (6e-8): the
// 64-bit function is a chain of microseconds for the one warp that needs it.
__device__ __forceinline__ double ln_wide(double z) {
  const long long b = __double_as_longlong(z);
  const int e = (int)(b >> 52) - 1023;                               // z is normal and positive, or NaN or +inf
  const double m = __longlong_as_double((b & 0x000fffffffffffffll) | 0x3ff0000000000000ll);
  if (!(z > 0.0) || !(z < 1.7e308)) return z == 0.0 ? -(double)kInf : z;   // 0, NaN, +inf
  return (double)e * 0.69314718055994530942 + (double)log1pf((float)(m - 1.0));
}

// Whole number in the order of the values (NaN aside); -0 equals +0.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

}  // namespace rows
}  // namespace remoe
