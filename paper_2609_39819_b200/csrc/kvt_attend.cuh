// kvt_attend.cuh — what the kernels on the paged KV pool share: lengths and slots of a batch, waits, loads of a block, matrix
// instructions.
#pragma once
#include "kvt_attend.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace kvt {

typedef uint8_t u8;
typedef uint16_t u16;
typedef uint32_t u32;
typedef uint64_t u64;

constexpr u32 BT = 16;   // tokens of a block

__device__ __forceinline__ void kv_err(u32 *err, u32 bits) { atomicOr(err, bits); }

template <class T> struct Elem;
template <> struct Elem<__nv_bfloat16> {
  typedef __nv_bfloat162 T2;
  static __device__ __forceinline__ float2 up(u32 x) { return __bfloat1622float2(*reinterpret_cast<T2 *>(&x)); }
  static __device__ __forceinline__ u32 down(float a, float b) { T2 r = __floats2bfloat162_rn(a, b); return *reinterpret_cast<u32 *>(&r); }
  static __device__ __forceinline__ float up1(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 down1(float x) { return __float2bfloat16_rn(x); }
  // powers (see raise_or_lower)
  static constexpr float AIM = 0.0f, HIGH = 8.0f, LOW = -INFINITY;
};
template <> struct Elem<__half> {
  typedef __half2 T2;
  static __device__ __forceinline__ float2 up(u32 x) { return __half22float2(*reinterpret_cast<T2 *>(&x)); }
  static __device__ __forceinline__ u32 down(float a, float b) { T2 r = __floats2half2_rn(a, b); return *reinterpret_cast<u32 *>(&r); }
  static __device__ __forceinline__ float up1(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half down1(float x) { return __float2half_rn(x); }
  static constexpr float AIM = 8.0f, HIGH = 15.9f, LOW = -4.0f;
};

// The new tokens [t0, t0 + n) of sequence s and the tokens it holds, cut to what the arrays can hold.
struct Seq { u32 t0, n, kv; };
__device__ __forceinline__ Seq load_seq(const KvBatch &b, u32 s, u32 *err) {
  const u32 a = b.q_start[s], z = b.q_start[s + 1], kv = b.kv_len[s];
  const u64 room = (u64)b.max_blocks * BT;
  Seq r;
  r.t0 = min(a, b.n_tokens);
  r.n = max(min(z, b.n_tokens), r.t0) - r.t0;
  r.kv = (u32)min((u64)kv, room);
  if (z < a || z > b.n_tokens || kv > room) kv_err(err, KVERR_RANGE);
  return r;
}

// Address of a slot's chunk; nullptr for an id beyond both pools.
__device__ __forceinline__ u8 *slot_ptr(const KvPools &p, const KvRow &r, u32 slot) {
  if (slot < p.n_slots) return r.base + slot * p.slot_stride;
  slot -= p.n_slots;
  return slot < p.n_tail ? r.tail + slot * p.tail_stride : nullptr;
}

// Where token t goes; the whole CTA, or one warp, asks. Every thread compares some of the starts with t, so the sequence is
// found with one round of loads instead of a chain of them.
struct Where { u32 seq, index; bool ok; };
template <bool WARP>
__device__ __forceinline__ Where find_token(const KvBatch &b, u32 t, u32 *err) {
  u32 seq = 0;
  if (t == 0)                                        // one of the tokens looks all starts over
    for (u32 s = threadIdx.x % (WARP ? 32 : blockDim.x); s < b.n_seqs; s += WARP ? 32 : blockDim.x)
      if (b.q_start[s] > b.q_start[s + 1]) kv_err(err, KVERR_RANGE);
  if (WARP) {
    for (u32 s0 = 0; s0 < b.n_seqs; s0 += 32) {
      const u32 s = s0 + (threadIdx.x & 31);
      seq += __popc(__ballot_sync(~0u, s < b.n_seqs && b.q_start[s + 1] <= t));
    }
  } else for (u32 s0 = 0; s0 < b.n_seqs; s0 += blockDim.x) {
    const u32 s = s0 + threadIdx.x;
    seq += __syncthreads_count(s < b.n_seqs && b.q_start[s + 1] <= t);
  }
  Where w{seq, 0, false};
  if (seq >= b.n_seqs) return w;                     // behind the last sequence
  const u32 a = b.q_start[seq], z = b.q_start[seq + 1], kv = b.kv_len[seq];
  const bool cut = t < a || t >= z || z > b.n_tokens || kv > (u64)b.max_blocks * BT || kv < z - a;
  w.index = kv - (z - t);
  // starts that decrease; a token in front of the sequence's first place or behind its last block
  w.ok = t >= a && t < z && kv >= z - t && w.index / BT < b.max_blocks;
  if (cut && threadIdx.x % (WARP ? 32 : blockDim.x) == 0) kv_err(err, KVERR_RANGE);
  return w;
}

// The sequence a token lies in; ~0 for none. A whole warp asks.
__device__ __forceinline__ u32 seq_of_token(const KvBatch &b, u32 t) {
  const u32 lane = threadIdx.x & 31;
  for (u32 s0 = 0; s0 < b.n_seqs; s0 += 32) {
    const u32 s = s0 + lane;
    const u32 hit = __ballot_sync(~0u, s < b.n_seqs && b.q_start[s] <= t && t < b.q_start[s + 1]);
    if (hit) return s0 + __ffs(hit) - 1;
  }
  return ~0u;
}
// Finds the sequence a tile belongs to: tiles are numbered sequence by sequence. All threads of the CTA take part.
// Returns false behind the last tile.
template <u32 THREADS>
__device__ bool find_tile(const KvBatch &b, u32 group, u32 *err, u32 rows, u32 want, Seq &q, u32 &seq, u32 &tile) {
  __shared__ u32 s_sum[THREADS / 32], s_seq, s_tile;
  const u32 lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) s_seq = 0xFFFFFFFFu;
  u32 base = 0;
  for (u32 s0 = 0; s0 < b.n_seqs; s0 += THREADS) {
    const u32 s = s0 + threadIdx.x;
    u32 n = 0;
    if (s < b.n_seqs) { const Seq x = load_seq(b, s, err); n = (u32)(((u64)x.n * group + rows - 1) / rows); }
    u32 incl = n;
#pragma unroll
    for (u32 o = 1; o < 32; o *= 2) { const u32 y = __shfl_up_sync(~0u, incl, o); if (lane >= o) incl += y; }
    __syncthreads();
    if (lane == 31) s_sum[warp] = incl;
    __syncthreads();
    u32 before = base, all = base;
#pragma unroll
    for (u32 w = 0; w < THREADS / 32; ++w) { if (w < warp) before += s_sum[w]; all += s_sum[w]; }
    if (want >= before + incl - n && want < before + incl) { s_seq = s; s_tile = want - (before + incl - n); }
    base = all;
  }
  __syncthreads();
  seq = s_seq;
  if (seq == 0xFFFFFFFFu) return false;
  tile = s_tile;
  q = load_seq(b, seq, err);
  return true;
}

// Keys row `token` (0 = first new token) sees: [lo, hi).
__device__ __forceinline__ void row_range(const AttendArgs &a, const Seq &q, u32 token, u32 &lo, u32 &hi) {
  const long long own = (long long)q.kv - q.n + token;     // index of the token in its sequence; < 0: it has none
  hi = a.full ? q.kv : own < 0 ? 0u : (u32)own + 1;
  lo = a.window && hi > a.window ? hi - a.window : 0u;
}

// ------------------------------------------------------------------------------------------------------
// Shared by the kernels that read the pool with TMA.
// ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ u32 smem_addr(const void *p) { return (u32)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(u32 bar, u32 count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count)); }
__device__ __forceinline__ void bar_expect(u32 bar, u32 bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(u32 bar, u32 parity) {
  u32 done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
// Waits for the barrier's phase, for a second at most. For what hardware does: a copy, a product, a cluster-launch answer, all of
// which take microseconds. (Warps that wait for one another's work: tc_wait.)
constexpr u64 WAIT_NS = 1000000000ull;
__device__ __forceinline__ u64 now_ns() { u64 t; asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t)); return t; }
__device__ __forceinline__ bool bar_wait_slow(u32 bar, u32 parity) {
  const u64 t0 = now_ns();
  do {
    for (u32 i = 0; i < 64; ++i) if (bar_try(bar, parity)) return true;
  } while (now_ns() - t0 < WAIT_NS);
  return false;
}
__device__ __forceinline__ bool bar_wait(u32 bar, u32 parity) { return bar_try(bar, parity) || bar_wait_slow(bar, parity); }

// One head of one block's K or V (chunk 2 * layer or 2 * layer + 1) into shared memory. A slot beyond both pools reads as
// zeros: its coordinate lies behind the pool's last slot.
__device__ __forceinline__ void load_block(const AttendArgs &a, const KvMaps &m, u32 dst, u32 bar, u32 slot, u32 chunk, u32 h, u32 halves) {
  const bool tail = slot >= a.p.n_slots && slot - a.p.n_slots < a.p.n_tail;
  const CUtensorMap *map = tail ? &m.tail : &m.pool;
  u32 c3 = 2 * chunk, c4 = tail ? slot - a.p.n_slots : min(slot, a.p.n_slots);
  if (!tail && a.layer_major) { c3 = 2 * c4; c4 = chunk; }
  asm volatile("cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
               ::"r"(dst), "l"(map), "r"(0), "r"(0), "r"(h * halves), "r"(c3), "r"(c4), "r"(bar) : "memory");
}

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// A row's powers 2^(s - m) and their sums are relative to a number m that follows the largest score `top` of each step at a
// distance: powers are between 2^LOW and 2^HIGH where a step's largest, and only when a step leaves that range is m moved, to
// top - AIM, and what has been summed up multiplied by 2^(old m - new m); most steps then need no rescaling. The result does not
// depend on m but for rounding: sums and m go together, wherever m is.
//   bf16  has the exponents of a 32-bit number: m rises once a score passes it by 2^8, and never falls.
//   fp16  ends at 2^16 and has a fixed step of 2^-24 below 2^-14. Powers of at most 1 would lose keys that are 2^25 below the
//         largest, which a long context can have enough of to make the result (behind a first key that takes nearly all of
//         the weight and whose value is small, for one). So the largest power aims at 2^8, and where a step's largest is
//         below 2^-4, m falls: what a step of 128 keys loses to the fixed step is then below 128 * 2^-25 * 2^4 = 2^-14 of the
//         step's largest power. (With 2^12 as the aim m moves more often: 8192-token prompt 485 us, with 2^8 454, before m
//         could fall 456.) m does not fall where that would bring a sum of powers above LIMIT = 2^90 (sums of powers times values, of all
//         parts together too, then stay below 2^120): what is that far below has no weight in 32 bits either.
constexpr float LIMIT = 0x1p90f;
template <class T> __device__ __forceinline__ bool must_fall(float m, float top) { return Elem<T>::LOW > -INFINITY && top < m + Elem<T>::LOW && top > -INFINITY; }
template <class T> __device__ __forceinline__ bool must_move(float m, float top) { return top > m + Elem<T>::HIGH || must_fall<T>(m, top); }
// Moves m; sum: the row's sum of powers so far. Returns what the sums are to be multiplied by.
template <class T> __device__ __forceinline__ float raise_or_lower(float &m, float top, float sum) {
  const bool fall = must_fall<T>(m, top);
  float next = fall ? top - Elem<T>::AIM : fmaxf(m, top - Elem<T>::AIM), f = next == -INFINITY ? 1.0f : ex2(m - next);
  if (fall && sum * f > LIMIT) { next = m; f = 1.0f; }
  m = next;
  return f;
}

template <class T> __device__ __forceinline__ void mma16816(float (&c)[4], const u32 (&a)[4], u32 b0, u32 b1);
template <> __device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], const u32 (&a)[4], u32 b0, u32 b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma16816<__half>(float (&c)[4], const u32 (&a)[4], u32 b0, u32 b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldm4(u32 (&r)[4], u32 addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldm4t(u32 (&r)[4], u32 addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Place of (token r, 16 bytes c of the head) in a loaded block: [r / 8][c / 8][r % 8][c % 8], swizzled.
template <u32 D> __device__ __forceinline__ u32 block_off(u32 r, u32 c) {
  return (r / 8) * (D * 16) + (c / 8) * 1024 + (r % 8) * 128 + (((c % 8) ^ (r % 8)) * 16);
}

// Heads that are not 64 or 128 wide, or not as TMA wants them: one head of one block, whole warp, in the same places; columns
// behind the head stay as they are. A slot beyond both pools reads as zeros.
template <u32 D>
__device__ __forceinline__ void copy_block(const AttendArgs &a, const KvRow &row, u32 slot, u32 h, u32 dst) {
  const u32 d = a.p.head_dim, n = (d + 7) / 8, lane = threadIdx.x & 31;
  const u8 *const src = slot_ptr(a.p, row, slot);
  const u64 pitch = (u64)a.p.n_kv_heads * d;             // elements
  const bool vec = src && d % 8 == 0 && ((uintptr_t)src & 15) == 0;
  u32 r = lane / n, c = lane % n;
  while (r < BT) {
    const u32 to = dst + block_off<D>(r, c);
    const u16 *const p = (const u16 *)src + (src ? r * pitch + (u64)h * d + c * 8 : 0);
    if (vec) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(p) : "memory");
    } else {
      u32 x[4] = {0, 0, 0, 0};
      if (src)
#pragma unroll
        for (u32 y = 0; y < 8; ++y) if (c * 8 + y < d) x[y / 2] |= (u32)p[y] << (y % 2 * 16);
      asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
    }
    r += 32 / n; c += 32 % n;
    if (c >= n) { c -= n; ++r; }
  }
}

constexpr u32 TC_TILE = 128;      // rows of a tcgen05 instruction
__device__ __forceinline__ void bar_arrive(u32 bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool elect_one() {
  u32 p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void tc_commit(u32 bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Shared-memory operand with 128-byte swizzle (bits 61-63 = 2; bit 46 = version 1): lbo, sbo = distances in bytes between 64-element
// parts / between groups of 8 rows.
__device__ __forceinline__ u64 tc_desc(u32 addr, u32 lbo, u32 sbo) {
  return (u64)((addr & 0x3FFFF) >> 4) | (u64)(lbo >> 4) << 16 | (u64)(sbo >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// Instruction descriptor of kind::f16: 32-bit sums, 128 rows, n columns; second operand with its columns (false: its sum
// index) in the outer place of shared memory.
__device__ __forceinline__ u32 tc_idesc(bool fp16, u32 n, bool b_transposed) {
  const u32 t = fp16 ? 0u : 1u;
  return 1u << 4 | t << 7 | t << 10 | (b_transposed ? 1u : 0u) << 16 | (n >> 3) << 17 | (TC_TILE >> 4) << 24;
}
__device__ __forceinline__ void tc_mma_ss(u32 d, u64 a, u64 b, u32 idesc, u32 acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void tc_mma_ts(u32 d, u32 a, u64 b, u32 idesc, u32 acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
#define TC_R4(f, x, i) f(x[i]), f(x[i + 1]), f(x[i + 2]), f(x[i + 3])
#define TC_R16(f, x, i) TC_R4(f, x, i), TC_R4(f, x, i + 4), TC_R4(f, x, i + 8), TC_R4(f, x, i + 12)
__device__ __forceinline__ void tc_ld32(u32 *r, u32 addr) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
               "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : TC_R16("=r", r, 0), TC_R16("=r", r, 16) : "r"(addr));
}
__device__ __forceinline__ void tc_st32(u32 addr, const u32 *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
               "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
               ::"r"(addr), TC_R16("r", r, 0), TC_R16("r", r, 16) : "memory");
}

__device__ __forceinline__ void tc_ld16(u32 *r, u32 addr) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : TC_R16("=r", r, 0) : "r"(addr));
}
__device__ __forceinline__ void tc_st16(u32 addr, const u32 *r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(addr), TC_R16("r", r, 0) : "memory");
}

__device__ __forceinline__ void st_global32(void *p, const u32 *x) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]) : "memory");
}

// Two 32-bit numbers at a time.
__device__ __forceinline__ u64 pack2(float a, float b) { u64 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float2 unpack2(u64 x) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x)); return r; }
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) { u64 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ u64 add2(u64 a, u64 b) { u64 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }

// What ends the waits of a CTA's warps for one another: another warp has given up, or the time is over. A warp may have to wait
// until the others are through with up to TC_JOBS jobs, each as long as a table row at most: 16 keys take 0.25 us (both tiles,
// at 1.5 GHz), so a job on 258 K keys 4 ms, and a second would be over at 64 M keys. Per block of a table row 4 us more are four times that.
constexpr u64 WAIT_BLOCK_NS = 4000;
__device__ __forceinline__ bool tc_wait_slow(u32 bar, u32 parity, volatile u32 *lost, u32 blocks) {
  const u64 t0 = now_ns(), limit = WAIT_NS + WAIT_BLOCK_NS * blocks;
  do {
    for (u32 i = 0; i < 32; ++i) if (bar_try(bar, parity)) return true;
    if (*lost) return false;
  } while (now_ns() - t0 < limit);
  *lost = 1;
  return false;
}
__device__ __forceinline__ bool tc_wait1(u32 bar, u32 parity, volatile u32 *lost, u32 blocks) { return bar_try(bar, parity) || tc_wait_slow(bar, parity, lost, blocks); }
// Whole warps wait, and come back with one answer.
__device__ __forceinline__ bool tc_wait(u32 bar, u32 parity, volatile u32 *lost, u32 blocks) {
  return __all_sync(~0u, bar_try(bar, parity) || tc_wait_slow(bar, parity, lost, blocks));
}

// Dynamic shared memory above 48 KB is asked for once per kernel and engine (a runtime call of half a microsecond).
template <class K>
cudaError_t allow_smem(K kern, u32 which, u32 bytes, u64 *allowed) {
  if (*allowed >> which & 1) return cudaSuccess;
  const cudaError_t r = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (r == cudaSuccess) *allowed |= 1ull << which;
  return r;
}

}  // namespace kvt
