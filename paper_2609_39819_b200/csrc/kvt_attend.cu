// kvt_attend.cu — model-side operators on the paged KV pool: rotation + append of new tokens, attention of new tokens
// over everything their sequences hold in the pool.
#include "kvt_attend.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda/ptx>

#include <algorithm>

namespace kvt {

typedef uint8_t u8;
typedef uint16_t u16;
typedef uint32_t u32;
typedef uint64_t u64;

constexpr u32 BT = 16;   // tokens of a block

__device__ __forceinline__ void kv_err(u32 *err, u32 bits) { atomicOr(err, bits); }

__global__ void k_take_error(u32 *err, u32 *out) { *out = atomicExch(err, 0u); }
cudaError_t launch_take_error(u32 *err, u32 *out, cudaStream_t s) {
  k_take_error<<<1, 1, 0, s>>>(err, out);
  return cudaGetLastError();
}

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

// ======================================================================================================
// Append: rotation of q and k by the tokens' positions, k and v into the blocks.
// ======================================================================================================
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

// Cosine and sine of pair j's angle at the token: position * freq is formed in turns and reduced in 64 bits (a position of
// 2^18 at frequency 1 would leave 32-bit angles 0.02 radians off), the rest is 32-bit work.
__device__ __forceinline__ float2 pair_angle(const AppendArgs &a, u32 t, u32 index, u32 j) {
  u32 axis = a.axis_of ? a.axis_of[j] : 0;
  if (a.axis_of && axis >= a.n_axes) { kv_err(a.err, KVERR_RANGE); axis = 0; }
  const double pos = a.positions ? (double)a.positions[axis * a.pos_stride + t] : (double)index;
  double turns = pos * (a.freqs[j] * 0.15915494309189533577);
  turns -= rint(turns);
  float s, c;
  sincospif(2.0f * (float)turns, &s, &c);
  return make_float2(c, s);
}

// One element (or one pair) at a time: any head size, stride and alignment. Bound by the number of its loads and stores of two bytes:
// 8192 tokens of 32 + 16 heads of 128 an odd distance apart 84 us (the 16-byte kernel 39), of heads of 72 51 us (floor 17).
template <class T>
__global__ void __launch_bounds__(128) k_append_any(AppendArgs a) {
  extern __shared__ float2 cs[];
  const u32 t = blockIdx.x;
  const Where w = find_token<false>(a.b, t, a.err);
  if (w.seq >= a.b.n_seqs) return;
  const u32 half = a.rot_dim / 2;
  for (u32 j = threadIdx.x; j < half; j += blockDim.x) cs[j] = pair_angle(a, t, w.index, j);
  const u32 D = a.p.head_dim, H = a.p.n_kv_heads;
  T *kd = nullptr, *vd = nullptr;
  if (w.ok) {
    const u32 slot = a.b.table[w.seq * a.b.table_stride + w.index / BT];
    kd = (T *)slot_ptr(a.p, a.p.k, slot);
    vd = (T *)slot_ptr(a.p, a.p.v, slot);
    if (!kd) { if (threadIdx.x == 0) kv_err(a.err, KVERR_RANGE); }
    else { const u64 off = (u64)(w.index % BT) * H * D; kd += off; vd += off; }
  }
  __syncthreads();
  const u32 rest = D - a.rot_dim, per = half + rest;   // work items of a rotated head
  auto rotate = [&](const T *x, T *y, u32 i) {
    if (i < half) {
      const u32 u = a.interleaved ? 2 * i : i, v = a.interleaved ? 2 * i + 1 : i + half;
      const float p = Elem<T>::up1(x[u]), q = Elem<T>::up1(x[v]);
      const float2 f = cs[i];
      y[u] = Elem<T>::down1(p * f.x - q * f.y);
      y[v] = Elem<T>::down1(q * f.x + p * f.y);
    } else {
      y[a.rot_dim + i - half] = x[a.rot_dim + i - half];
    }
  };
  for (u32 i = threadIdx.x; i < a.n_q_heads * per; i += blockDim.x) {
    const u32 h = i / per;
    rotate((const T *)a.q + t * a.q_ts + h * a.q_hs, (T *)a.q_out + t * a.qo_ts + h * a.qo_hs, i - h * per);
  }
  if (!kd) return;
  for (u32 i = threadIdx.x; i < H * per; i += blockDim.x) {
    const u32 h = i / per;
    rotate((const T *)a.k + t * a.k_ts + h * a.k_hs, kd + h * D, i - h * per);
  }
  for (u32 i = threadIdx.x; i < H * D; i += blockDim.x) {
    const u32 h = i / D;
    vd[i] = ((const T *)a.v)[t * a.v_ts + h * a.v_hs + (i - h * D)];
  }
}

// 16-byte accesses: head_dim and rot_dim multiples of 16, strides of 8 elements, aligned addresses. Memory-bound: q, k and v are
// read once and written once. Work item: 16 elements (two vectors) of a head; with pairs (j, j + rot/2) a rotated item is
// 8 elements from either half, with neighbouring pairs 16 in a row. All loads of a thread's UNROLL items are in flight
// before the token's sines are waited for. GROUP threads work on a token: the whole CTA, or with few heads a warp, so that
// a CTA of four takes four tokens. SHIFT: log2 of a head's items, -1 where that is no whole number.
// Measured (bf16, heads of 128, in a captured graph; call after call in brackets): 8192 tokens of 32 + 16 heads 38.7 us (41.0;
// 201 MB, 79 % of the measured copy bandwidth), 44,130 tokens of 96 + 16 heads 410-420 us (427; 92-94 %), a decode step of
// 32 tokens 4.2 us (launch and two rounds of loads).
template <class T, u32 THREADS, u32 GROUP, u32 UNROLL, int SHIFT>
__global__ void __launch_bounds__(THREADS) k_append_vec(AppendArgs a) {
  extern __shared__ float2 cs_all[];
  const u32 t = blockIdx.x * (THREADS / GROUP) + threadIdx.x / GROUP, tid = threadIdx.x % GROUP;
  if (t >= a.b.n_tokens) return;         // the last CTA's spare warps
  const u32 D = a.p.head_dim, H = a.p.n_kv_heads, half = a.rot_dim / 2;
  float2 *const cs = cs_all + threadIdx.x / GROUP * half;
  const u32 per = SHIFT < 0 ? D / 16 : 1u << SHIFT, rot_items = a.rot_dim / 16, n_q = a.n_q_heads * per, n_k = H * per, n = n_q + 2 * n_k;
  auto head_of = [&](u32 i) { return SHIFT < 0 ? i / per : i >> SHIFT; };
  const u16 *const tq = (const u16 *)a.q + t * a.q_ts, *const tk = (const u16 *)a.k + t * a.k_ts, *const tv = (const u16 *)a.v + t * a.v_ts;
  // Place of item i: heads are numbered q, k, v one after the other.
  struct Item { u32 head, lo, hi, pair; };               // vectors at lo and hi of the head; pair: its first pair, or ~0
  auto item = [&](u32 i) {
    Item x;
    x.head = head_of(i);
    const u32 c = i - x.head * per;
    const bool turn = c < rot_items && i < n_q + n_k;
    x.pair = turn ? 8 * c : 0xFFFFFFFFu;
    x.lo = turn && !a.interleaved ? 8 * c : 16 * c;
    x.hi = turn && !a.interleaved ? 8 * c + half : 16 * c + 8;
    return x;
  };
  auto source = [&](const Item &x) {
    return x.head < a.n_q_heads ? tq + x.head * a.q_hs
                                : x.head < a.n_q_heads + H ? tk + (x.head - a.n_q_heads) * a.k_hs : tv + (x.head - a.n_q_heads - H) * a.v_hs;
  };
  uint4 in[UNROLL][2];
  const bool inside = t < a.b.q_start[a.b.n_seqs];       // else behind the last sequence: loads nothing, finds nothing below
#pragma unroll
  for (u32 y = 0; y < UNROLL; ++y) {
    const u32 i = tid + y * GROUP;
    if (inside && i < n) {
      const Item x = item(i);
      const u16 *const src = source(x);
      in[y][0] = __ldcs((const uint4 *)(src + x.lo));
      in[y][1] = __ldcs((const uint4 *)(src + x.hi));
    }
  }
  const Where w = find_token<GROUP == 32>(a.b, t, a.err);
  if (w.seq >= a.b.n_seqs) return;
  u16 *kd = nullptr, *vd = nullptr;
  if (w.ok) {
    const u32 slot = a.b.table[w.seq * a.b.table_stride + w.index / BT];
    kd = (u16 *)slot_ptr(a.p, a.p.k, slot);
    vd = (u16 *)slot_ptr(a.p, a.p.v, slot);
    if (!kd) { if (tid == 0) kv_err(a.err, KVERR_RANGE); }
    else { const u64 off = (u64)(w.index % BT) * H * D; kd += off; vd += off; }
  }
  for (u32 j = tid; j < half; j += GROUP) cs[j] = pair_angle(a, t, w.index, j);
  if (GROUP == 32) __syncwarp(); else __syncthreads();
  u16 *const to = (u16 *)a.q_out + t * a.qo_ts;
  auto finish = [&](u32 i, uint4 v0, uint4 v1) {
    const Item x = item(i);
    u32 r0[4] = {v0.x, v0.y, v0.z, v0.w}, r1[4] = {v1.x, v1.y, v1.z, v1.w};
    if (x.pair != 0xFFFFFFFFu) {
      const float4 *f = (const float4 *)(cs + x.pair);   // two pairs' (cosine, sine)
      if (a.interleaved) {
#pragma unroll
        for (u32 y = 0; y < 4; ++y) {
          const float4 g = f[y];
          u32 &p = y < 2 ? r0[2 * y] : r1[2 * y - 4], &q = y < 2 ? r0[2 * y + 1] : r1[2 * y - 3];
          const float2 e = Elem<T>::up(p), o = Elem<T>::up(q);
          p = Elem<T>::down(e.x * g.x - e.y * g.y, e.y * g.x + e.x * g.y);
          q = Elem<T>::down(o.x * g.z - o.y * g.w, o.y * g.z + o.x * g.w);
        }
      } else {
#pragma unroll
        for (u32 y = 0; y < 4; ++y) {
          const float4 g = f[y];
          const float2 e = Elem<T>::up(r0[y]), o = Elem<T>::up(r1[y]);
          r0[y] = Elem<T>::down(e.x * g.x - o.x * g.y, e.y * g.z - o.y * g.w);
          r1[y] = Elem<T>::down(o.x * g.x + e.x * g.y, o.y * g.z + e.y * g.w);
        }
      }
    }
    u16 *d;
    if (i < n_q) d = to + x.head * a.qo_hs;
    else if (!kd) return;
    else d = i < n_q + n_k ? kd + (x.head - a.n_q_heads) * D : vd + (x.head - a.n_q_heads - H) * D;
    *(uint4 *)(d + x.lo) = make_uint4(r0[0], r0[1], r0[2], r0[3]);
    *(uint4 *)(d + x.hi) = make_uint4(r1[0], r1[1], r1[2], r1[3]);
  };
#pragma unroll
  for (u32 y = 0; y < UNROLL; ++y) if (tid + y * GROUP < n) finish(tid + y * GROUP, in[y][0], in[y][1]);
  for (u32 i = tid + UNROLL * GROUP; i < n; i += GROUP) {
    const Item x = item(i);
    const u16 *const src = source(x);
    const uint4 v0 = __ldcs((const uint4 *)(src + x.lo)), v1 = __ldcs((const uint4 *)(src + x.hi));
    finish(i, v0, v1);
  }
}

template <class T, u32 THREADS, u32 GROUP, u32 UNROLL>
static void append_vec(const AppendArgs &a, u32 smem, cudaStream_t s) {
  constexpr u32 TOKENS = THREADS / GROUP;
  const u32 ctas = (a.b.n_tokens + TOKENS - 1) / TOKENS;
  if (a.p.head_dim == 128) k_append_vec<T, THREADS, GROUP, UNROLL, 3><<<ctas, THREADS, smem * TOKENS, s>>>(a);
  else if (a.p.head_dim == 64) k_append_vec<T, THREADS, GROUP, UNROLL, 2><<<ctas, THREADS, smem * TOKENS, s>>>(a);
  else k_append_vec<T, THREADS, GROUP, UNROLL, -1><<<ctas, THREADS, smem * TOKENS, s>>>(a);
}
template <class T>
static void append_vec(const AppendArgs &a, u32 smem, cudaStream_t s) {
  const u64 items = ((u64)a.n_q_heads + 2 * a.p.n_kv_heads) * (a.p.head_dim / 16);
  if (items <= 128) append_vec<T, 128, 32, 4>(a, smem, s);
  else if (items <= 384) append_vec<T, 128, 128, 3>(a, smem, s);
  else append_vec<T, 256, 256, 4>(a, smem, s);
}

cudaError_t launch_append(const AppendArgs &a, cudaStream_t s, u32 *launches) {
  const u32 smem = a.rot_dim / 2 * sizeof(float2);
  ++*launches;
  const u64 strides = a.k_ts | a.k_hs | a.v_ts | a.v_hs | (a.n_q_heads ? a.q_ts | a.q_hs | a.qo_ts | a.qo_hs : 0);
  const uintptr_t bases = (uintptr_t)a.k | (uintptr_t)a.v | (a.n_q_heads ? (uintptr_t)a.q | (uintptr_t)a.q_out : 0);
  if (!(a.p.head_dim % 16 || a.rot_dim % 16 || strides % 8 || bases % 16)) {
    if (a.fp16) append_vec<__half>(a, smem, s);
    else append_vec<__nv_bfloat16>(a, smem, s);
    return cudaGetLastError();
  }
  if (a.fp16) k_append_any<__half><<<a.b.n_tokens, 128, smem, s>>>(a);
  else k_append_any<__nv_bfloat16><<<a.b.n_tokens, 128, smem, s>>>(a);
  return cudaGetLastError();
}

// ======================================================================================================
// Attention. Rows: the (token, query head of the group) pairs of one sequence and one KV head, token-major, so that row r
// is token r / group, head r % group. A CTA takes a tile of consecutive rows, which all read the same K and V once:
//   l = sum_j 2^(s_j - m), o = sum_j 2^(s_j - m) v_j, s_j = scale log2(e) q.k_j, result o / l,
// with m near max_j s_j, over one block of keys after the other: where m moves, l and o are multiplied by 2^(old m - new m).
// Parts of the keys that different warps or CTAs went over are put together by the same rule. Scores, m, l and o are 32-bit numbers.
// ======================================================================================================
// Keys row `token` (0 = first new token) sees: [lo, hi).
__device__ __forceinline__ void row_range(const AttendArgs &a, const Seq &q, u32 token, u32 &lo, u32 &hi) {
  const long long own = (long long)q.kv - q.n + token;     // index of the token in its sequence; < 0: it has none
  hi = a.full ? q.kv : own < 0 ? 0u : (u32)own + 1;
  lo = a.window && hi > a.window ? hi - a.window : 0u;
}

// Blocks of keys that any of the rows r0 .. r1 sees: how many from block b_first on.
__device__ __forceinline__ u32 tile_blocks(const AttendArgs &a, const Seq &q, u32 r0, u32 r1, u32 &b_first) {
  u32 first, last, dummy;
  row_range(a, q, r0 / a.group, first, dummy);
  row_range(a, q, r1 / a.group, dummy, last);
  b_first = first / BT;
  const u32 b_last = (last + BT - 1) / BT;
  return b_last > b_first ? b_last - b_first : 0;
}

// Finds the sequence a tile belongs to: tiles are numbered sequence by sequence. All threads of the CTA take part.
// Returns false behind the last tile.
template <u32 THREADS>
__device__ bool find_tile(const AttendArgs &a, u32 rows, u32 want, Seq &q, u32 &seq, u32 &tile) {
  __shared__ u32 s_sum[THREADS / 32], s_seq, s_tile;
  const u32 lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) s_seq = 0xFFFFFFFFu;
  u32 base = 0;
  for (u32 s0 = 0; s0 < a.b.n_seqs; s0 += THREADS) {
    const u32 s = s0 + threadIdx.x;
    u32 n = 0;
    if (s < a.b.n_seqs) { const Seq x = load_seq(a.b, s, a.err); n = (u32)(((u64)x.n * a.group + rows - 1) / rows); }
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
  q = load_seq(a.b, seq, a.err);
  return true;
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

// Which CTA does what is worked out by every CTA for itself from the device-side lengths, so a captured launch follows
// them. `unit`: one tile of rows of one sequence and KV head, against all its keys. Its number of blocks is bounded per
// sequence (whole sequence, or window plus the tokens of a tile).
__device__ __forceinline__ u32 seq_blocks(const AttendArgs &a, const Seq &q, u32 rows) {
  u32 span = q.kv;
  if (a.window) { const u64 w = (u64)a.window + min(q.n, rows / a.group + 2) + 2 * BT; span = (u32)min((u64)span, w); }
  return max(1u, (span + BT - 1) / BT);
}
__device__ __forceinline__ u32 seq_tiles(const AttendArgs &a, const Seq &q, u32 rows) { return (u32)(((u64)q.n * a.group + rows - 1) / rows); }

// Exclusive prefix sum over the CTA's threads; `all`: the total. Ends without a barrier: s_sum is free after the next one.
template <u32 THREADS>
__device__ __forceinline__ u64 block_scan(u64 n, u64 *s_sum, u64 &all) {
  const u32 lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  u64 incl = n;
#pragma unroll
  for (u32 o = 1; o < 32; o *= 2) { const u64 y = __shfl_up_sync(~0u, incl, o); if (lane >= o) incl += y; }
  __syncthreads();
  if (lane == 31) s_sum[warp] = incl;
  __syncthreads();
  u64 before = 0; all = 0;
#pragma unroll
  for (u32 w = 0; w < THREADS / 32; ++w) { if (w < warp) before += s_sum[w]; all += s_sum[w]; }
  return before + incl - n;
}

// Partial results in scratch: a header, a plan record per sequence, `rows` rows of head_dim sums per partial result, then the
// (maximum, sum) pairs of all of them.
//   kind 1 (few rows): header: the stretches, record {first unit's place in the work (64 bits), length of a unit, -}
//   kind 2:            header {any sequence cut, -}, record {first partial, pieces, tiles, -}
__device__ __forceinline__ uint4 *scratch_plan(const AttendArgs &a) { return (uint4 *)a.scratch; }
__host__ __device__ __forceinline__ u64 plan_bytes(u32 n_seqs) { return (16ull * (n_seqs + 1) + 255) & ~255ull; }
__device__ __forceinline__ float *scratch_sums(const AttendArgs &a) { return (float *)(a.scratch + plan_bytes(a.b.n_seqs)); }

// Kind 1: the blocks of all units, one after the other, are dealt out in stretches, one per CTA, so that every CTA reads as much
// as any other whatever the lengths are; a unit that crosses a border is joined from its parts. Order of units: sequence,
// tile, KV head. A unit counts UNIT_COST blocks more than it has, at its front, for what it costs besides its blocks.
// As many stretches as CTAs run at once, none below MIN_STRETCH. SMs do not get equal shares of the memory's bandwidth (with
// equal stretches the last CTA ends 15 % after the mean), so of long work, LONG_STRETCH blocks per CTA and more, only the
// first four fifths are dealt out like that; the rest goes in two short stretches per CTA to whoever is through first.
constexpr u32 MIN_STRETCH = 8, LONG_STRETCH = 128, UNIT_COST = 8;
struct Stretches {
  u32 per, n1, per2;         // the first n1 are of `per` blocks, the others of `per2`
  __device__ __forceinline__ u64 start(u32 c) const { return c <= n1 ? (u64)c * per : (u64)n1 * per + (u64)(c - n1) * per2; }
  __device__ __forceinline__ u32 of(u64 x) const { const u64 y = (u64)n1 * per; return x < y ? (u32)(x / per) : n1 + (u32)((x - y) / per2); }
};
template <u32 THREADS>
__device__ void find_stretch(const AttendArgs &a, u32 rows, u32 slots, u64 most, bool publish, u64 &x, u64 &total, Stretches &st, u32 &seq, u64 &base) {
  __shared__ u64 s_sum[THREADS / 32], s_base;
  __shared__ u32 s_seq;
  auto units = [&](u32 s) -> u64 {
    if (s >= a.b.n_seqs) return 0;
    const Seq q = load_seq(a.b, s, a.err);
    return (u64)seq_tiles(a, q, rows) * a.p.n_kv_heads * (seq_blocks(a, q, rows) + UNIT_COST);
  };
  u64 all, mine = 0, at = 0;
  total = 0;
  for (u32 s0 = 0; s0 < a.b.n_seqs; s0 += THREADS) {
    mine = units(s0 + threadIdx.x);
    at = block_scan<THREADS>(mine, s_sum, all);
    total += all;
  }
  // More work than non-overlapping sequences can bring (starts that go up and down make the same tokens count again and
  // again): nothing is done. load_seq has set the error word.
  if (total > most) total = 0;
  if (gridDim.x >= 3 * slots && total >= (u64)LONG_STRETCH * slots) {
    st.n1 = slots;
    st.per = (u32)(total * 4 / 5 / slots);
    st.per2 = (u32)((total - (u64)st.per * slots + 2 * slots - 1) / (2 * slots));
  } else {
    const u64 n = max(1ull, min((unsigned long long)min(slots, gridDim.x), (unsigned long long)(total / MIN_STRETCH)));
    st.n1 = (u32)n; st.per = st.per2 = (u32)((total + n - 1) / n);
  }
  x = st.start(blockIdx.x);
  const bool any = x < total;            // else the stretch is empty; seq and base are the first sequence's
  if (publish && threadIdx.x == 0) scratch_plan(a)[0] = make_uint4(st.per, st.n1, st.per2, 0);
  u64 base0 = 0;
  for (u32 s0 = 0; s0 < a.b.n_seqs; s0 += THREADS) {
    const u32 s = s0 + threadIdx.x;
    if (a.b.n_seqs > THREADS) { mine = units(s); at = block_scan<THREADS>(mine, s_sum, all); }
    at += base0;
    if (mine && x >= at && x < at + mine) { s_seq = s; s_base = at; }
    if (publish && s < a.b.n_seqs)
      scratch_plan(a)[1 + s] = make_uint4((u32)at, (u32)(at >> 32), seq_blocks(a, load_seq(a.b, s, a.err), rows) + UNIT_COST, 0);
    base0 += all;
    if (!publish && (!any || x < base0)) break;
  }
  seq = 0; base = 0;
  __syncthreads();
  if (any) { seq = s_seq; base = s_base; }
}

// Kind 2: tiles are cut into pieces, of at most so many blocks. With n pieces in all, the longest of them of p blocks, the
// kernel ends after about the lesser of
//   rounds of one piece per SM, ceil(n / SMs) * (p + c)                          (all pieces alike)
//   the longest piece, or the SMs' mean share and a third of a mean piece        (pieces of all lengths, the longest first)
// with c = PIECE_COST blocks for what a piece costs besides, and joining costs JOIN_COST blocks and a quarter of one per
// partial result. Tried for the longest sequence cut into CUTS[] pieces, and the others into pieces no longer; `most` bounds
// the partial results. Measured: reckoning with a whole longest piece beyond the mean share cuts too often (8 sequences of 1 to
// 246 new tokens on 108 to 4121: 56.7 us, so 47.0; 2 prompts 154 -> 112); shares of 1/4 to 3/4 of a mean piece, c from 10 to 24
// and 24 candidates in the place of 12 differ by 1 to 3 % on average.
// More than 32 sequences are in order 32 by 32 only: two thirds of a mean piece (40 sequences of 60 to 140 tokens on 10 to 3000:
// 91 us, with half the mean share as the piece's length 110). For more than MOST_WEIGHED the search would take longer than it
// gains: pieces of the mean share.
// Every warp takes part with the candidates warp, warp + warps, ...; lane: one of the first 32 sequences.
constexpr u32 PIECE_COST = 12, JOIN_COST = 24, MIN_PIECE = 16, N_CUTS = 12 /* one for each warp */, MOST_WEIGHED = 512;
__constant__ const u8 CUTS[N_CUTS] = {1, 2, 3, 4, 5, 6, 7, 9, 12, 16, 22, 32};
__device__ __forceinline__ u32 cut_length(u32 longest, u32 cuts) { return max(MIN_PIECE, ((longest + cuts - 1) / cuts + 7) / 8 * 8); }   // whole stages
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (u32 o = 16; o; o /= 2) x += __shfl_xor_sync(~0u, x, o);
  return x;
}
struct Cut { u32 longest; float share; bool sound; };    // sound: no more tiles than the host reckons with
__device__ __forceinline__ Cut weigh_cuts(const AttendArgs &a, u32 rows, u32 most, u32 sms, float most_tiles, u32 warp, u32 warps, float *s_cost, Seq &q) {
  const u32 lane = threadIdx.x & 31;
  const float H = a.p.n_kv_heads;
  u32 longest = 1, tiles = 0, nb = 0;
  float blocks = 0.0f, all_tiles = 0.0f;
  q = Seq{0, 0, 0};
  for (u32 s = lane; s < a.b.n_seqs; s += 32) {
    const Seq x = load_seq(a.b, s, a.err);
    if (s == lane) q = x;
    if (!x.n) continue;
    tiles = seq_tiles(a, x, rows); nb = seq_blocks(a, x, rows);
    blocks += (float)tiles * nb; all_tiles += tiles;
    longest = max(longest, nb);
  }
  Cut c;
  c.sound = warp_sum(all_tiles) <= most_tiles * 1.001f;
  c.longest = __reduce_max_sync(~0u, longest);
  c.share = warp_sum(blocks) * H / sms;
  if (c.longest <= MIN_PIECE || !most || a.b.n_seqs > MOST_WEIGHED) return c;
  for (u32 k = warp; k < N_CUTS; k += warps) {
    const u32 piece = k ? cut_length(c.longest, CUTS[k]) : c.longest;
    u32 mine = 0, cut = 0;
    auto count = [&](u32 tiles, u32 nb) {
      const u32 pieces = tiles * ((nb + piece - 1) / piece);
      mine += pieces; cut += nb > piece ? pieces : 0;
    };
    if (a.b.n_seqs <= 32) count(tiles, nb);
    else
      for (u32 s = lane; s < a.b.n_seqs; s += 32) {
        const Seq x = load_seq(a.b, s, a.err);
        if (x.n) count(seq_tiles(a, x, rows), seq_blocks(a, x, rows));
      }
    const float n = __reduce_add_sync(~0u, mine) * H, parts = __reduce_add_sync(~0u, cut) * H;
    const float rounds = ceilf(n / sms) * (piece + PIECE_COST), mean = c.share + n * PIECE_COST / sms;
    float cost = a.b.n_seqs == 1 ? rounds : fminf(rounds, fmaxf(piece + PIECE_COST, mean + (a.b.n_seqs > 32 ? 0.7f : 0.35f) * mean * sms / n));
    if (parts > 0.0f) cost += JOIN_COST + parts * 0.25f;
    if (lane == 0) s_cost[k] = k && parts > most ? INFINITY : cost;
  }
  return c;
}
// The length of a piece; the scheduling warp asks, behind a barrier.
__device__ __forceinline__ u32 choose_cut(const AttendArgs &a, u32 most, const Cut &c, const float *s_cost) {
  if (c.longest <= MIN_PIECE || !most) return c.longest;
  if (a.b.n_seqs > MOST_WEIGHED) return (u32)fminf((float)c.longest, fmaxf((float)MIN_PIECE, ceilf((c.share + 1) / 8) * 8));
  const u32 lane = threadIdx.x & 31, cost = lane < N_CUTS ? __float_as_uint(s_cost[lane]) : ~0u;      // positive: ordered as integers
  const u32 k = __ffs(__ballot_sync(~0u, cost == __reduce_min_sync(~0u, cost))) - 1;
  return k ? cut_length(c.longest, CUTS[k]) : c.longest;
}

// Joining the parts of a row: out = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i. Rows of units that were not cut are already
// written. Launched behind the kernel that leaves the parts, waits for all of it.
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
template <u32 C> __device__ __forceinline__ void load_sums(float (&v)[C], const float *p) {
  if (C == 4) *(float4 *)v = *(const float4 *)p; else *(float2 *)v = *(const float2 *)p;
}

// Kind 1, few rows of many parts: a CTA per row, its warps take the parts in turn. Four warps, or sixteen where short
// stretches make hundreds of parts (258 K tokens, 370 parts at most: 171 us for both kernels against 183).
template <class T, u32 D, u32 WARPS>
__global__ void __launch_bounds__(WARPS * 32) k_attend_join_split(AttendArgs a, u32 n_parts) {
  constexpr u32 C = D / 32, ROWS = 16;   // columns per lane; rows of a tile
  __shared__ float s_acc[WARPS][D], s_l[WARPS], s_m[WARPS];
  const u32 lane = threadIdx.x & 31, warp = threadIdx.x >> 5, H = a.p.n_kv_heads;
  const float *sums = scratch_sums(a);
  const float2 *ml = (const float2 *)(sums + (u64)n_parts * ROWS * D);
  const u64 n_rows = (u64)a.b.n_tokens * a.n_q_heads;
  Stretches str{0, 0, 0};
  for (u64 id = blockIdx.x; id < n_rows; id += gridDim.x) {
    const u32 t = (u32)(id / a.n_q_heads), hq = (u32)(id - (u64)t * a.n_q_heads), seq = seq_of_token(a.b, t);
    const u32 h = hq / a.group;
    if (!str.per) {                      // the batch's arrays are older than the kernel before this one
      asm volatile("griddepcontrol.wait;" ::: "memory");
      const uint4 head = scratch_plan(a)[0];
      str = Stretches{head.x, head.y, head.z};
      if (!str.per) return;
    }
    if (seq == ~0u) continue;
    const uint4 plan = scratch_plan(a)[1 + seq];
    const u32 r = (t - a.b.q_start[seq]) * a.group + hq - h * a.group, tile = r / ROWS, row = r % ROWS;
    const u64 s = ((u64)plan.y << 32 | plan.x) + ((u64)tile * H + h) * plan.z;
    const u32 c0 = str.of(s), c1 = str.of(s + plan.z - 1), n = c1 - c0 + 1, p0 = 2 * c0, odd = s > str.start(c0);
    if (n <= 1) continue;
    if (p0 + 2ull * (n - 1) >= n_parts) { if (lane == 0) kv_err(a.err, KVERR_RANGE); continue; }
    auto place = [&](u32 i) { return (p0 + 2 * i + (i == 0 ? odd : 0)) * ROWS + row; };
    // a warp's parts: warp + y * WARPS, 32 of them at a time, a lane for the maximum and sum of each
    float m = -INFINITY, l = 0.0f, acc[C];
#pragma unroll
    for (u32 c = 0; c < C; ++c) acc[c] = 0.0f;
    for (u32 i0 = warp; i0 < n; i0 += 32 * WARPS) {
      const u32 mine = i0 + lane * WARPS, here = min(32u, (n - i0 + WARPS - 1) / WARPS);
      const float2 x = mine < n ? ml[place(mine)] : make_float2(-INFINITY, 0.0f);
      float now = x.x;
#pragma unroll
      for (u32 o = 16; o; o /= 2) now = fmaxf(now, __shfl_xor_sync(~0u, now, o));
      now = fmaxf(m, now);
      const float ref = now == -INFINITY ? 0.0f : now, f = ex2(m - ref), w = ex2(x.x - ref);    // no keys for this row: weight 2^-inf, zeros
      m = now;
      l = l * f + warp_sum(w * x.y);
#pragma unroll
      for (u32 c = 0; c < C; ++c) acc[c] *= f;
#pragma unroll 8
      for (u32 y = 0; y < here; ++y) {
        float v[C];
        load_sums<C>(v, sums + (u64)place(i0 + y * WARPS) * D + lane * C);
        const float wy = __shfl_sync(~0u, w, y);
#pragma unroll
        for (u32 c = 0; c < C; ++c) acc[c] += wy * v[c];
      }
    }
    __syncthreads();                     // the row before this one is read
#pragma unroll
    for (u32 c = 0; c < C; ++c) s_acc[warp][lane * C + c] = acc[c];
    if (lane == 0) { s_l[warp] = l; s_m[warp] = m; }
    __syncthreads();
    if (warp) continue;
    float all = -INFINITY;
#pragma unroll
    for (u32 w = 0; w < WARPS; ++w) all = fmaxf(all, s_m[w]);
    const float ref = all == -INFINITY ? 0.0f : all, f0 = ex2(m - ref);
    m = all; l *= f0;
#pragma unroll
    for (u32 c = 0; c < C; ++c) acc[c] *= f0;
#pragma unroll
    for (u32 w = 1; w < WARPS; ++w) {
      const float f = ex2(s_m[w] - ref);
      l += f * s_l[w];
#pragma unroll
      for (u32 c = 0; c < C; ++c) acc[c] += f * s_acc[w][lane * C + c];
    }
    const float inv = l > 0.0f ? 1.0f / l : l;
    T *o = (T *)a.out + (u64)t * a.o_ts + (u64)hq * a.o_hs + lane * C;
#pragma unroll
    for (u32 c = 0; c < C; ++c) o[c] = Elem<T>::down1(acc[c] * inv);
    if (a.lse && lane == 0) a.lse[(u64)t * a.n_q_heads + hq] = (m + log2f(l)) * 0.69314718055994531f;
  }
}

// Kind 2, many rows of few parts: a warp takes BATCH heads of a token at a time and keeps the loads of STEP parts of each in
// flight together.
template <class T, u32 D>
__global__ void __launch_bounds__(128) k_attend_join_tc(AttendArgs a, u32 rows, u32 n_parts) {
  constexpr u32 C = D / 32, BATCH = 4, STEP = 4;
  const u32 lane = threadIdx.x & 31, H = a.p.n_kv_heads;
  const float *sums = scratch_sums(a);
  const float2 *ml = (const float2 *)(sums + (u64)n_parts * rows * D);
  const u32 groups = (a.n_q_heads + BATCH - 1) / BATCH, warps = gridDim.x * 4;
  u32 last_t = ~0u, seq = ~0u, start = 0;
  bool waited = false;
  uint4 plan = make_uint4(0, 0, 0, 0);
  for (u64 id = blockIdx.x * 4 + (threadIdx.x >> 5); id < (u64)a.b.n_tokens * groups; id += warps) {
    const u32 t = (u32)(id / groups), hq0 = (u32)(id - (u64)t * groups) * BATCH;
    if (t != last_t) {
      last_t = t;
      seq = seq_of_token(a.b, t);
      if (seq != ~0u) start = a.b.q_start[seq];
      if (!waited) {                     // the batch's arrays are older than the kernel before this one
        asm volatile("griddepcontrol.wait;" ::: "memory");
        waited = true;
        if (!scratch_plan(a)[0].x) return;
      }
      if (seq != ~0u) plan = scratch_plan(a)[1 + seq];
    }
    const u32 n = plan.y, stride = plan.z * H;
    if (seq == ~0u || n <= 1) continue;
    u32 at[BATCH];                       // first partial's row
    float m[BATCH], l[BATCH], acc[BATCH][C];
#pragma unroll
    for (u32 b = 0; b < BATCH; ++b) {
      const u32 hq = min(hq0 + b, a.n_q_heads - 1), h = hq / a.group, r = (t - start) * a.group + hq - h * a.group, tile = r / rows;
      const u32 p0 = (plan.x + tile) * H + h;
      at[b] = (p0 + (u64)(n - 1) * stride < n_parts ? p0 : 0) * rows + r - tile * rows;
      if (p0 + (u64)(n - 1) * stride >= n_parts && lane == 0) kv_err(a.err, KVERR_RANGE);     // cannot happen
      m[b] = -INFINITY; l[b] = 0.0f;
#pragma unroll
      for (u32 c = 0; c < C; ++c) acc[b][c] = 0.0f;
    }
    for (u32 i = 0; i < n; i += STEP) {
      float2 x[STEP][BATCH];
      float v[STEP][BATCH][C];
#pragma unroll
      for (u32 y = 0; y < STEP; ++y)
#pragma unroll
        for (u32 b = 0; b < BATCH; ++b) {
          const u32 p = at[b] + min(i + y, n - 1) * stride * rows;
          x[y][b] = ml[p];
          load_sums<C>(v[y][b], sums + (u64)p * D + lane * C);
        }
#pragma unroll
      for (u32 b = 0; b < BATCH; ++b) {
        float now = m[b];
#pragma unroll
        for (u32 y = 0; y < STEP; ++y) { if (i + y >= n) x[y][b] = make_float2(-INFINITY, 0.0f); now = fmaxf(now, x[y][b].x); }
        const float ref = now == -INFINITY ? 0.0f : now, f = ex2(m[b] - ref);
        m[b] = now;
        l[b] *= f;
#pragma unroll
        for (u32 c = 0; c < C; ++c) acc[b][c] *= f;
#pragma unroll
        for (u32 y = 0; y < STEP; ++y) {
          const float w = ex2(x[y][b].x - ref);        // a part without keys for this row holds zeros, weight 2^-inf
          l[b] += w * x[y][b].y;
          if (i + y < n)
#pragma unroll
            for (u32 c = 0; c < C; ++c) acc[b][c] += w * v[y][b][c];
        }
      }
    }
#pragma unroll
    for (u32 b = 0; b < BATCH; ++b) {
      const u32 hq = hq0 + b;
      if (hq >= a.n_q_heads) break;
      const float inv = l[b] > 0.0f ? 1.0f / l[b] : l[b];
      u16 *o = (u16 *)a.out + (u64)t * a.o_ts + (u64)hq * a.o_hs + lane * C;
      u32 e[C / 2];
#pragma unroll
      for (u32 c = 0; c < C / 2; ++c) e[c] = Elem<T>::down(acc[b][2 * c] * inv, acc[b][2 * c + 1] * inv);
      if (C == 4 && ((uintptr_t)o & 7) == 0) *(uint2 *)o = make_uint2(e[0], e[C / 2 - 1]);
      else {
#pragma unroll
        for (u32 c = 0; c < C; ++c) o[c] = (u16)(e[c / 2] >> (16 * (c % 2)));
      }
      if (a.lse && lane == 0) a.lse[(u64)t * a.n_q_heads + hq] = (m[b] + log2f(l[b])) * 0.69314718055994531f;
    }
  }
}

// ------------------------------------------------------------------------------------------------------
// Few rows (one new token per sequence, small chunks): bound by reading K and V once. A CTA of four warps takes a piece of
// the keys for up to 16 rows of one KV head, the height of a warp-level matrix instruction. Every warp has its own ring
// of TMA loads (a block's K and V per stage) and its own running maximum and sums over every fourth block, so warps
// never wait for one another until the end of a unit. Two CTAs per SM keep up to 192 KB of loads in flight.
// The matrix units idle most of the time (30 % busy), so the warp-level instructions do, whose sums and operands lie in
// registers: nothing has to be handed from one kind of warp to another.
// Measured, heads of 128, 8 KV heads, groups of 4, in a captured graph (call after call in brackets): one token on 258,047 (1.06
// GB) 174-177 us (180) with the join, 6.0 TB/s, 92 % of the measured copy bandwidth; 32 tokens on 2,000 to 130,000 each (6.1 GB,
// groups of 12) 915-922 us (950), 101 %.
// ------------------------------------------------------------------------------------------------------
constexpr u32 SPLIT_ROWS = 16, SPLIT_WARPS = 4, SPLIT_THREADS = SPLIT_WARPS * 32;
template <u32 D> struct SplitShape {
  static constexpr u32 BLOCK = BT * D * 2, STAGES = D == 64 ? 6 : 3, RING = STAGES * 2 * BLOCK, SMEM = SPLIT_WARPS * RING + 1024;
};

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

// The keys in blocks [b0, b1) for rows r0 .. r1 of a sequence: this warp's share of them, every fourth block. o, m, l: sums,
// maximum and sum of powers of rows lane / 4 and lane / 4 + 8, this lane's columns and keys. `it`: stages used so far. false: a
// wait ran out. ANY: heads of any size up to D, filled up with zeros.
template <class T, u32 D, bool ANY = false>
__device__ __forceinline__ bool split_keys(const AttendArgs &a, const KvMaps &maps, const Seq &q, u32 seq, u32 h, u32 r0, u32 r1, u32 b0, u32 b1,
                                           u32 ring, u32 bar0, u32 &it, float (&o)[D / 8][4], float (&m)[2], float (&l)[2]) {
  typedef SplitShape<D> S;
  const u32 lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  u32 first, last, all_lo, all_hi;       // keys any row sees: [first, last), keys every row sees: [all_lo, all_hi)
  row_range(a, q, r0 / a.group, first, all_hi);
  row_range(a, q, r1 / a.group, all_lo, last);
  bool ok = true;
  const u32 n_mine = b0 + warp < b1 ? (b1 - b0 - warp + SPLIT_WARPS - 1) / SPLIT_WARPS : 0;   // blocks b0 + warp + 4 i
  const u32 *row = a.b.table + seq * a.b.table_stride;
  u32 held = 0;                        // lane i: the slot of this warp's block number (i mod 32) of the current 32
  auto load = [&](u32 i) {             // i-th block of this warp here; whole warp
    if (i % 32 == 0) {
      held = i + lane < n_mine ? row[b0 + warp + (i + lane) * SPLIT_WARPS] : 0;
      if (i + lane < n_mine && held >= a.p.n_slots && held - a.p.n_slots >= a.p.n_tail) kv_err(a.err, KVERR_RANGE);
    }
    const u32 slot = __shfl_sync(~0u, held, i % 32);
    if (ANY) {
      const u32 dst = ring + (it + i) % S::STAGES * 2 * S::BLOCK;
      copy_block<D>(a, a.p.k, slot, h, dst);
      copy_block<D>(a, a.p.v, slot, h, dst + S::BLOCK);
    } else if (lane == 0) {
      const u32 st = (it + i) % S::STAGES, bar = bar0 + st * 8, dst = ring + st * 2 * S::BLOCK;
      bar_expect(bar, 2 * S::BLOCK);
      load_block(a, maps, dst, bar, slot, 2 * a.layer, h, D / 64);
      load_block(a, maps, dst + S::BLOCK, bar, slot, 2 * a.layer + 1, h, D / 64);
    }
  };
  if (ANY) {
    const u32 n = (a.p.head_dim + 7) / 8;
    if (n < D / 8)
      for (u32 i = lane; i < S::STAGES * 2 * BT * (D / 8 - n); i += 32) {
        const u32 r = i / (D / 8 - n);
        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(ring + r / BT * S::BLOCK + block_off<D>(r % BT, n + i % (D / 8 - n))), "r"(0) : "memory");
      }
  }
#pragma unroll 1
  for (u32 i = 0; i < S::STAGES; ++i) {
    if (i < n_mine) load(i);
    if (ANY) asm volatile("cp.async.commit_group;" ::: "memory");
  }

  // queries: rows lane / 4 and lane / 4 + 8 of the tile, in the registers of the first operand
  u32 qf[D / 16][4];
  u32 lo[2], hi[2];
#pragma unroll
  for (u32 y = 0; y < 2; ++y) {
    const u32 r = min(r0 + lane / 4 + 8 * y, r1);     // rows behind the last one repeat it and are not written
    row_range(a, q, r / a.group, lo[y], hi[y]);
    const u16 *src = (const u16 *)a.q + (u64)(q.t0 + r / a.group) * a.q_ts + (u64)(h * a.group + r % a.group) * a.q_hs + (lane % 4) * 2;
    const bool even = ((uintptr_t)src & 3) == 0;
#pragma unroll
    for (u32 k = 0; k < D / 16; ++k)
#pragma unroll
      for (u32 z = 0; z < 2; ++z) {
        const u16 *p = src + k * 16 + z * 8;
        if (ANY) {
          const u32 c = (lane % 4) * 2 + k * 16 + z * 8;
          qf[k][y + 2 * z] = (c < a.p.head_dim ? (u32)p[0] : 0u) | (c + 1 < a.p.head_dim ? (u32)p[1] << 16 : 0u);
        } else {
          qf[k][y + 2 * z] = even ? *(const u32 *)p : (u32)p[0] | (u32)p[1] << 16;
        }
      }
  }
  m[0] = m[1] = -INFINITY; l[0] = l[1] = 0.0f;
#pragma unroll
  for (u32 n = 0; n < D / 8; ++n)
#pragma unroll
    for (u32 y = 0; y < 4; ++y) o[n][y] = 0.0f;

  for (u32 i = 0; ok && i < n_mine; ++i) {
    const u32 st = (it + i) % S::STAGES, kb = ring + st * 2 * S::BLOCK, vb = kb + S::BLOCK;
    if (ANY) {
      asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 1) : "memory");
      __syncwarp();
    } else if (!(ok = __all_sync(~0u, bar_wait(bar0 + st * 8, ((it + i) / S::STAGES) & 1)))) break;
    const u32 key0 = (b0 + warp + i * SPLIT_WARPS) * BT;
    // scores of 16 keys: two column groups of 8
    float s[2][4] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
    for (u32 k = 0; k < D / 16; ++k) {
      u32 f[4];
      ldm4(f, kb + block_off<D>((lane / 16) * 8 + lane % 8, 2 * k + (lane / 8) % 2));
      mma16816<T>(s[0], qf[k], f[0], f[1]);
      mma16816<T>(s[1], qf[k], f[2], f[3]);
    }
    // Tokens that no row sees, in front of the window in the first block and behind the length in the last: whatever their
    // values hold, weight 0 must not meet an Inf or a NaN.
    if (key0 < first || key0 + BT > q.kv) {
      const u32 r = lane / 2;
      if (key0 + r < first || key0 + r >= q.kv)
#pragma unroll
        for (u32 c = 0; c < D / 16; ++c)
          asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vb + block_off<D>(r, (lane % 2) * (D / 16) + c)), "r"(0) : "memory");
      if (!ANY) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // a load writes here next
      __syncwarp();
    }
    const bool whole = key0 >= all_lo && key0 + BT <= all_hi;
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (u32 n = 0; n < 2; ++n)
#pragma unroll
      for (u32 y = 0; y < 4; ++y) {
        const u32 key = key0 + n * 8 + (lane % 4) * 2 + (y & 1);
        float v = s[n][y] * a.scale_log2;
        if (!whole && (key < lo[y >> 1] || key >= hi[y >> 1])) v = -INFINITY;
        s[n][y] = v;
        top[y >> 1] = fmaxf(top[y >> 1], v);
      }
#pragma unroll
    for (u32 y = 0; y < 2; ++y) {
      top[y] = fmaxf(top[y], __shfl_xor_sync(~0u, top[y], 1));
      top[y] = fmaxf(top[y], __shfl_xor_sync(~0u, top[y], 2));
    }
    if (__any_sync(~0u, must_move<T>(m[0], top[0]) || must_move<T>(m[1], top[1]))) {
#pragma unroll
      for (u32 y = 0; y < 2; ++y) {
        float all = l[y];                // four lanes hold a row's sum, and must come to the same m
        all = fmaxf(all, __shfl_xor_sync(~0u, all, 1));
        all = fmaxf(all, __shfl_xor_sync(~0u, all, 2));
        const float f = raise_or_lower<T>(m[y], top[y], all);
        l[y] *= f;
#pragma unroll
        for (u32 n = 0; n < D / 8; ++n) { o[n][2 * y] *= f; o[n][2 * y + 1] *= f; }
      }
    }
    const float ref[2] = {m[0] == -INFINITY ? 0.0f : m[0], m[1] == -INFINITY ? 0.0f : m[1]};
#pragma unroll
    for (u32 n = 0; n < 2; ++n)
#pragma unroll
      for (u32 y = 0; y < 4; ++y) { s[n][y] = ex2(s[n][y] - ref[y >> 1]); l[y >> 1] += s[n][y]; }
    // The second product takes powers of the element type. Rounded once they would add a third (bf16) or half (fp16) to the error
    // of the result's own rounding, so they are taken as the sum of two such numbers, which leaves 2^-16 or 2^-22 of a power (or
    // fp16's fixed step): the results are those of 32-bit powers. Loading K and V leaves the matrix units the time, or nearly (bf16,
    // call after call: one token on 1000 8.2 us with and without, on 258 K 175 -> 180, 32 long sessions 924 -> 950). Second numbers in
    // the rows of the operand that are nobody's, where there are that many, save the second product but were slower (182, 957).
    u32 p[4], rest[4];
#pragma unroll
    for (u32 y = 0; y < 4; ++y) {
      const float e0 = s[y / 2][2 * (y % 2)], e1 = s[y / 2][2 * (y % 2) + 1];
      p[y] = Elem<T>::down(e0, e1);
      const float2 z = Elem<T>::up(p[y]);
      rest[y] = Elem<T>::down(e0 - z.x, e1 - z.y);
    }
#pragma unroll
    for (u32 n = 0; n < D / 16; n += 2) {      // a sum's two products some distance apart
      u32 f[2][4];
#pragma unroll
      for (u32 y = 0; y < 2; ++y) ldm4t(f[y], vb + block_off<D>(lane % 16, 2 * (n + y) + lane / 16));
#pragma unroll
      for (u32 y = 0; y < 4; ++y) mma16816<T>(o[2 * n + y], p, f[y / 2][y % 2 * 2], f[y / 2][y % 2 * 2 + 1]);
#pragma unroll
      for (u32 y = 0; y < 4; ++y) mma16816<T>(o[2 * n + y], rest, f[y / 2][y % 2 * 2], f[y / 2][y % 2 * 2 + 1]);
    }
    __syncwarp();                      // the stage is read: refill it
    if (i + S::STAGES < n_mine) load(i + S::STAGES);
    if (ANY) asm volatile("cp.async.commit_group;" ::: "memory");
  }
  it += n_mine;
  return ok;
}
// Leaves the warps' results for the CTA: sums in the (now idle) rings, row pitch split_pitch() floats, maxima and sums in s_ml.
template <u32 D> __device__ __forceinline__ constexpr u32 split_pitch() { return D + 8; }      // four rows of a quarter warp fall on different banks
template <u32 D>
__device__ __forceinline__ void split_leave(u8 *smem_raw, u32 ring, float (&o)[D / 8][4], float (&m)[2], float (&l)[2],
                                            float (&s_ml)[SPLIT_WARPS][SPLIT_ROWS][2]) {
  typedef SplitShape<D> S;
  const u32 lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (u32 y = 0; y < 2; ++y) {
    l[y] += __shfl_xor_sync(~0u, l[y], 1);
    l[y] += __shfl_xor_sync(~0u, l[y], 2);
    if (lane % 4 == 0) { s_ml[warp][lane / 4 + 8 * y][0] = m[y]; s_ml[warp][lane / 4 + 8 * y][1] = l[y]; }
  }
  constexpr u32 LD = split_pitch<D>();
  static_assert(SPLIT_ROWS * LD * 4 <= S::RING, "sums fit a warp's ring");
  float *const so = (float *)(smem_raw + (ring - smem_addr(smem_raw)));
#pragma unroll
  for (u32 n = 0; n < D / 8; ++n)
#pragma unroll
    for (u32 y = 0; y < 2; ++y)
      *(float2 *)&so[(lane / 4 + 8 * y) * LD + n * 8 + (lane % 4) * 2] = make_float2(o[n][2 * y], o[n][2 * y + 1]);
}
// Row r (of 16) as the CTA's four warps have it together: maximum, sum of powers, and the weight of each warp's sums.
__device__ __forceinline__ void split_row(const float (&s_ml)[SPLIT_WARPS][SPLIT_ROWS][2], u32 r, float &mm, float &ll, float (&f)[SPLIT_WARPS]) {
  mm = -INFINITY; ll = 0.0f;
#pragma unroll
  for (u32 y = 0; y < SPLIT_WARPS; ++y) mm = fmaxf(mm, s_ml[y][r][0]);
  const float ref = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
  for (u32 y = 0; y < SPLIT_WARPS; ++y) { f[y] = ex2(s_ml[y][r][0] - ref); ll += f[y] * s_ml[y][r][1]; }
}
template <u32 D>
__device__ __forceinline__ float4 split_sum(const u8 *smem_raw, u32 ring0, u32 r, u32 c, const float (&f)[SPLIT_WARPS]) {
  const float *sum = (const float *)(smem_raw + (ring0 - smem_addr(smem_raw))) + r * split_pitch<D>() + c;
  float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
  for (u32 y = 0; y < SPLIT_WARPS; ++y) {
    const float4 z = *(const float4 *)(sum + y * (SplitShape<D>::RING / 4));
    v.x += f[y] * z.x; v.y += f[y] * z.y; v.z += f[y] * z.z; v.w += f[y] * z.w;
  }
  return v;
}

template <class T, u32 D>
__global__ void __launch_bounds__(SPLIT_THREADS, 2)
k_attend_split(const __grid_constant__ AttendArgs a, const __grid_constant__ KvMaps maps, u32 n_parts, u32 slots, u64 most) {
  typedef SplitShape<D> S;
  extern __shared__ u8 smem_raw[];
  __shared__ __align__(8) u64 bars[SPLIT_WARPS * S::STAGES];
  __shared__ float s_ml[SPLIT_WARPS][SPLIT_ROWS][2];
  __shared__ __align__(16) longlong2 s_next;             // answer to the request for another stretch
  __shared__ __align__(8) u64 s_next_bar;
  asm volatile("griddepcontrol.launch_dependents;");
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = a.p.n_kv_heads;
  const u32 bar0 = smem_addr(bars) + warp * S::STAGES * 8;
  if (lane == 0) {
    for (u32 i = 0; i < S::STAGES; ++i) bar_init(bar0 + i * 8, 1);
    if (warp == 0) bar_init(smem_addr(&s_next_bar), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (tid < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(tid ? &maps.tail : &maps.pool) : "memory");
  u64 x, total, base;
  Stretches str;
  u32 seq, cta = blockIdx.x, taken = 0;                  // whose stretch this is; stretches taken over so far
  find_stretch<SPLIT_THREADS>(a, SPLIT_ROWS, slots, most, n_parts && blockIdx.x == 0, x, total, str, seq, base);
  const u32 ring0 = (smem_addr(smem_raw) + 1023) & ~1023u, ring = ring0 + warp * S::RING;
  Seq q = load_seq(a.b, seq, a.err);
  u32 tiles = seq_tiles(a, q, SPLIT_ROWS), unit = seq_blocks(a, q, SPLIT_ROWS) + UNIT_COST;
  u32 it = 0;                            // stages this warp has used
  bool ok = true;
  const bool steal = n_parts && gridDim.x > slots;       // else all CTAs run at once
  // A CTA that has not been launched yet is called off and its stretch taken over; the answer arrives during the join of the
  // last unit. CTAs with empty stretches do so too, which is sooner over than launching the others.
  auto ask = [&]() {
    if (tid == 0) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      bar_expect(smem_addr(&s_next_bar), 16);
      cuda::ptx::clusterlaunchcontrol_try_cancel(&s_next, &s_next_bar);
    }
  };

  for (;;) {                             // a stretch
    const u64 x_begin = x, x_end = min((unsigned long long)total, (unsigned long long)str.start(cta + 1));
    bool asked = false;
    for (bool more = x < total; more;) {
      // the unit x lies in, and the part of it in this stretch
      while (x >= base + (u64)tiles * H * unit) {
        base += (u64)tiles * H * unit;
        if (++seq >= a.b.n_seqs) return;   // cannot happen: x < x_end <= all work
        q = load_seq(a.b, seq, a.err);
        tiles = seq_tiles(a, q, SPLIT_ROWS); unit = seq_blocks(a, q, SPLIT_ROWS) + UNIT_COST;
      }
      const u32 u = (u32)((x - base) / unit), tile = u / H, h = u % H;
      const u64 u0 = base + (u64)u * unit;
      if (!n_parts && x > u0) {            // nothing is cut (one stretch per CTA): a unit goes whole to the one it begins in
        x = u0 + unit;
        more = x < x_end;
        continue;
      }
      const u64 x1 = n_parts ? min((unsigned long long)x_end, (unsigned long long)(u0 + unit)) : u0 + unit;
      const bool direct = x == u0 && x1 == u0 + unit;
      const u32 part = 2 * cta + (x == u0 && x > x_begin);
      const u32 n_rows = q.n * a.group, r0 = tile * SPLIT_ROWS, r1 = min(r0 + SPLIT_ROWS, n_rows) - 1;
      u32 b_first;
      const u32 nb = tile_blocks(a, q, r0, r1, b_first);
      const u32 o0 = (u32)(x - u0), o1 = (u32)(x1 - u0);
      const u32 b0 = b_first + min(o0 > UNIT_COST ? o0 - UNIT_COST : 0, nb), b1 = b_first + min(o1 > UNIT_COST ? o1 - UNIT_COST : 0, nb);
      float o[D / 8][4], m[2], l[2];
      ok = split_keys<T, D>(a, maps, q, seq, h, r0, r1, b0, b1, ring, bar0, it, o, m, l);
      if (steal && x1 >= x_end) { ask(); asked = true; }

      split_leave<D>(smem_raw, ring, o, m, l, s_ml);
      if (__syncthreads_or(!ok)) { ok = false; break; }      // a wait ran out somewhere: nothing is written
      const u32 r = tid / 8, c0 = (tid % 8) * 4;             // thread: row r, four columns out of every 32
      if (r0 + r <= r1 && (direct || part < n_parts)) {
        float mm, ll, f[SPLIT_WARPS];
        split_row(s_ml, r, mm, ll, f);
        const u32 t = q.t0 + (r0 + r) / a.group, hq = h * a.group + (r0 + r) % a.group;
        const float inv = !direct ? 1.0f : ll > 0.0f ? 1.0f / ll : ll;
        u16 *const out = (u16 *)a.out + (u64)t * a.o_ts + (u64)hq * a.o_hs;
        float *const sums = scratch_sums(a) + ((u64)part * SPLIT_ROWS + r) * D;
#pragma unroll
        for (u32 c = c0; c < D; c += 32) {
          const float4 v = split_sum<D>(smem_raw, ring0, r, c, f);
          if (direct) {
            const u32 p0 = Elem<T>::down(v.x * inv, v.y * inv), p1 = Elem<T>::down(v.z * inv, v.w * inv);
            u16 *d = out + c;
            if (((uintptr_t)d & 7) == 0) *(uint2 *)d = make_uint2(p0, p1);
            else { d[0] = (u16)p0; d[1] = (u16)(p0 >> 16); d[2] = (u16)p1; d[3] = (u16)(p1 >> 16); }
          } else {
            *(float4 *)(sums + c) = v;
          }
        }
        if (tid % 8 == 0) {
          if (!direct) ((float2 *)(scratch_sums(a) + (u64)n_parts * SPLIT_ROWS * D))[part * SPLIT_ROWS + r] = make_float2(mm, ll);
          else if (a.lse) a.lse[(u64)t * a.n_q_heads + hq] = (mm + log2f(ll)) * 0.69314718055994531f;
        }
      } else if (r0 + r <= r1 && tid == 0) {
        kv_err(a.err, KVERR_RANGE);        // cannot happen: two parts per CTA
      }
      x = x1;
      more = x < x_end;
      if (more) {                          // the rings are read: loads may write them again
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
      }
    }
    if (!ok || !steal) break;
    if (!asked) ask();
    if (__syncthreads_or(!bar_wait(smem_addr(&s_next_bar), taken & 1))) { ok = false; break; }
    const longlong2 answer = s_next;
    if (!cuda::ptx::clusterlaunchcontrol_query_cancel_is_canceled(answer)) break;    // there is none left to take
    cta = cuda::ptx::clusterlaunchcontrol_query_cancel_get_first_ctaid_x<u32>(answer);
    ++taken;
    x = str.start(cta);
    if (x < base) {                        // CTAs are called off in ascending order as a rule: then the search goes on from here
      seq = 0; base = 0;
      q = load_seq(a.b, 0, a.err);
      tiles = seq_tiles(a, q, SPLIT_ROWS); unit = seq_blocks(a, q, SPLIT_ROWS) + UNIT_COST;
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // rings and answer are read
    __syncthreads();
  }
  if (!ok) {                             // let the copies in flight land, for a while, before the CTA ends
    if (lane == 0) kv_err(a.err, KVERR_WAIT);
    for (u32 i = 0; i < S::STAGES; ++i) for (u32 y = 0; y < 2; ++y) bar_wait(bar0 + i * 8, y);
    for (u32 y = 0; y < 2; ++y) bar_wait(smem_addr(&s_next_bar), y);
  }
}

// Few units of moderate length: a cluster of CTAs takes a unit, its blocks dealt out evenly, and joins the parts through the
// CTAs' shared memory: one launch, no scratch. Bound by latency: 4 us for the launch, the lengths and the first block, then a
// block of each warp's every 0.8 us, then the join through shared memory. One token, 8 KV heads of 128, groups of 4: 300 cached
// tokens 6.2 us, 1000 7.1, 4000 11.1, 8000 14.8 (33 MB, 2.2 TB/s); the kernel with two launches took 11.6, 13.7 and 14.8 for the
// last three when this one took 7.0, 10.5 and 13.9.
//
// ANY: heads of every other size up to 256 and every alignment, filled up to 64, 128 or 256 columns with zeros (three widths are
// enough: the matrix units have time, and no more bytes are read). K and V come with 16-byte copies where the head allows it,
// element by element elsewhere. Long sequences and prompts are its work too, without a kernel of their own. Heads of 96, 8 KV
// heads, groups of 4: one token on 4000 22 us, 1000 new tokens 185 us, 32 on 1000 19 us (with 32-bit arithmetic on the CUDA
// cores and one CTA per unit 1613, 1064 and 424). Far from the floor where there is much to do, since every tile of 16 rows reads its
// keys again and a unit has 8 CTAs at most: 8192 new tokens 8.3 ms (floor 0.25), one token on 100 K 386 us (47).
template <class T, u32 D, u32 CLUSTER, bool ANY>
__global__ void __launch_bounds__(SPLIT_THREADS, D > 128 ? 1 : 2)
k_attend_cluster(const __grid_constant__ AttendArgs a, const __grid_constant__ KvMaps maps) {
  typedef SplitShape<D> S;
  extern __shared__ u8 smem_raw[];
  __shared__ __align__(8) u64 bars[SPLIT_WARPS * S::STAGES];
  __shared__ float s_ml[SPLIT_WARPS][SPLIT_ROWS][2];
  __shared__ float s_part_ml[SPLIT_ROWS][2];
  __shared__ u32 s_lost;
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = a.p.n_kv_heads;
  const u32 bar0 = smem_addr(bars) + warp * S::STAGES * 8, rank = blockIdx.x % CLUSTER, unit = blockIdx.x / CLUSTER, h = unit % H;
  if (lane == 0) {
    for (u32 i = 0; i < S::STAGES; ++i) bar_init(bar0 + i * 8, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (!ANY && tid < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(tid ? &maps.tail : &maps.pool) : "memory");
  Seq q; u32 seq, tile;
  if (!find_tile<SPLIT_THREADS>(a, SPLIT_ROWS, unit / H, q, seq, tile)) return;      // the whole cluster
  const u32 ring0 = (smem_addr(smem_raw) + 1023) & ~1023u, ring = ring0 + warp * S::RING;
  const u32 r0 = tile * SPLIT_ROWS, r1 = min(r0 + SPLIT_ROWS, q.n * a.group) - 1;
  u32 b_first, it = 0;
  const u32 nb = tile_blocks(a, q, r0, r1, b_first), per = (nb + CLUSTER - 1) / CLUSTER;
  float o[D / 8][4], m[2], l[2];
  const bool ok = split_keys<T, D, ANY>(a, maps, q, seq, h, r0, r1, b_first + min(rank * per, nb), b_first + min((rank + 1) * per, nb), ring, bar0, it, o, m, l);
  split_leave<D>(smem_raw, ring, o, m, l, s_ml);
  const bool lost = __syncthreads_or(!ok);
  // this CTA's part: sums behind warp 0's in its ring
  constexpr u32 PART = (SPLIT_ROWS * split_pitch<D>() * 4 + 127) / 128 * 128;
  static_assert(PART + SPLIT_ROWS * D * 4 <= S::RING, "the part fits warp 0's ring");
  float *const part = (float *)(smem_raw + (ring0 - smem_addr(smem_raw)) + PART);
  {
    const u32 r = tid / 8;
    float mm, ll, f[SPLIT_WARPS];
    split_row(s_ml, r, mm, ll, f);
#pragma unroll
    for (u32 c = (tid % 8) * 4; c < D; c += 32) *(float4 *)(part + r * D + c) = split_sum<D>(smem_raw, ring0, r, c, f);
    if (tid % 8 == 0) { s_part_ml[r][0] = mm; s_part_ml[r][1] = ll; }
    if (tid == 0) s_lost = lost;
  }
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  // a CTA joins 16 / CLUSTER of the rows, a thread COLS columns of one
  constexpr u32 ROWS_HERE = SPLIT_ROWS / CLUSTER, COLS = D * ROWS_HERE < SPLIT_THREADS ? 1 : D * ROWS_HERE / SPLIT_THREADS, PER_ROW = D / COLS;
  auto there = [&](const void *p, u32 cta) {             // the same place in another CTA's shared memory
    u32 r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr(p)), "r"(cta));
    return r;
  };
  const bool busy = tid < ROWS_HERE * PER_ROW;
  const u32 r = rank * ROWS_HERE + (busy ? tid / PER_ROW : 0), c = tid % PER_ROW * COLS;
  float top = -INFINITY, sum = 0.0f, e[COLS];
  u32 any_lost = 0;
#pragma unroll
  for (u32 z = 0; z < COLS; ++z) e[z] = 0.0f;
  constexpr u32 STEP = CLUSTER < 8 ? CLUSTER : 8;        // parts read together
#pragma unroll 1
  for (u32 y0 = 0; y0 < CLUSTER; y0 += STEP) {
    float mm[STEP], ll[STEP], v[STEP][COLS], now = top;
#pragma unroll
    for (u32 y = 0; y < STEP; ++y) {
      u32 x;
      asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(mm[y]), "=f"(ll[y]) : "r"(there(&s_part_ml[r][0], y0 + y)) : "memory");
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(there(&s_lost, y0 + y)) : "memory");
      any_lost |= x;
      const u32 at = there(part + r * D + c, y0 + y);
#pragma unroll
      for (u32 z = 0; z < COLS; z += 4) {
        if (COLS >= 4) asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                    : "=f"(v[y][z]), "=f"(v[y][(z + 1) % COLS]), "=f"(v[y][(z + 2) % COLS]), "=f"(v[y][(z + 3) % COLS]) : "r"(at + 4 * z) : "memory");
        else if (COLS == 2) asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v[y][0]), "=f"(v[y][1 % COLS]) : "r"(at) : "memory");
        else asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[y][0]) : "r"(at) : "memory");
      }
      now = fmaxf(now, mm[y]);
    }
    const float ref = now == -INFINITY ? 0.0f : now, f = ex2(top - ref);
    top = now; sum *= f;
#pragma unroll
    for (u32 z = 0; z < COLS; ++z) e[z] *= f;
#pragma unroll
    for (u32 y = 0; y < STEP; ++y) {
      const float w = ex2(mm[y] - ref);
      sum += w * ll[y];
#pragma unroll
      for (u32 z = 0; z < COLS; ++z) e[z] += w * v[y][z];
    }
  }
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");    // nobody reads here any more
  if (any_lost) {
    if (tid == 0) kv_err(a.err, KVERR_WAIT);
    if (!ok) for (u32 i = 0; i < S::STAGES; ++i) for (u32 y = 0; y < 2; ++y) bar_wait(bar0 + i * 8, y);   // copies in flight
    return;
  }
  if (!busy || r0 + r > r1) return;
  const float inv = sum > 0.0f ? 1.0f / sum : sum;
  const u32 t = q.t0 + (r0 + r) / a.group, hq = h * a.group + (r0 + r) % a.group;
  u16 *const out = (u16 *)a.out + (u64)t * a.o_ts + (u64)hq * a.o_hs + c;
  const u32 d = ANY ? a.p.head_dim : D;
  if (COLS >= 4 && ((uintptr_t)out & 7) == 0 && c + COLS <= d) {
#pragma unroll
    for (u32 z = 0; z < COLS; z += 4)
      *(uint2 *)(out + z) = make_uint2(Elem<T>::down(e[z] * inv, e[(z + 1) % COLS] * inv), Elem<T>::down(e[(z + 2) % COLS] * inv, e[(z + 3) % COLS] * inv));
  } else {
#pragma unroll
    for (u32 z = 0; z < COLS; ++z) if (c + z < d) ((T *)out)[z] = Elem<T>::down1(e[z] * inv);
  }
  if (a.lse && c == 0) a.lse[(u64)t * a.n_q_heads + hq] = (top + log2f(sum)) * 0.69314718055994531f;
}

// ------------------------------------------------------------------------------------------------------
// Many rows (prompts, chunks of new tokens): bound by the tensor cores and the exponentials. A CTA takes up to 256 rows
// of one KV head as two tiles of 128, the height of a tcgen05 matrix instruction, and walks over the keys 128 at a time.
//   warp 11     brings the coming jobs' queries into the L2 cache
//   warp 10     works out the CTA's jobs
//   warp 9      loads K and V (TMA, one box per block) into a ring of 128-key stages
//   warp 8      issues the matrix products: S = Q K^T and O += P V, both accumulated in tensor memory
//   warps 0-7   one thread per row: maximum, powers, sum; P goes back to tensor memory in the place of S, as the first
//               operand of the second product
// The two tiles take turns: while one tile's powers are computed the tensor cores work on the other. Tensor memory: S0,
// S1 (128 columns each), O0, O1 (head_dim columns each): full with heads of 128, so S is not held twice, and a tile's next S
// waits for the second product of its P.
// Measured (heads of 128, bf16): 128 keys for both tiles take 2950 cycles, of which the tensor cores need 2040 and the exponential
// units 2048: a row waits 830 cycles for its S, then 50 to load it, 350 for the maximum, 1460 for the powers, 160 for the store.
// 8192 new tokens, 8 KV heads, groups of 4: 432-441 us in a captured graph (1260 TFLOP/s; 76 % of the measured matrix rate), 500-514 us at
// the 1.58 GHz that the power limit leaves when it runs on and on (1085 TFLOP/s, 78 % of the sustained rate). 500 tokens on 130,500:
// 960-1000 us, 1011-1032 on and on. Tried and slower or the same: two threads per row (480 us where this took 465), a thread issuing the products
// for each tile (525: the tiles fall into step), P handed over in four parts, a polynomial for every fourth power (0-4 %).
// Between two jobs of a CTA 4 us pass, and a launch has its first S after 6 us, most of it for working out the jobs.
// ------------------------------------------------------------------------------------------------------
constexpr u32 TC_ROWS = 256, TC_TILE = 128, TC_KEYS = 128, TC_KB = TC_KEYS / BT, TC_THREADS = 384;
template <u32 D> struct TcShape {
  static constexpr u32 BLOCK = BT * D * 2, STAGE = TC_KEYS * D * 2, Q = TC_ROWS * D * 2, STAGES = (224 * 1024 - Q) / STAGE;
  static constexpr u32 SMEM = Q + STAGES * STAGE + 1024;
};

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

// A piece of a tile, as the scheduling warp hands it to the others.
struct Job {
  u32 t0, kv, seq, h;        // first token row, length and number of the sequence; KV head
  u32 r0, r1;                // rows of the tile, counted in the sequence: first and last
  u32 shift;                 // index in the sequence of its first new token, as a signed number
  u32 b0, b1, all_lo, all_hi;// blocks of keys [b0, b1); keys every row sees
  u32 first;                 // first key any row sees
  u32 part, direct, last;    // place of the partial result, or the whole result at once; last: no job, the end
};
constexpr u32 TC_JOBS = 4, TC_PARTS = 2;      // P is handed to the second product in so many parts

template <class T, u32 D>
__global__ void __launch_bounds__(TC_THREADS, 1)
k_attend_tc(const __grid_constant__ AttendArgs a, const __grid_constant__ KvMaps maps, u32 n_parts, u64 most_tiles) {
  typedef TcShape<D> S;
  constexpr bool FP16 = !__is_same(T, __nv_bfloat16);
  extern __shared__ u8 smem_raw[];
  __shared__ __align__(8) u64 s_full[S::STAGES], s_empty[S::STAGES], s_sready[2], s_pready[2][TC_PARTS], s_qready[2], s_oready[2], s_drain, s_jfull[TC_JOBS], s_jempty[TC_JOBS];
  __shared__ u32 s_tmem;
  __shared__ volatile u32 s_lost;
  __shared__ Job s_job[TC_JOBS];
  __shared__ float s_cost[N_CUTS];
  __shared__ u8 s_order[32];
  asm volatile("griddepcontrol.launch_dependents;");
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = a.p.n_kv_heads;
  const u32 full = smem_addr(s_full), empty = smem_addr(s_empty), sready = smem_addr(s_sready), pready = smem_addr(s_pready),
            qready = smem_addr(s_qready), oready = smem_addr(s_oready), drain = smem_addr(&s_drain), jfull = smem_addr(s_jfull), jempty = smem_addr(s_jempty);
  if (tid == 0) {
    for (u32 i = 0; i < S::STAGES; ++i) { bar_init(full + i * 8, 1); bar_init(empty + i * 8, 1); }
    for (u32 i = 0; i < 2; ++i) { bar_init(sready + i * 8, 1); bar_init(oready + i * 8, 1); bar_init(qready + i * 8, 4); }
    for (u32 i = 0; i < 2 * TC_PARTS; ++i) bar_init(pready + i * 8, 4);
    for (u32 i = 0; i < TC_JOBS; ++i) { bar_init(jfull + i * 8, 1); bar_init(jempty + i * 8, 11); }
    bar_init(drain, 1);
    s_lost = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (warp == 9 && lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(lane ? &maps.tail : &maps.pool) : "memory");
  Seq mine;                              // the sequence of this lane among the first 32
  const Cut cut = weigh_cuts(a, TC_ROWS, n_parts, gridDim.x, (float)most_tiles, warp, TC_THREADS / 32, s_cost, mine);
  tc_before();
  __syncthreads();
  tc_after();
  const u32 tmem = s_tmem;
  const u32 sq = (smem_addr(smem_raw) + 1023) & ~1023u, ring = sq + S::Q;
  volatile u32 *const lost = &s_lost;
  // the next job, for a whole warp; false: no more, or a wait ran out
  u32 jobs = 0;
  auto next_job = [&](Job &j) {
    const u32 at = jobs % TC_JOBS;
    if (!tc_wait(jfull + at * 8, (jobs / TC_JOBS) & 1, lost, a.b.max_blocks)) return false;
    j = s_job[at];
    __syncwarp();
    if (lane == 0) bar_arrive(jempty + at * 8);
    ++jobs;
    return j.last == 0;
  };

  // registers: 168 for each of 384 threads at the launch; 208 for a thread that holds a row of S, 88 for the others (with 224 and
  // 56 the others spill)
  if (warp == 11) {
    // ---- queries of the jobs to come into the L2 cache
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    for (Job j; next_job(j);)
      for (u32 r = j.r0 + lane; r <= j.r1; r += 32) {
        const u32 tok = r / a.group;
        const u16 *src = (const u16 *)a.q + (u64)(j.t0 + tok) * a.q_ts + (u64)(j.h * a.group + r - tok * a.group) * a.q_hs;
        if (((uintptr_t)src & 15) == 0) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(D * 2) : "memory");
      }
  } else if (warp == 10) {
    // ---- scheduling: this CTA's jobs, one per round of the grid, every other round in reverse so that the long first jobs of
    // a causal prompt even out. Jobs of a sequence: piece, tile (last tokens first), KV head; those that run at the same
    // time then mostly read the same keys.
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    const u32 piece = choose_cut(a, n_parts, cut, s_cost);
    // (a launch has fewer than 2^32 jobs: tokens times query heads and a few thousand pieces)
    u32 base = 0, part0 = 0, s0 = 0;     // first job and first partial of the 32 sequences in hand
    Seq q = mine;
    u32 tiles = 0, pieces = 0;
    u32 my_jobs = 0, at = 0, all = 0, my_part = 0, all_parts = 0;
    u32 my_seq = 0;
    bool ok = true, first = true;
    if (blockIdx.x == 0 && n_parts) { if (lane == 0) scratch_plan(a)[0] = make_uint4(0, 0, 0, 0); __syncwarp(); }
    for (u32 k = 0;; ++k) {
      const u32 want = k * gridDim.x + (k % 2 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
#pragma unroll 1
      while (first || (want >= base + all && s0 + 32 < a.b.n_seqs)) {
        // the next 32 sequences, one per lane, those with the longest pieces first: jobs that get shorter, dealt out back and
        // forth, come out even
        if (!first) { base += all; part0 += all_parts; s0 += 32; }
        my_seq = s0 + lane;
        tiles = pieces = 0;
        u32 length = 0;
        // starts that go up and down make the same tokens count again and again: then nothing is done (load_seq has set the
        // error word)
        if (my_seq < a.b.n_seqs && cut.sound) {
          if (!first) q = load_seq(a.b, my_seq, a.err);
          tiles = seq_tiles(a, q, TC_ROWS);
          const u32 nb = seq_blocks(a, q, TC_ROWS);
          pieces = (nb + piece - 1) / piece;
          length = tiles ? (nb + pieces - 1) / pieces : 0;
        }
        first = false;
        const u32 n = min(32u, a.b.n_seqs - s0);
        if (n > 1) {
          u32 rank = lane;               // lanes behind the last sequence stay where they are
          if (lane < n) rank = 0;
#pragma unroll 4
          for (u32 y = 0; y < n; ++y) {
            const u32 z = __shfl_sync(~0u, length, y);
            if (lane < n) rank += z > length || (z == length && y < lane);
          }
          s_order[rank] = (u8)lane;
          __syncwarp();
          const u32 from = s_order[lane];
          q.t0 = __shfl_sync(~0u, q.t0, from); q.n = __shfl_sync(~0u, q.n, from); q.kv = __shfl_sync(~0u, q.kv, from);
          tiles = __shfl_sync(~0u, tiles, from); pieces = __shfl_sync(~0u, pieces, from);
          my_seq = s0 + from;
          __syncwarp();
        }
        my_jobs = tiles * pieces * H;
        const u32 parts = pieces > 1 ? tiles * pieces : 0;
        u32 incl = my_jobs, pincl = parts;
#pragma unroll
        for (u32 o = 1; o < 32; o *= 2) {
          const u32 y = __shfl_up_sync(~0u, incl, o), z = __shfl_up_sync(~0u, pincl, o);
          if (lane >= o) { incl += y; pincl += z; }
        }
        at = base + incl - my_jobs; my_part = part0 + pincl - parts;
        all = __shfl_sync(~0u, incl, 31); all_parts = __shfl_sync(~0u, pincl, 31);
        if (blockIdx.x == 0 && n_parts && my_seq < a.b.n_seqs) {
          scratch_plan(a)[1 + my_seq] = make_uint4(my_part, pieces, tiles, 0);
          if (pieces > 1) scratch_plan(a)[0].x = 1;
        }
      }
      const u32 hit = __ballot_sync(~0u, want >= at && want < at + my_jobs);
      const u32 slot = k % TC_JOBS;
      if (k >= TC_JOBS && !(ok = tc_wait(jempty + slot * 8, (k / TC_JOBS - 1) & 1, lost, a.b.max_blocks))) break;
      if (hit && lane == __ffs(hit) - 1) {
        Job j;
        const u32 x = want - at, y = x / H, h = x - y * H, pc = y / tiles, tile = tiles - 1 - (y - pc * tiles);
        j.t0 = q.t0; j.kv = q.kv; j.seq = my_seq; j.h = h; j.shift = q.kv - q.n;
        j.r0 = tile * TC_ROWS; j.r1 = min(j.r0 + TC_ROWS, q.n * a.group) - 1;
        u32 last;
        row_range(a, q, j.r0 / a.group, j.first, j.all_hi);
        row_range(a, q, j.r1 / a.group, j.all_lo, last);
        const u32 b_first = j.first / BT, b_last = (last + BT - 1) / BT, nb = b_last > b_first ? b_last - b_first : 0;
        const u32 per = ((nb + pieces - 1) / pieces + TC_KB - 1) / TC_KB * TC_KB;       // whole stages
        j.b0 = b_first + min(pc * per, nb); j.b1 = b_first + min((pc + 1) * per, nb);
        j.direct = pieces == 1;
        j.part = (my_part + pc * tiles + tile) * H + h;
        j.last = 0;
        if (!j.direct && j.part >= n_parts) { kv_err(a.err, KVERR_RANGE); j.part = 0; j.b1 = j.b0; }     // cannot happen
        s_job[slot] = j;
      } else if (!hit && lane == 0) {
        s_job[slot].last = 1;
      }
      __syncwarp();
      if (lane == 0) bar_arrive(jfull + slot * 8);
      if (!hit) break;                   // behind the last job, and so behind the last sequence
    }
  } else if (warp == 9) {
    // ---- loads: K0, V0, K1, V1, ...; blocks behind the piece's last one read as zeros (a slot behind both pools)
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    u32 it = 0;
    bool ok = true;
    for (Job j; ok && next_job(j);) {
      const u32 *row = a.b.table + j.seq * a.b.table_stride;
      const u32 n = (j.b1 - j.b0 + TC_KB - 1) / TC_KB;
      u32 slots = 0;
      for (u32 s = 0; s < n && ok; ++s) {
        if (s % 4 == 0) {
          const u32 b = j.b0 + s * TC_KB + lane;
          slots = b < j.b1 ? row[b] : 0xFFFFFFFFu;
          if (b < j.b1 && slots >= a.p.n_slots && slots - a.p.n_slots >= a.p.n_tail) kv_err(a.err, KVERR_RANGE);
        }
        const u32 slot = __shfl_sync(~0u, slots, (s % 4) * TC_KB + lane % TC_KB);
        for (u32 kv = 0; kv < 2; ++kv, ++it) {
          const u32 st = it % S::STAGES;
          if (it >= S::STAGES && !tc_wait(empty + st * 8, (it / S::STAGES - 1) & 1, lost, a.b.max_blocks)) { ok = false; break; }
          if (lane == 0) bar_expect(full + st * 8, S::STAGE);
          __syncwarp();
          if (lane < TC_KB) load_block(a, maps, ring + st * S::STAGE + lane * S::BLOCK, full + st * 8, slot, 2 * a.layer + kv, j.h, D / 64);
          __syncwarp();
        }
      }
    }
    // whatever was loaded has landed before the CTA ends, if the products have waited for it or not
    for (u32 i = it > S::STAGES ? it - S::STAGES : 0; i < it; ++i) bar_wait(full + (i % S::STAGES) * 8, (i / S::STAGES) & 1);
  } else if (warp == 8) {
    // ---- matrix products: one thread does all of it, the tiles strictly in turn, which keeps their powers half a period apart
    // (a thread per tile was tried: the tiles fall into step and compete, first for the tensor cores, then for the powers).
    // What it does between two products is in the way of the tensor cores, so that is kept short: stages are counted up,
    // not divided out, descriptors differ by constants, arrivals of K and V are looked at before those of P.
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (elect_one()) {
      const u32 id_s = tc_idesc(FP16, TC_KEYS, false), id_o = tc_idesc(FP16, D, true);
      const u64 dq0 = tc_desc(sq, 16, 1024), dk0 = tc_desc(ring, 16, D * 16), dv0 = tc_desc(ring, 1024, D * 16);
      struct Place { u32 st, ph; };      // a stage and its phase
      auto after = [](Place x) { return x.st + 1 == S::STAGES ? Place{0, x.ph ^ 1} : Place{x.st + 1, x.ph}; };
      auto has = [&](Place x) { return bar_try(full + x.st * 8, x.ph); };
      auto landed = [&](Place x) { return tc_wait1(full + x.st * 8, x.ph, lost, a.b.max_blocks); };
      auto product_s = [&](u32 i, u32 st) {
        const u64 dk = dk0 + st * (S::STAGE / 16);
#pragma unroll
        for (u32 k = 0; k < D / 16; ++k)
          tc_mma_ss(tmem + i * 128, dq0 + (i * (TC_TILE * D * 2) + (k / 4) * (TC_TILE * 128) + (k % 4) * 32) / 16,
                    dk + ((k / 4) * 1024 + (k % 4) * 32) / 16, id_s, k > 0);
        tc_commit(sready + i * 8);
      };
      Place at_k{0, 0};                  // the first K of the job in turn
      u32 seen_q[2] = {0, 0}, seen_p[2] = {0, 0};
      bool ok = true;
      for (;;) {
        const u32 at = jobs % TC_JOBS;
        if (!(ok = tc_wait1(jfull + at * 8, (jobs / TC_JOBS) & 1, lost, a.b.max_blocks))) break;
        ++jobs;
        const u32 r0 = s_job[at].r0, r1 = s_job[at].r1, b0 = s_job[at].b0, b1 = s_job[at].b1, kv = s_job[at].kv, first = s_job[at].first,
                  end = s_job[at].last;
        bar_arrive(jempty + at * 8);
        if (end) break;
        const u32 n = (b1 - b0 + TC_KB - 1) / TC_KB;
        const bool two = r1 - r0 >= TC_TILE;
        if (!n) continue;
        if (!(ok = landed(at_k))) break;
#pragma unroll
        for (u32 i = 0; i < 2; ++i)
          if (ok && (i == 0 || two)) {
            ok = tc_wait1(qready + i * 8, seen_q[i]++ & 1, lost, a.b.max_blocks);
            tc_after();
            if (ok) product_s(i, at_k.st);
          }
        if (!ok) break;
        // stages to hand back, V of the keys before and the K in use: not at once, which would hold up the next product, but
        // in the pause before the second tile's powers are there. The arrivals of the next keys are looked at there too.
        Place v = after(at_k), k = after(v);
        u32 free_k = at_k.st, free_v = ~0u;
        bool has_v = false, has_k = false;
        for (u32 s = 0; s < n; ++s) {
          const bool more = s + 1 < n;
          const Place v1 = after(k), k1 = after(v1);
          if (!has_v && !(ok = landed(v))) break;
          // Tokens that no row sees, in front of the window in the first block and behind the length in the last: whatever
          // their values hold, weight 0 must not meet an Inf or a NaN.
          auto clear = [&](u32 block, u32 r0, u32 r1) {
            for (u32 r = r0; r < r1; ++r)
              for (u32 c = 0; c < D / 8; ++c)
                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(ring + v.st * S::STAGE + block * S::BLOCK + block_off<D>(r, c)), "r"(0) : "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          };
          if (s == 0 && b0 * BT < first) clear(0, 0, first - b0 * BT);      // fewer than a block's
          if (!more && b1 * BT > kv) clear((b1 - 1 - b0) % TC_KB, kv % BT, BT);
          const u64 dv = dv0 + v.st * (S::STAGE / 16);
#pragma unroll
          for (u32 i = 0; i < 2; ++i)
            if (i == 0 || two) {
              const u32 phase = seen_p[i]++ & 1;
#pragma unroll
              for (u32 part = 0; part < TC_PARTS; ++part) {
                ok = ok && tc_wait1(pready + (i * TC_PARTS + part) * 8, phase, lost, a.b.max_blocks);
                if (!ok) break;
                tc_after();
#pragma unroll
                for (u32 y = part * (TC_KB / TC_PARTS); y < (part + 1) * (TC_KB / TC_PARTS); ++y)
                  tc_mma_ts(tmem + 256 + i * D, tmem + i * 128 + y * 8, dv + y * (D * 32 / 16), id_o, s > 0 || y > 0);
              }
              if (!ok) break;
              if (!more) tc_commit(oready + i * 8);      // the finished sums
              else if (i == 0 && !has_k && !(ok = landed(k))) break;
              else product_s(i, k.st);
              if (i == 0) {
                if (free_v != ~0u) tc_commit(empty + free_v * 8);
                tc_commit(empty + free_k * 8);
                has_v = more && has(v1);
                has_k = s + 2 < n && has(k1);
              }
            }
          if (!ok || !more) break;
          free_v = v.st; free_k = k.st;
          v = v1; k = k1;
        }
        if (!ok) break;
        tc_commit(empty + v.st * 8);     // the last V; behind it lies the next job's first K
        at_k = k;
      }
      // all products and their arrivals are done before the CTA ends
      tc_commit(drain);
      bar_wait(drain, 0);
    }
    __syncwarp();
  } else {
    // ---- one thread per row. Between two jobs the tensor cores would stand still while queries come and results go, so the
    // next job's queries are brought in as soon as the last S is made, and its first S is made while the results are written.
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const u32 i = warp / 4, rt = tid % TC_TILE;
    const u32 lanes = (warp % 4) << 21, ts = tmem + lanes + i * 128, to = tmem + lanes + 256 + i * D;
    u32 seen_s = 0, seen_o = 0;          // completions of sready[i], oready[i]
    bool ok = true;
    // The next job with rows in this tile; its queries into shared memory.
    auto begin = [&](Job &j) {
      do { if (!next_job(j)) return false; } while (i && j.r1 - j.r0 < TC_TILE);
      if (j.b0 >= j.b1) return true;
      const u32 rr = min(j.r0 + i * TC_TILE + rt, j.r1), tok = rr / a.group;      // rows behind the last one repeat it
      const u16 *const src = (const u16 *)a.q + (u64)(j.t0 + tok) * a.q_ts + (u64)(j.h * a.group + rr - tok * a.group) * a.q_hs;
      const bool wide = __all_sync(~0u, ((uintptr_t)src & 15) == 0);
      uint4 v[D / 8];                    // lanes take 16 bytes each of as many rows as make 512 bytes
      auto from = [&](u32 k) { return (const u16 *)__shfl_sync(~0u, (u64)src, (k * 32 + lane) / (D / 8)) + lane % (D / 8) * 8; };
      if (wide) {                        // (a branch for each would make each load wait for the one before)
#pragma unroll
        for (u32 k = 0; k < D / 8; ++k) v[k] = *(const uint4 *)from(k);
      } else {
#pragma unroll
        for (u32 k = 0; k < D / 8; ++k) {
          const u16 *const f = from(k);
          u32 x[4];
#pragma unroll
          for (u32 y = 0; y < 4; ++y) x[y] = (u32)f[2 * y] | (u32)f[2 * y + 1] << 16;
          v[k] = make_uint4(x[0], x[1], x[2], x[3]);
        }
      }
#pragma unroll
      for (u32 k = 0; k < D / 8; ++k) {
        const u32 at = k * 32 + lane, row = warp % 4 * 32 + at / (D / 8), c = at % (D / 8);
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};"
                     ::"r"(sq + i * (TC_TILE * D * 2) + (c / 8) * (TC_TILE * 128) + row * 128 + (((c % 8) ^ (row % 8)) * 16)),
                       "r"(v[k].x), "r"(v[k].y), "r"(v[k].z), "r"(v[k].w) : "memory");
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      tc_before();
      __syncwarp();
      if (lane == 0) bar_arrive(qready + i * 8);
      return true;
    };
    Job j;
    for (bool have = begin(j); have;) {
      const u32 n = (j.b1 - j.b0 + TC_KB - 1) / TC_KB;
      const u32 r = j.r0 + i * TC_TILE + rt, rr = min(r, j.r1);
      const bool mine = r <= j.r1;
      const u32 tok = rr / a.group, t = j.t0 + tok, hq = j.h * a.group + rr - tok * a.group;
      u32 lo, hi;
      {
        const long long own = (long long)(int)j.shift + tok;
        hi = a.full ? j.kv : own < 0 ? 0u : (u32)own + 1;
        lo = a.window && hi > a.window ? hi - a.window : 0u;
      }
      float m = -INFINITY, l = 0.0f;
      for (u32 s = 0; s < n; ++s) {
        if (!(ok = tc_wait(sready + i * 8, seen_s++ & 1, lost, a.b.max_blocks))) break;
        tc_after();
        u32 x[128];
        float *const v = reinterpret_cast<float *>(x);
#pragma unroll
        for (u32 c = 0; c < 4; ++c) tc_ld32(x + 32 * c, ts + 32 * c);
        tc_wait_ld();
        const u32 key0 = (j.b0 + s * TC_KB) * BT;
        if (key0 < j.all_lo || key0 + TC_KEYS > j.all_hi) {
          const int from = (int)lo - (int)key0, to_ = (int)hi - (int)key0;
#pragma unroll
          for (int b = 0; b < 128; b += 32) {     // a bit for each key the row sees
            const u32 see = (from >= b + 32 ? 0u : from > b ? ~0u << (from - b) : ~0u) & (to_ >= b + 32 ? ~0u : to_ > b ? ~(~0u << (to_ - b)) : 0u);
#pragma unroll
            for (int c = 0; c < 32; ++c) v[b + c] = see >> c & 1 ? v[b + c] : -INFINITY;
          }
        }
        float top[4] = {max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), max3(v[6], v[7], v[8]), max3(v[9], v[10], v[11])};
#pragma unroll
        for (u32 c = 12; c < 124; c += 8)
#pragma unroll
          for (u32 y = 0; y < 4; ++y) top[y] = max3(top[y], v[c + 2 * y], v[c + 2 * y + 1]);
        const float now = fmaxf(max3(max3(top[0], v[124], v[125]), max3(top[1], v[126], v[127]), top[2]), top[3]) * a.scale_log2;
        if (__any_sync(~0u, must_move<T>(m, now))) {
          const float f = raise_or_lower<T>(m, now, l);
          l *= f;
          if (s > 0) {                   // the product before S of these keys has been waited for: O is at rest
#pragma unroll
            for (u32 c = 0; c < D / 16; ++c) {
              u32 y[16];
              tc_ld16(y, to + 16 * c);
              tc_wait_ld();
#pragma unroll
              for (u32 z = 0; z < 16; ++z) y[z] = __float_as_uint(__uint_as_float(y[z]) * f);
              tc_st16(to + 16 * c, y);
            }
          }
        }
        const float ref = m == -INFINITY ? 0.0f : m;
        const u64 scale2 = pack2(a.scale_log2, a.scale_log2), ref2 = pack2(-ref, -ref);
        u64 sum[2] = {0, 0};
#pragma unroll
        for (u32 b = 0; b < 4; ++b) {
          u32 p[16];
#pragma unroll
          for (u32 c = 0; c < 16; ++c) {
            const u64 y = fma2(pack2(v[32 * b + 2 * c], v[32 * b + 2 * c + 1]), scale2, ref2);
            const float2 z = unpack2(y);
            const float p0 = ex2(z.x), p1 = ex2(z.y);
            sum[c % 2] = add2(sum[c % 2], pack2(p0, p1));
            p[c] = Elem<T>::down(p0, p1);
          }
          if (b && b % (4 / TC_PARTS) == 0) {    // the store of the part before has had these powers to finish
            tc_wait_st();
            tc_before();
            __syncwarp();
            if (lane == 0) bar_arrive(pready + (i * TC_PARTS + b / (4 / TC_PARTS) - 1) * 8);
          }
          tc_st16(ts + 16 * b, p);
        }
        const float2 add = unpack2(add2(sum[0], sum[1]));
        l += add.x + add.y;
        tc_wait_st();
        tc_before();
        __syncwarp();
        if (lane == 0) bar_arrive(pready + (i * TC_PARTS + TC_PARTS - 1) * 8);
      }
      if (!ok) break;
      // ---- results: every thread writes its row, 32 bytes at a time
      const bool direct = j.direct != 0;
      const float inv = !direct ? 1.0f : l > 0.0f ? 1.0f / l : l;
      const u64 prow = (u64)j.part * TC_ROWS + i * TC_TILE + rt;
      u8 *const out = direct ? (u8 *)((u16 *)a.out + (u64)t * a.o_ts + (u64)hq * a.o_hs) : (u8 *)(scratch_sums(a) + prow * D);
      have = begin(j);
      if (n && !(ok = tc_wait(oready + i * 8, seen_o++ & 1, lost, a.b.max_blocks))) break;
      tc_after();
      if (mine) {
        if (!direct) ((float2 *)(scratch_sums(a) + (u64)n_parts * TC_ROWS * D))[prow] = make_float2(m, l);
        else if (a.lse) a.lse[(u64)t * a.n_q_heads + hq] = (m + log2f(l)) * 0.69314718055994531f;
      }
      const bool wide = ((uintptr_t)out & 31) == 0;
#pragma unroll
      for (u32 c = 0; c < D; c += 64) {
        u32 y[64];
        tc_ld32(y, to + c);
        tc_ld32(y + 32, to + c + 32);
        tc_wait_ld();
        if (!n) {                        // no keys: nothing was ever summed up
#pragma unroll
          for (u32 z = 0; z < 64; ++z) y[z] = 0;
        }
        if (!mine) {
        } else if (direct) {
          u32 e[32];
#pragma unroll
          for (u32 z = 0; z < 32; ++z) e[z] = Elem<T>::down(__uint_as_float(y[2 * z]) * inv, __uint_as_float(y[2 * z + 1]) * inv);
          u8 *const dst = out + c * 2;
          if (wide) {
#pragma unroll
            for (u32 z = 0; z < 4; ++z) st_global32(dst + 32 * z, e + 8 * z);
          } else {
#pragma unroll
            for (u32 z = 0; z < 32; ++z) { ((u16 *)dst)[2 * z] = (u16)e[z]; ((u16 *)dst)[2 * z + 1] = (u16)(e[z] >> 16); }
          }
        } else {
          u8 *const dst = out + c * 4;
          if (wide) {
#pragma unroll
            for (u32 z = 0; z < 8; ++z) st_global32(dst + 32 * z, y + 8 * z);
          } else {                       // scratch is aligned to 16 bytes
#pragma unroll
            for (u32 z = 0; z < 16; ++z) *(uint4 *)(dst + 16 * z) = make_uint4(y[4 * z], y[4 * z + 1], y[4 * z + 2], y[4 * z + 3]);
          }
        }
        __syncwarp();
      }
    }
  }
  tc_before();
  __syncthreads();
  tc_after();
  if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  if (tid == 0 && s_lost) kv_err(a.err, KVERR_WAIT);
}

// ------------------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------------------
bool make_kv_map(CUtensorMap *m, void *base, bool layer_major, u64 n_slots, u64 n_chunks, u64 n_kv_heads, u64 head_dim) {
  typedef CUresult (*Encode)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                             const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  void *fn = nullptr;
  cudaDriverEntryPointQueryResult got;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &got) != cudaSuccess ||
      got != cudaDriverEntryPointSuccess || !fn) {
    cudaGetLastError();
    return false;
  }
  const u64 tok = n_kv_heads * head_dim * 2, chunk = BT * tok;
  // 64 elements | 8 tokens | 64-element parts of a token's heads | halves of blocks | the other index
  const cuuint64_t dims[5] = {64, 8, n_kv_heads * head_dim / 64, 2 * (layer_major ? n_slots : n_chunks), layer_major ? n_chunks : n_slots};
  const cuuint64_t strides[4] = {tok, 128, 8 * tok, chunk * (layer_major ? n_slots : n_chunks)};
  const cuuint32_t box[5] = {64, 8, (cuuint32_t)(head_dim / 64), 2, 1}, es[5] = {1, 1, 1, 1, 1};
  return ((Encode)fn)(m, CU_TENSOR_MAP_DATA_TYPE_UINT16, 5, base, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                      CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class... Exp, class... Act>
static cudaError_t launch_join(void (*kern)(Exp...), u32 threads, u64 ctas, u32 sms, cudaStream_t s, u32 *launches, Act... args) {
  cudaLaunchConfig_t c{};
  c.gridDim = dim3((u32)std::min<u64>(ctas, 8ull * sms)); c.blockDim = dim3(threads); c.stream = s;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  c.attrs = &at; c.numAttrs = 1;
  ++*launches;
  return cudaLaunchKernelEx(&c, kern, args...);
}

AttendPlan plan_attend(const AttendArgs &a, u32 max_q_len, int sm_count) {
  AttendPlan p{};
  const u64 H = a.p.n_kv_heads;
  p.sms = sm_count;
  // no more tiles than this: every sequence adds less than one to the quotient
  auto tiles = [&](u64 rows) { return ((u64)a.b.n_tokens * a.group + a.b.n_seqs * (rows - 1)) / rows; };
  if (a.p.head_dim != 64 && a.p.head_dim != 128) {
    // a unit's keys over up to 8 CTAs, as long as all run at once and each of their warps has a block or more
    const u64 units = tiles(SPLIT_ROWS) * H, slots = (a.p.head_dim > 128 ? 1ull : 2ull) * sm_count;
    p.rows = SPLIT_ROWS;
    for (p.cluster = 1; p.cluster < 8 && units * p.cluster * 2 <= slots && a.b.max_blocks >= 8 * p.cluster; p.cluster *= 2) {}
    p.grid = (u32)std::min<u64>(units * p.cluster, 0x7FFFFFFFu / p.cluster * p.cluster);
    return p;
  }
  // Units so few that several CTAs fit on each: clusters of as many as run at once (16 of them only for 8 units and less: more
  // such clusters do not find room together). A cluster's CTAs take 4 us and 0.2 us per block of theirs; stretches take 11 us
  // (with the join) and as much per block, but use all SMs and are even whatever the lengths. One sequence of 8 heads of 128:
  // 1000 tokens 7.0 us against 11.6, 4000 tokens 10.5 against 13.7, 8000 tokens 13.8 (clusters of 8: 17.5) against 14.8;
  // 4 sequences of 8000 27.4 against 32.8. Bounded, since only the longest sequence the table has room for is known here.
  const u64 units16 = tiles(SPLIT_ROWS) * H, nb = a.b.max_blocks, slots = 2ull * sm_count;
  u32 cluster = 0;
  for (u32 c = units16 <= 8 && nb > 192 ? 16 : 8; c >= 2; c /= 2) {
    if (units16 * c > slots) continue;
    if (nb > 64 * c || nb * (slots - units16 * c) > 28 * slots * c) break;
    cluster = nb <= 4 ? 0 : nb <= 2 * c ? std::max(2u, c / 2) : c;     // no more CTAs than there is something to do for
    break;
  }
  // One tile of 16 rows reads K and V once. With more rows the kernels for few rows read them once per tile, but they start and
  // end 7 us sooner, which decides when there is little to do: up to 8 K blocks (of 16 rows and one KV head, as many as fit
  // the table rows), 24 K in clusters, or 32 K where a sequence has two tiles only. Measured, us of few / many rows, heads of 128:
  //   64 tokens 6.4 / 13.4, 128 tokens 8.3 / 13.6, 200 tokens 16.4 / 12.9 (1.5 K, 4.1 K, 8.4 K blocks; groups of 4, 8 KV heads)
  //   clusters: 64 on 1000 14.7 / 25.1, 2 x 20 on 3000 17.1 / 30.4, 32 on 4000 20.8 / 29.6 (9.6 K, 12 K, 17 K); others: 100 on
  //   2000 38.8 / 28.0 (28 K)
  //   two tiles: 16 x 8 on 500 14.1 / 17.0, 10 x 8 on 1000 20.8 / 23.1, 32 x 8 on 500 24.4 / 24.0 (15 K, 16 K, 30 K; heads of 64: 20.2 / 21.2)
  const u64 rows = (u64)(max_q_len && max_q_len < a.b.n_tokens ? max_q_len : a.b.n_tokens) * a.group, few = units16 * (nb + UNIT_COST);
  if (rows <= SPLIT_ROWS || few <= (cluster ? 24576 : 8192) || (rows <= 2 * SPLIT_ROWS && few <= 32768)) {
    p.rows = SPLIT_ROWS;
    if (cluster) {
      p.kind = 3;
      p.cluster = cluster;
      p.grid = (u32)(units16 * cluster);
      return p;
    }
    p.kind = 1;
    const u64 units = units16, pieces = std::max<u64>(1, (nb + UNIT_COST) / MIN_STRETCH);
    // Short sequences are not cut: a CTA is through them sooner than a second kernel has joined their parts, the more so when
    // there is a unit for every SM. One sequence of 200 tokens, 8 heads of 128: 7.9 us against 11.3 cut, of 500 tokens 11.0
    // against 9.0; 32 sequences of 500: 13.1 against 19.3, of 1000 27.8 against 31.8.
    const bool cut = a.b.max_blocks > (units < (u64)sm_count ? 16u : 64u);
    p.most = units * (a.b.max_blocks + UNIT_COST);                   // work, if every sequence fills its table row
    p.grid = (u32)std::max<u64>(1, cut ? (p.most >= 2ull * sm_count * LONG_STRETCH ? 6ull * sm_count : std::min<u64>(2ull * sm_count, units * pieces))
                                       : std::min<u64>(2ull * sm_count, units));
    p.parts = p.grid > 1 && cut ? 2 * p.grid : 0;
  } else {
    p.kind = 2;
    p.rows = TC_ROWS;
    p.most = tiles(p.rows);
    const u64 units = p.most * H, pieces = std::max<u64>(1, (a.b.max_blocks + MIN_PIECE - 1) / MIN_PIECE);
    p.grid = (u32)std::max<u64>(1, std::min<u64>(sm_count, units * pieces));
    p.parts = pieces > 1 && (units < (u64)sm_count || a.b.max_blocks > 64) ? 4 * sm_count + 64 : 0;     // 64: rounding of the mean share
  }
  if (p.parts) p.scratch_bytes = plan_bytes(a.b.n_seqs) + (u64)p.parts * p.rows * (a.p.head_dim + 2) * 4;
  return p;
}

// Dynamic shared memory above 48 KB is asked for once per kernel and engine (a runtime call of half a microsecond).
template <class K>
static cudaError_t allow_smem(K kern, u32 which, u32 bytes, u64 *allowed) {
  if (*allowed >> which & 1) return cudaSuccess;
  const cudaError_t r = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (r == cudaSuccess) *allowed |= 1ull << which;
  return r;
}

template <class T, u32 D>
static cudaError_t launch_split(const AttendArgs &a, const AttendPlan &p, const KvMaps &m, cudaStream_t s, u64 *allowed, u32 *launches) {
  cudaError_t r = allow_smem(k_attend_split<T, D>, (D == 128) * 2 + a.fp16, SplitShape<D>::SMEM, allowed);
  if (r != cudaSuccess) return r;
  k_attend_split<T, D><<<p.grid, SPLIT_THREADS, SplitShape<D>::SMEM, s>>>(a, m, p.parts, 2 * p.sms, p.most);
  ++*launches;
  if ((r = cudaGetLastError()) != cudaSuccess || !p.parts) return r;
  const u64 rows = (u64)a.b.n_tokens * a.n_q_heads;
  if (p.grid > 2 * p.sms) return launch_join(k_attend_join_split<T, D, 16>, 512, rows, p.sms, s, launches, a, p.parts);
  return launch_join(k_attend_join_split<T, D, 4>, 128, rows, p.sms, s, launches, a, p.parts);
}

template <class T, u32 D, u32 CLUSTER, bool ANY>
static cudaError_t launch_cluster(const AttendArgs &a, const AttendPlan &p, const KvMaps &m, cudaStream_t s, u64 *allowed, u32 *launches) {
  constexpr u32 size = CLUSTER == 16 ? 4 : CLUSTER == 8 ? 3 : CLUSTER == 4 ? 2 : CLUSTER == 2 ? 1 : 0, width = D == 256 ? 2 : D == 128 ? 1 : 0;
  constexpr u32 which = 8 + ((ANY ? 10 : 0) + (ANY ? 4 : 5) * width + size) * 2 + __is_same(T, __half);      // 8 .. 51
  auto const kern = k_attend_cluster<T, D, CLUSTER, ANY>;
  if (CLUSTER > 8 && !(*allowed >> which & 1)) {
    const cudaError_t r = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (r != cudaSuccess) return r;
  }
  cudaError_t r = allow_smem(kern, which, SplitShape<D>::SMEM, allowed);
  if (r != cudaSuccess) return r;
  cudaLaunchConfig_t c{};
  c.gridDim = dim3(p.grid); c.blockDim = dim3(SPLIT_THREADS); c.dynamicSmemBytes = SplitShape<D>::SMEM; c.stream = s;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = CLUSTER; at.val.clusterDim.y = at.val.clusterDim.z = 1;
  c.attrs = &at; c.numAttrs = 1;
  ++*launches;
  return cudaLaunchKernelEx(&c, kern, a, m);
}
template <class T, u32 D>
static cudaError_t launch_cluster(const AttendArgs &a, const AttendPlan &p, const KvMaps &m, cudaStream_t s, u64 *allowed, u32 *launches) {
  switch (p.cluster) {
    case 2: return launch_cluster<T, D, 2, false>(a, p, m, s, allowed, launches);
    case 4: return launch_cluster<T, D, 4, false>(a, p, m, s, allowed, launches);
    case 8: return launch_cluster<T, D, 8, false>(a, p, m, s, allowed, launches);
    default: return launch_cluster<T, D, 16, false>(a, p, m, s, allowed, launches);
  }
}
template <class T, u32 D>
static cudaError_t launch_any(const AttendArgs &a, const AttendPlan &p, const KvMaps &m, cudaStream_t s, u64 *allowed, u32 *launches) {
  switch (p.cluster) {
    case 1: return launch_cluster<T, D, 1, true>(a, p, m, s, allowed, launches);
    case 2: return launch_cluster<T, D, 2, true>(a, p, m, s, allowed, launches);
    case 4: return launch_cluster<T, D, 4, true>(a, p, m, s, allowed, launches);
    default: return launch_cluster<T, D, 8, true>(a, p, m, s, allowed, launches);
  }
}

template <class T, u32 D>
static cudaError_t launch_tc(const AttendArgs &a, const AttendPlan &p, const KvMaps &m, cudaStream_t s, u64 *allowed, u32 *launches) {
  cudaError_t r = allow_smem(k_attend_tc<T, D>, 4 + (D == 128) * 2 + a.fp16, TcShape<D>::SMEM, allowed);
  if (r != cudaSuccess) return r;
  k_attend_tc<T, D><<<p.grid, TC_THREADS, TcShape<D>::SMEM, s>>>(a, m, p.parts, p.most);
  ++*launches;
  if ((r = cudaGetLastError()) != cudaSuccess || !p.parts) return r;
  return launch_join(k_attend_join_tc<T, D>, 128, ((u64)a.b.n_tokens * ((a.n_q_heads + 3) / 4) + 3) / 4, p.sms, s, launches, a, p.rows, p.parts);
}

cudaError_t launch_attend(const AttendArgs &a, const AttendPlan &p, const KvMaps &m, cudaStream_t s, u64 *allowed, u32 *launches) {
  if (p.kind == 2) {
    if (a.p.head_dim == 64) return a.fp16 ? launch_tc<__half, 64>(a, p, m, s, allowed, launches) : launch_tc<__nv_bfloat16, 64>(a, p, m, s, allowed, launches);
    return a.fp16 ? launch_tc<__half, 128>(a, p, m, s, allowed, launches) : launch_tc<__nv_bfloat16, 128>(a, p, m, s, allowed, launches);
  }
  if (p.kind == 3) {
    if (a.p.head_dim == 64) return a.fp16 ? launch_cluster<__half, 64>(a, p, m, s, allowed, launches) : launch_cluster<__nv_bfloat16, 64>(a, p, m, s, allowed, launches);
    return a.fp16 ? launch_cluster<__half, 128>(a, p, m, s, allowed, launches) : launch_cluster<__nv_bfloat16, 128>(a, p, m, s, allowed, launches);
  }
  if (p.kind == 1) {
    if (a.p.head_dim == 64) return a.fp16 ? launch_split<__half, 64>(a, p, m, s, allowed, launches) : launch_split<__nv_bfloat16, 64>(a, p, m, s, allowed, launches);
    return a.fp16 ? launch_split<__half, 128>(a, p, m, s, allowed, launches) : launch_split<__nv_bfloat16, 128>(a, p, m, s, allowed, launches);
  }
  if (a.p.head_dim <= 64) return a.fp16 ? launch_any<__half, 64>(a, p, m, s, allowed, launches) : launch_any<__nv_bfloat16, 64>(a, p, m, s, allowed, launches);
  if (a.p.head_dim <= 128) return a.fp16 ? launch_any<__half, 128>(a, p, m, s, allowed, launches) : launch_any<__nv_bfloat16, 128>(a, p, m, s, allowed, launches);
  return a.fp16 ? launch_any<__half, 256>(a, p, m, s, allowed, launches) : launch_any<__nv_bfloat16, 256>(a, p, m, s, allowed, launches);
}

}  // namespace kvt
