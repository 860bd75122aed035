// kvt_attend.cu — model-side operators on the paged KV pool: rotation + append of new tokens, attention of new tokens
// over everything their sequences hold in the pool.
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
};
template <> struct Elem<__half> {
  typedef __half2 T2;
  static __device__ __forceinline__ float2 up(u32 x) { return __half22float2(*reinterpret_cast<T2 *>(&x)); }
  static __device__ __forceinline__ u32 down(float a, float b) { T2 r = __floats2half2_rn(a, b); return *reinterpret_cast<u32 *>(&r); }
  static __device__ __forceinline__ float up1(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half down1(float x) { return __float2half_rn(x); }
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
// Where token t goes; the whole CTA asks. Every thread compares some of the starts with t, so the sequence is found
// with one round of loads instead of a chain of them.
struct Where { u32 seq, index; bool ok; };
__device__ __forceinline__ Where find_token(const KvBatch &b, u32 t, u32 *err) {
  u32 seq = 0;
  for (u32 s0 = 0; s0 < b.n_seqs; s0 += blockDim.x) {
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
  if (cut && threadIdx.x == 0) kv_err(err, KVERR_RANGE);
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

// One element (or one pair) at a time: any head size, stride and alignment.
template <class T>
__global__ void __launch_bounds__(128) k_append_any(AppendArgs a) {
  extern __shared__ float2 cs[];
  const u32 t = blockIdx.x;
  const Where w = find_token(a.b, t, a.err);
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

cudaError_t launch_append(const AppendArgs &a, cudaStream_t s, u32 *launches) {
  const u32 smem = a.rot_dim / 2 * sizeof(float2);
  if (a.fp16) k_append_any<__half><<<a.b.n_tokens, 128, smem, s>>>(a);
  else k_append_any<__nv_bfloat16><<<a.b.n_tokens, 128, smem, s>>>(a);
  ++*launches;
  return cudaGetLastError();
}

// ======================================================================================================
// Attention. Rows: the (token, query head of the group) pairs of one sequence and one KV head, token-major, so that row r
// is token r / group, head r % group. A CTA takes a tile of consecutive rows, which all read the same K and V.
// ======================================================================================================
// Keys row `token` (0 = first new token) sees: [lo, hi).
__device__ __forceinline__ void row_range(const AttendArgs &a, const Seq &q, u32 token, u32 &lo, u32 &hi) {
  const long long own = (long long)q.kv - q.n + token;     // index of the token in its sequence; < 0: it has none
  hi = a.full ? q.kv : own < 0 ? 0u : (u32)own + 1;
  lo = a.window && hi > a.window ? hi - a.window : 0u;
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

// Any head size up to 256, any alignment: 32-bit arithmetic on the CUDA cores. A CTA takes 16 rows, a warp 4 of them;
// K and V of 32 keys at a time go through shared memory as 32-bit values; a lane forms the scores of one key, and in
// the second product owns every 32nd column of the output.
constexpr u32 ANY_ROWS = 16, ANY_KEYS = 32, ANY_THREADS = 128, ANY_MAX_DIM = 256;

template <class T>
__global__ void __launch_bounds__(ANY_THREADS) k_attend_any(AttendArgs a) {
  extern __shared__ float sm[];
  const u32 D = a.p.head_dim, H = a.p.n_kv_heads, h = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float *const sq = sm, *const sk = sq + ANY_ROWS * D, *const sv = sk + ANY_KEYS * (D + 1);
  Seq q; u32 seq, tile;
  if (!find_tile<ANY_THREADS>(a, ANY_ROWS, blockIdx.x, q, seq, tile)) return;
  const u32 n_rows = q.n * a.group, r0 = tile * ANY_ROWS;
  for (u32 i = tid; i < ANY_ROWS * D; i += ANY_THREADS) {
    const u32 r = r0 + i / D, d = i % D;
    sq[i] = r < n_rows ? Elem<T>::up1(((const T *)a.q)[(q.t0 + r / a.group) * a.q_ts + (h * a.group + r % a.group) * a.q_hs + d]) : 0.0f;
  }
  u32 lo[4], hi[4];
#pragma unroll
  for (u32 x = 0; x < 4; ++x) {
    const u32 r = r0 + warp * 4 + x;
    lo[x] = hi[x] = 0;
    if (r < n_rows) row_range(a, q, r / a.group, lo[x], hi[x]);
  }
  u32 first, last, dummy;      // keys any row of the tile sees
  row_range(a, q, r0 / a.group, first, dummy);
  row_range(a, q, (min(r0 + ANY_ROWS, n_rows) - 1) / a.group, dummy, last);
  float m[4], l[4], acc[4][ANY_MAX_DIM / 32];
#pragma unroll
  for (u32 x = 0; x < 4; ++x) {
    m[x] = -INFINITY; l[x] = 0.0f;
#pragma unroll
    for (u32 c = 0; c < ANY_MAX_DIM / 32; ++c) acc[x][c] = 0.0f;
  }
  for (u32 k0 = first; k0 < last; k0 += ANY_KEYS) {
    __syncthreads();
    for (u32 i = tid; i < ANY_KEYS * D; i += ANY_THREADS) {
      const u32 kk = i / D, d = i - kk * D, key = k0 + kk;
      float kx = 0.0f, vx = 0.0f;
      if (key < last) {
        const u32 slot = a.b.table[seq * a.b.table_stride + key / BT];
        const T *kp = (const T *)slot_ptr(a.p, a.p.k, slot), *vp = (const T *)slot_ptr(a.p, a.p.v, slot);
        if (kp) {
          const u64 off = ((u64)(key % BT) * H + h) * D + d;
          kx = Elem<T>::up1(kp[off]); vx = Elem<T>::up1(vp[off]);
        } else if (d == 0) kv_err(a.err, KVERR_RANGE);
      }
      sk[kk * (D + 1) + d] = kx; sv[kk * D + d] = vx;
    }
    __syncthreads();
    float p[4] = {0, 0, 0, 0};
    for (u32 d = 0; d < D; ++d) {
      const float kx = sk[lane * (D + 1) + d];
#pragma unroll
      for (u32 x = 0; x < 4; ++x) p[x] += sq[(warp * 4 + x) * D + d] * kx;
    }
#pragma unroll
    for (u32 x = 0; x < 4; ++x) {
      const u32 key = k0 + lane;
      const float s = key >= lo[x] && key < hi[x] ? p[x] * a.scale_log2 : -INFINITY;
      float top = s;
#pragma unroll
      for (u32 o = 16; o; o /= 2) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
      const float now = fmaxf(m[x], top), ref = now == -INFINITY ? 0.0f : now, f = exp2f(m[x] - ref);
      p[x] = exp2f(s - ref);
      float sum = p[x];
#pragma unroll
      for (u32 o = 16; o; o /= 2) sum += __shfl_xor_sync(~0u, sum, o);
      l[x] = l[x] * f + sum;
      m[x] = now;
#pragma unroll
      for (u32 c = 0; c < ANY_MAX_DIM / 32; ++c) acc[x][c] *= f;
    }
    for (u32 kk = 0; kk < ANY_KEYS; ++kk) {
      float w[4];
#pragma unroll
      for (u32 x = 0; x < 4; ++x) w[x] = __shfl_sync(~0u, p[x], kk);
#pragma unroll
      for (u32 c = 0; c < ANY_MAX_DIM / 32; ++c) {
        const u32 d = c * 32 + lane;
        if (d < D) {
          const float vx = sv[kk * D + d];
#pragma unroll
          for (u32 x = 0; x < 4; ++x) acc[x][c] += w[x] * vx;
        }
      }
    }
  }
#pragma unroll
  for (u32 x = 0; x < 4; ++x) {
    const u32 r = r0 + warp * 4 + x;
    if (r >= n_rows) continue;
    const u32 t = q.t0 + r / a.group, hq = h * a.group + r % a.group;
    const float inv = l[x] > 0.0f ? 1.0f / l[x] : l[x] == 0.0f ? 0.0f : l[x];   // no key: zeros; a NaN stays one
    T *o = (T *)a.out + t * a.o_ts + hq * a.o_hs;
#pragma unroll
    for (u32 c = 0; c < ANY_MAX_DIM / 32; ++c) { const u32 d = c * 32 + lane; if (d < D) o[d] = Elem<T>::down1(acc[x][c] * inv); }
    if (a.lse && lane == 0) a.lse[(u64)t * a.n_q_heads + hq] = (m[x] + log2f(l[x])) * 0.69314718055994531f;
  }
}

cudaError_t launch_attend(const AttendArgs &a, int sm_count, cudaStream_t s, u32 *launches) {
  const u32 D = a.p.head_dim;
  const u64 tiles = ((u64)a.b.n_tokens * a.group + ANY_ROWS - 1) / ANY_ROWS + a.b.n_seqs;   // no more than this many
  const u32 smem = (ANY_ROWS * D + ANY_KEYS * (D + 1) + ANY_KEYS * D) * 4;
  auto kern = a.fp16 ? k_attend_any<__half> : k_attend_any<__nv_bfloat16>;
  cudaError_t r = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (r != cudaSuccess) return r;
  kern<<<dim3((u32)tiles, a.p.n_kv_heads), ANY_THREADS, smem, s>>>(a);
  ++*launches;
  return cudaGetLastError();
}

}  // namespace kvt
