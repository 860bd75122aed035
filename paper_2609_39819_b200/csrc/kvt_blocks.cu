// kvt_blocks.cu — model-side operators that choose among the blocks of the paged KV pool: bounds of a block's keys, selection of
// blocks by them, attention over the selected blocks, attention weight per block, eviction by it.
#include "kvt_attend.cuh"

#include <algorithm>

namespace kvt {

__device__ __forceinline__ u32 max_over_warp(u32 x) { return __reduce_max_sync(~0u, x); }
__device__ __forceinline__ float sum_over_warp(float x) {
#pragma unroll
  for (u32 o = 16; o; o /= 2) x += __shfl_xor_sync(~0u, x, o);
  return x;
}

// ======================================================================================================
// Bounds of a block's keys. For one block and KV head, channel d: up_d = max_r k_rd, down_d = max_r -k_rd over its 16 tokens, both
// as whole steps of 2^e, rounded up: ceil(x 2^-e), where e is the least with max |k| <= 127 * 2^e. For any query q then
//   q.k_r <= sum_d max(q_d, 0) up_d + max(-q_d, 0) down_d          for every key of the block.
// Steps are powers of two so that nothing but the rounding up is rounded, and equal keys get equal codes whoever makes them.
// Bound by reading the keys once: 130,500 tokens, 8 heads of 128 (284 MB) 48 us in a captured graph, 90 % of the measured copy bandwidth; a
// step of 32 sessions 3.5 us, launch and three dependent loads.
// ======================================================================================================
constexpr int BOUND_E_MIN = -126, BOUND_E_MAX = 103;     // 2^24 steps of 2^103 are a 32-bit number
__device__ __forceinline__ int bound_exponent(float most) {
  const u32 b = __float_as_uint(most);
  const int e = (int)(b >> 23) - 127 - 6 + ((b & 0x7FFFFF) > 0x7E0000);      // 127 = 1.984375 * 2^6
  return max(BOUND_E_MIN, min(BOUND_E_MAX, b >> 23 ? e : BOUND_E_MIN));
}
__device__ __forceinline__ int bound_code(float x, float inv) {
  float c = fminf(ceilf(x * inv), 127.0f);
  if (x > 0.0f) c = fmaxf(c, 1.0f);                      // the product may have vanished
  return (int)fmaxf(c, -127.0f);
}
__device__ __forceinline__ float number(float x) { return x == x ? x : 0.0f; }       // a NaN does not count

template <class T> struct Pair;
template <> struct Pair<__nv_bfloat16> { typedef __nv_bfloat162 T2; };
template <> struct Pair<__half> { typedef __half2 T2; };

// A CTA looks at `rows` tokens, one per thread; a warp takes a head of a block that one of them fills. VEC: heads of D channels, 16 bytes
// of a token per lane, all loads of a lane in flight at once.
constexpr u32 BOUND_ROWS = 64;
template <class T, u32 D>
__global__ void __launch_bounds__(256) k_bound_keys(BoundArgs a, u32 rows) {
  __shared__ u32 s_slot[BOUND_ROWS], s_n;
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = a.p.n_kv_heads;
  if (blockIdx.x == 0 && blockIdx.y == 0)                // one CTA looks all starts over
    for (u32 s = tid; s < a.b.n_seqs; s += 256) if (a.b.q_start[s] > a.b.q_start[s + 1]) kv_err(a.err, KVERR_RANGE);
  if (tid == 0) s_n = 0;
  __syncthreads();
  const u32 t = blockIdx.x * rows + tid;
  if (tid < rows && t < a.b.n_tokens) {
    u32 lo = 0, hi = a.b.n_seqs;                         // the sequence: the first that ends behind the token
    while (lo < hi) { const u32 mid = (lo + hi) / 2; if (a.b.q_start[mid + 1] <= t) lo = mid + 1; else hi = mid; }
    if (lo < a.b.n_seqs) {
      const u32 from = a.b.q_start[lo], to = a.b.q_start[lo + 1], kv = a.b.kv_len[lo], index = kv - (to - t);
      if (t < from || to > a.b.n_tokens || kv > (u64)a.b.max_blocks * BT || kv < to - from) kv_err(a.err, KVERR_RANGE);
      if (t >= from && kv >= to - t && index / BT < a.b.max_blocks && index % BT == BT - 1) {
        const u32 slot = a.b.table[lo * a.b.table_stride + index / BT];
        if (slot >= a.k.n_slots || !slot_ptr(a.p, a.p.k, slot)) kv_err(a.err, KVERR_RANGE);
        else s_slot[atomicAdd(&s_n, 1u)] = slot;
      }
    }
  }
  __syncthreads();
  const u32 n_items = s_n * H;
  for (u32 item = blockIdx.y * 8 + warp; item < n_items; item += 8 * gridDim.y) {
    const u32 which = item / H, h = item - which * H, slot = s_slot[which];
    const u16 *const src = (const u16 *)slot_ptr(a.p, a.p.k, slot);
    int8_t *const to = a.k.codes + ((u64)slot * H + h) * 2 * a.k.width;
    u8 *const exp_to = a.k.exps + (u64)slot * H + h;
    if constexpr (D != 0) {
      typedef typename Pair<T>::T2 T2;
      constexpr u32 LANES = D / 8, PER = 32 / LANES, STEPS = BT / PER;       // lanes of a token, tokens of a load, loads
      const u32 c = lane % LANES * 8;
      uint4 v[STEPS];
#pragma unroll
      for (u32 y = 0; y < STEPS; ++y) v[y] = *(const uint4 *)(src + (u64)(y * PER + lane / LANES) * H * D + h * D + c);
      T2 hi[4], lo[4];
#pragma unroll
      for (u32 z = 0; z < 4; ++z) {
        auto part = [&](u32 y) { u32 x = z == 0 ? v[y].x : z == 1 ? v[y].y : z == 2 ? v[y].z : v[y].w; return *reinterpret_cast<T2 *>(&x); };
        hi[z] = lo[z] = part(0);
#pragma unroll
        for (u32 y = 1; y < STEPS; ++y) { hi[z] = __hmax2(hi[z], part(y)); lo[z] = __hmin2(lo[z], part(y)); }
#pragma unroll
        for (u32 o = LANES; o < 32; o *= 2) {
          hi[z] = __hmax2(hi[z], __shfl_xor_sync(~0u, hi[z], o));
          lo[z] = __hmin2(lo[z], __shfl_xor_sync(~0u, lo[z], o));
        }
      }
      float up[8], down[8], most = 0.0f;
#pragma unroll
      for (u32 z = 0; z < 4; ++z) {
        const float2 x = Elem<T>::up(*reinterpret_cast<u32 *>(&hi[z])), y = Elem<T>::up(*reinterpret_cast<u32 *>(&lo[z]));
        up[2 * z] = number(x.x); up[2 * z + 1] = number(x.y); down[2 * z] = -number(y.x); down[2 * z + 1] = -number(y.y);
      }
#pragma unroll
      for (u32 z = 0; z < 8; ++z) most = fmaxf(most, fmaxf(fabsf(up[z]), fabsf(down[z])));
      const int e = bound_exponent(__uint_as_float(max_over_warp(__float_as_uint(most))));
      const float inv = __uint_as_float((u32)(127 - e) << 23);
      u32 x[4] = {0, 0, 0, 0};
#pragma unroll
      for (u32 z = 0; z < 8; ++z) {
        x[z / 4] |= (u32)(bound_code(up[z], inv) & 0xFF) << (z % 4 * 8);
        x[2 + z / 4] |= (u32)(bound_code(down[z], inv) & 0xFF) << (z % 4 * 8);
      }
      if (lane < LANES) {
        *(uint2 *)(to + c) = make_uint2(x[0], x[1]);
        *(uint2 *)(to + D + c) = make_uint2(x[2], x[3]);
      }
      if (lane == 0) *exp_to = (u8)(e + 127);
    } else {
      const u32 d = a.p.head_dim;
      float up[8], down[8], most = 0.0f;
#pragma unroll
      for (u32 z = 0; z < 8; ++z) {
        const u32 c = lane + 32 * z;
        float hi = -INFINITY, lo = INFINITY;
        if (c < d) for (u32 r = 0; r < BT; ++r) {
          const float x = Elem<T>::up1(((const T *)src)[(u64)r * H * d + (u64)h * d + c]);
          hi = fmaxf(hi, x); lo = fminf(lo, x);          // neither takes a NaN
        }
        up[z] = hi < lo || c >= d ? 0.0f : hi; down[z] = hi < lo || c >= d ? 0.0f : -lo;
        most = fmaxf(most, fmaxf(fabsf(up[z]), fabsf(down[z])));
      }
      const int e = bound_exponent(__uint_as_float(max_over_warp(__float_as_uint(most))));
      const float inv = __uint_as_float((u32)(127 - e) << 23);
#pragma unroll
      for (u32 z = 0; z < 8; ++z) {
        const u32 c = lane + 32 * z;
        if (c < a.k.width) { to[c] = (int8_t)bound_code(up[z], inv); to[a.k.width + c] = (int8_t)bound_code(down[z], inv); }
      }
      if (lane == 0) *exp_to = (u8)(e + 127);
    }
  }
}

template <class T>
static void bound_keys(const BoundArgs &a, dim3 grid, u32 rows, cudaStream_t s) {
  const bool aligned = (((uintptr_t)a.p.k.base | (uintptr_t)a.p.k.tail) & 15) == 0;
  if (aligned && a.p.head_dim == 128) k_bound_keys<T, 128><<<grid, 256, 0, s>>>(a, rows);
  else if (aligned && a.p.head_dim == 64) k_bound_keys<T, 64><<<grid, 256, 0, s>>>(a, rows);
  else k_bound_keys<T, 0><<<grid, 256, 0, s>>>(a, rows);
}
cudaError_t launch_bound(const BoundArgs &a, int sm_count, cudaStream_t s, u32 *launches) {
  // long batches: several blocks per CTA, since finding them costs as much as one
  const u32 rows = a.b.n_tokens >= 64u * sm_count ? BOUND_ROWS : 16, ctas = (a.b.n_tokens + rows - 1) / rows;
  const dim3 grid(ctas, std::max(1u, std::min(a.p.n_kv_heads, 2u * sm_count / ctas)));
  ++*launches;
  if (a.fp16) bound_keys<__half>(a, grid, rows, s);
  else bound_keys<__nv_bfloat16>(a, grid, rows, s);
  return cudaGetLastError();
}

// ======================================================================================================
// The m-th largest of n keys, for a whole CTA, by digits from the top: 12, 12 and 8 bits. Once few keys begin like the one in question they
// are put into a list, which the next digits are counted in. each(f) calls f with every key that is this thread's.
// A key x is among the m largest if x > at, or x == at and fewer than `ties` keys equal to it come before.
// ======================================================================================================
struct Kth { u32 at, ties; };
constexpr u32 KTH_LIST = 1024;
template <u32 THREADS, class Each>
__device__ __forceinline__ Kth kth_largest(Each each, u32 n, u32 m) {
  constexpr u32 BINS = 4096, PER = BINS / THREADS, WARPS = THREADS / 32;
  __shared__ u32 s_hist[BINS], s_list[KTH_LIST], s_sum[WARPS], s_digit, s_left, s_here, s_n;
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (m >= n) return Kth{0, ~0u};                        // all: no key is below 0
  u32 prefix = 0, left = m, listed = 0;                  // prefix: the digits in front of the one in hand
#pragma unroll 1
  for (u32 bits = 32; bits;) {
    const u32 shift = bits == 32 ? 20 : bits == 20 ? 8 : 0, mask = (1u << (bits - shift)) - 1;
    for (u32 i = tid; i < BINS; i += THREADS) s_hist[i] = 0;
    if (tid == 0) s_n = 0;
    __syncthreads();
    auto count = [&](u32 x) { if ((u64)x >> bits == prefix) atomicAdd(&s_hist[x >> shift & mask], 1u); };
    if (listed) { for (u32 i = tid; i < listed; i += THREADS) count(s_list[i]); }
    else each(count);
    __syncthreads();
    // this thread's digits: PER of them downwards from BINS - 1 - tid * PER
    u32 c[PER], sum = 0;
#pragma unroll
    for (u32 y = 0; y < PER; ++y) { c[y] = s_hist[BINS - 1 - tid * PER - y]; sum += c[y]; }
    u32 incl = sum;
#pragma unroll
    for (u32 o = 1; o < 32; o *= 2) { const u32 z = __shfl_up_sync(~0u, incl, o); if (lane >= o) incl += z; }
    if (lane == 31) s_sum[warp] = incl;
    __syncthreads();
    u32 before = incl - sum;
#pragma unroll 8
    for (u32 w = 0; w < WARPS; ++w) before += w < warp ? s_sum[w] : 0u;
    if (before < left && left <= before + sum) {
#pragma unroll
      for (u32 y = 0; y < PER; ++y) {
        if (before < left && left <= before + c[y]) { s_digit = BINS - 1 - tid * PER - y; s_left = left - before; s_here = c[y]; }
        before += c[y];
      }
    }
    __syncthreads();
    prefix = prefix << (bits - shift) | s_digit;
    left = s_left;
    bits = shift;
    const u32 here = s_here;
    if (here == left) return Kth{prefix << bits, ~0u};   // all that begin like this
    if (bits && !listed && here <= KTH_LIST) {
      each([&](u32 x) { if (x >> bits == prefix) s_list[atomicAdd(&s_n, 1u)] = x; });
      listed = here;
    }
    __syncthreads();                                     // the digit is read, the list is written
  }
  return Kth{prefix, left};
}

// Deals the numbers i of [0, n) out in order: pick(i) says which list each goes to (bit 0: the first, bit 1: the second), put(i, which, place)
// is called with its place in that list. Every warp has a stretch of its own.
template <u32 THREADS, class Pick, class Put>
__device__ __forceinline__ void deal(u32 n, Pick pick, Put put) {
  constexpr u32 WARPS = THREADS / 32;
  __shared__ u32 s_n[WARPS][2];
  const u32 lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = (n + THREADS - 1) / THREADS * 32;
  const u32 from = min(n, warp * per), to = min(n, from + per);
  u32 count[2] = {0, 0};
  for (u32 i = from; i < to; i += 32) {
    const u32 w = i + lane < to ? pick(i + lane) : 0;
    count[0] += __popc(__ballot_sync(~0u, w & 1)); count[1] += __popc(__ballot_sync(~0u, w & 2));
  }
  __syncthreads();
  if (lane == 0) { s_n[warp][0] = count[0]; s_n[warp][1] = count[1]; }
  __syncthreads();
  u32 at[2] = {0, 0};
  for (u32 w = 0; w < warp; ++w) { at[0] += s_n[w][0]; at[1] += s_n[w][1]; }
  for (u32 i = from; i < to; i += 32) {
    const u32 w = i + lane < to ? pick(i + lane) : 0;
    const u32 b0 = __ballot_sync(~0u, w & 1), b1 = __ballot_sync(~0u, w & 2), below = (1u << lane) - 1;
    if (w & 1) put(i + lane, 0u, at[0] + __popc(b0 & below));
    if (w & 2) put(i + lane, 1u, at[1] + __popc(b1 & below));
    at[0] += __popc(b0); at[1] += __popc(b1);
  }
}

// Order of floating numbers as order of whole ones.
__device__ __forceinline__ u32 ordered(float x) {
  const u32 b = __float_as_uint(x);
  return b ^ ((u32)((int)b >> 31) | 0x80000000u);
}

// ======================================================================================================
// Selection of blocks. The group's queries of a token and KV head are added up, what is above zero and what is below apart, and
// rounded to 8 bits without sign: u = rint(2^-f sum), f the least with max <= 255 * 2^f. With the bounds (up, down, e) of a block
//   score = 2^e sum_d u+_d up_d + u-_d down_d,
// an estimate of what bounds the sum of the group's products with any key of the block (in steps of 2^f, which all blocks of the query
// share; the bounds are rounded up, but the queries to the nearest, so it may be short of that by half a step per channel). The sum is of at most 512 products of 255 * 127, a whole number below 2^24, so it is a 32-bit floating number
// exactly, and so is the score: all kernels, batches and orders of summation give the same selection, bit by bit.
// Two kernels: scores into scratch, then each list from its scores. 8 KV heads of 128, groups of 4, lists of 64, in a captured graph: one
// token on 258,047 17.3 us (floor 5.1: 33 MB of codes; the kernels take 8 and 7 us, each of them a chain of dependent loads), 500 tokens
// on 130,500 123 us (71 and 48: scores and their stores, 134 MB of them), a prompt of 8192 166 us.
// ======================================================================================================
// New tokens [t0, t0 + n) of a sequence that lie among the tokens in hand; index of the first in its sequence.
struct Part { u32 t0, n; long long index; };
__device__ __forceinline__ Part part_of(const SelectArgs &a, u32 s) {
  const Seq q = load_seq(a.b, s, a.err);
  Part p;
  p.t0 = max(q.t0, a.slab_begin);
  const u32 end = min(q.t0 + q.n, a.slab_end);
  p.n = end > p.t0 ? end - p.t0 : 0;
  p.index = (long long)q.kv - q.n + (p.t0 - q.t0);
  return p;
}

__device__ __forceinline__ void mma_u8s8(int (&c)[4], u32 a0, u32 a1, u32 a2, u32 a3, u32 b0, u32 b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Scores of M * 16 tokens of one sequence with one KV head's share of the blocks. blockIdx.x: tile of tokens, y: KV head, z: share of the
// blocks. A warp takes 8 blocks at a time, with a ring of bulk copies of its own: the codes of the next groups come in while one is worked
// on, those of the first while the queries are rounded. A lane's 16 bytes of every 64 of a block's codes are the operand of the matrix
// instruction if the channels are counted in that order on both sides.
constexpr u32 SCORE_STAGES = 4;
template <u32 G> struct ScoreRing { static constexpr u32 PITCH = G * 64 + 64 /* lanes of two blocks on different banks */, STAGE = 8 * PITCH, SMEM = 8 * SCORE_STAGES * STAGE; };
template <class T, u32 G, u32 M>      // G: 64-byte parts of (up, down)
__global__ void __launch_bounds__(256, G > 4 ? 1 : 2) k_score_blocks(SelectArgs a, u32 shares) {
  typedef ScoreRing<G> S;
  constexpr u32 ROW = G * 64 + 16, TOKENS = M * 16;
  extern __shared__ __align__(16) u8 smem_raw[];
  __shared__ __align__(8) u64 bars[8 * SCORE_STAGES];
  __shared__ __align__(16) u8 su[TOKENS * ROW];
  __shared__ u32 s_sum[8], s_seq, s_tile;
  asm volatile("griddepcontrol.launch_dependents;");
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, h = blockIdx.y, H = a.n_kv_heads, W = a.k.width;
  // the tile's sequence
  if (tid == 0) s_seq = ~0u;
  u32 base = 0;
  for (u32 s0 = 0; s0 < a.b.n_seqs; s0 += 256) {
    const u32 n = s0 + tid < a.b.n_seqs ? (part_of(a, s0 + tid).n + TOKENS - 1) / TOKENS : 0;
    u32 incl = n;
#pragma unroll
    for (u32 o = 1; o < 32; o *= 2) { const u32 y = __shfl_up_sync(~0u, incl, o); if (lane >= o) incl += y; }
    __syncthreads();
    if (lane == 31) s_sum[warp] = incl;
    __syncthreads();
    u32 before = base, all = base;
#pragma unroll
    for (u32 w = 0; w < 8; ++w) { if (w < warp) before += s_sum[w]; all += s_sum[w]; }
    if (blockIdx.x >= before + incl - n && blockIdx.x < before + incl) { s_seq = s0 + tid; s_tile = blockIdx.x - (before + incl - n); }
    base = all;
  }
  __syncthreads();
  const u32 seq = s_seq;
  if (seq == ~0u) return;
  Part p = part_of(a, seq);
  p.t0 += s_tile * TOKENS; p.index += s_tile * TOKENS; p.n = min(TOKENS, p.n - s_tile * TOKENS);
  // blocks that any of the tokens may choose from: [first, its own - last]; scored from a multiple of 8 on
  const long long own = (p.index + p.n - 1) / BT;
  const long long end_ = p.index + p.n - 1 < 0 ? 0 : min(own + 1 - (long long)a.last, (long long)a.b.max_blocks);
  const u32 begin = a.first & ~7u, end = end_ > (long long)begin ? (u32)end_ : begin;
  const u32 per = ((end - begin + shares - 1) / shares + 63) / 64 * 64;
  const u32 b0 = begin + min(end - begin, blockIdx.z * per), b1 = begin + min(end - begin, (blockIdx.z + 1) * per);
  if (b0 >= b1 || own + 1 <= (long long)a.n_blocks) return;       // nobody chooses

  const u32 j = lane % 4, r = lane / 4;
  const u32 *const table = a.b.table + seq * a.b.table_stride;
  const u32 ring = smem_addr(smem_raw) + warp * SCORE_STAGES * S::STAGE, bar0 = smem_addr(bars) + warp * SCORE_STAGES * 8;
  if (lane == 0) {
    for (u32 i = 0; i < SCORE_STAGES; ++i) bar_init(bar0 + i * 8, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncwarp();
  auto slot_of = [&](u32 b) { return lane < 8 && b + lane < b1 ? table[b + lane] : ~0u; };      // lane i: slot of block b + i
  u32 e[SCORE_STAGES];                   // lane i: exponent of block i of the stage; 256: none
  auto load = [&](u32 st, u32 b, u32 slot) {
    const bool fine = slot < a.k.n_slots;
    if (!fine && lane < 8 && b + lane < b1) kv_err(a.err, KVERR_RANGE);
    const u32 n = __popc(__ballot_sync(~0u, fine)), bar = bar0 + st * 8;
    if (lane == 0) bar_expect(bar, n * 2 * W);
    __syncwarp();
    if (fine)
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                   ::"r"(ring + st * S::STAGE + lane * S::PITCH), "l"(a.k.codes + ((u64)slot * H + h) * 2 * W), "r"(2 * W), "r"(bar) : "memory");
    return fine ? (u32)a.k.exps[(u64)slot * H + h] : 256u;
  };
  u32 b = b0 + warp * 8, phase = 0;
#pragma unroll
  for (u32 st = 0; st < SCORE_STAGES; ++st) { e[st] = 256; if (b + 64 * st < b1) e[st] = load(st, b + 64 * st, slot_of(b + 64 * st)); }
  u32 slot = slot_of(b + 64 * SCORE_STAGES);

  // queries: a warp per token; V channels in a row per lane
  constexpr u32 V = G;
  for (u32 t = warp; t < TOKENS; t += 8) {
    double up[V], down[V], most = 0.0;
#pragma unroll
    for (u32 z = 0; z < V; ++z) up[z] = down[z] = 0.0;
    if (t < p.n && lane * V < a.head_dim) {
      const u16 *const src = (const u16 *)a.q + (u64)(p.t0 + t) * a.q_ts + (u64)(h * a.group) * a.q_hs + lane * V;
      const bool vec = lane * V + V <= a.head_dim && (((uintptr_t)src | a.q_hs * 2) & (V * 2 - 1)) == 0;
      for (u32 y0 = 0; y0 < a.group; y0 += 4) {
        u32 raw[4][V / 2];
#pragma unroll
        for (u32 y = 0; y < 4; ++y) {
          const u16 *const from = src + min(y0 + y, a.group - 1) * a.q_hs;
          if (vec) {
            if (V == 2) raw[y][0] = *(const u32 *)from;
            else if (V == 4) *(uint2 *)raw[y] = *(const uint2 *)from;
            else *(uint4 *)raw[y] = *(const uint4 *)from;
          } else {
#pragma unroll
            for (u32 z = 0; z < V / 2; ++z) {
              const u32 c = lane * V + 2 * z;
              raw[y][z] = (c < a.head_dim ? (u32)from[2 * z] : 0u) | (c + 1 < a.head_dim ? (u32)from[2 * z + 1] << 16 : 0u);
            }
          }
        }
#pragma unroll
        for (u32 y = 0; y < 4; ++y) {
          if (y0 + y >= a.group) continue;
#pragma unroll
          for (u32 z = 0; z < V; ++z) {
            const float2 pair = Elem<T>::up(raw[y][z / 2]);
            const float top = __is_same(T, __half) ? 65504.0f : 3.3895314e38f;       // Inf counts as the largest number
            const float v = fminf(fmaxf(number(z % 2 ? pair.y : pair.x), -top), top);
            up[z] += (double)fmaxf(v, 0.0f); down[z] += (double)fmaxf(-v, 0.0f);
          }
        }
      }
    }
#pragma unroll
    for (u32 z = 0; z < V; ++z) most = fmax(most, fmax(up[z], down[z]));
    // the exponent alone, and whether it is above 255 / 256 of the power: 255 = 1.9921875 * 2^7
    const u64 bits = (u64)__double_as_longlong(most);
    const int e = most > 0.0 ? (int)(bits >> 52) - 1023 - 7 + ((bits & 0xFFFFFFFFFFFFFull) > 0xFE00000000000ull) : -2000;
    const int f_ = (int)__reduce_max_sync(~0u, e), f = f_ == -2000 ? 0 : f_;
    const double inv = __longlong_as_double((u64)(1023 - f) << 52);
    u32 pu[V / 2 > 1 ? V / 4 : 1], pd[V / 2 > 1 ? V / 4 : 1];
#pragma unroll
    for (u32 z = 0; z < V; ++z) {
      const u32 x = __double2uint_rn(up[z] * inv), y = __double2uint_rn(down[z] * inv);
      if (z % 4 == 0) { pu[z / 4] = x; pd[z / 4] = y; } else { pu[z / 4] |= x << (z % 4 * 8); pd[z / 4] |= y << (z % 4 * 8); }
    }
    // (a lane's channels lie all in front of the width or all behind it: it is a multiple of 16)
    if (lane * V < W) {
      u8 *const to = su + t * ROW + lane * V;
      if (V == 2) { *(u16 *)to = (u16)pu[0]; *(u16 *)(to + W) = (u16)pd[0]; }
      else if (V == 4) { *(u32 *)to = pu[0]; *(u32 *)(to + W) = pd[0]; }
      else { *(uint2 *)to = make_uint2(pu[0], pu[V / 4 - 1]); *(uint2 *)(to + W) = make_uint2(pd[0], pd[V / 4 - 1]); }
    }
    for (u32 c = 2 * W + lane; c < G * 64; c += 32) su[t * ROW + c] = 0;
  }
  __syncthreads();
  uint4 qa[M][G][2];
#pragma unroll
  for (u32 m = 0; m < M; ++m)
#pragma unroll
    for (u32 g = 0; g < G; ++g) {
      qa[m][g][0] = *(const uint4 *)(su + (m * 16 + r) * ROW + g * 64 + j * 16);
      qa[m][g][1] = *(const uint4 *)(su + (m * 16 + r + 8) * ROW + g * 64 + j * 16);
    }
  const u64 token = (u64)H * a.scores_stride;
  u32 *out = a.scores + ((u64)(p.t0 - a.slab_begin + r) * H + h) * a.scores_stride + b + 2 * j;      // token r's, blocks b + 2 j and the next
  bool ok = true;
  while (ok && b < b1) {
#pragma unroll
    for (u32 st = 0; st < SCORE_STAGES; ++st) {
      if (b >= b1 || !(ok = __all_sync(~0u, bar_wait(bar0 + st * 8, phase)))) break;
      // scale and, where there is no slot, a score below all others
      const u32 e0 = __shfl_sync(~0u, e[st], 2 * j), e1 = __shfl_sync(~0u, e[st], 2 * j + 1);
      const float s0 = __uint_as_float(e0 > 255 ? 0u : e0 << 23), s1 = __uint_as_float(e1 > 255 ? 0u : e1 << 23), d0 = e0 > 255 ? -INFINITY : 0.0f, d1 = e1 > 255 ? -INFINITY : 0.0f;
      int c[M][4];
#pragma unroll
      for (u32 m = 0; m < M; ++m) c[m][0] = c[m][1] = c[m][2] = c[m][3] = 0;
#pragma unroll
      for (u32 g = 0; g < G; ++g) {
        u32 v[4];
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(ring + st * S::STAGE + r * S::PITCH + g * 64 + j * 16) : "memory");
#pragma unroll
        for (u32 m = 0; m < M; ++m) {
          mma_u8s8(c[m], qa[m][g][0].x, qa[m][g][1].x, qa[m][g][0].y, qa[m][g][1].y, v[0], v[1]);
          mma_u8s8(c[m], qa[m][g][0].z, qa[m][g][1].z, qa[m][g][0].w, qa[m][g][1].w, v[2], v[3]);
        }
      }
      __syncwarp();                      // the stage is read
      if (b + 64 * SCORE_STAGES < b1) {
        e[st] = load(st, b + 64 * SCORE_STAGES, slot);
        slot = slot_of(b + 64 * (SCORE_STAGES + 1));
      }
#pragma unroll
      for (u32 m = 0; m < M; ++m)
#pragma unroll
        for (u32 y = 0; y < 2; ++y)
          if (m * 16 + r + 8 * y < p.n)
            *(uint2 *)(out + (m * 16 + 8 * y) * token) = make_uint2(ordered(fmaf((float)c[m][2 * y], s0, d0)), ordered(fmaf((float)c[m][2 * y + 1], s1, d1)));
      b += 64; out += 64;
    }
    phase ^= 1;
  }
  if (!ok) {                             // let the copies in flight land, for a while
    if (lane == 0) kv_err(a.err, KVERR_WAIT);
    for (u32 i = 0; i < SCORE_STAGES; ++i) for (u32 y = 0; y < 2; ++y) bar_wait(bar0 + i * 8, y);
  }
}

// The blocks of a token and KV head, in order: the first ones, those of the largest scores, the last ones.
constexpr u32 PICK_CAP = 512;            // candidates
// VECTORS: the row's scores in registers, 16 bytes so many times per thread; 0: in shared memory as far as `held` of them fit, else where they are.
template <u32 THREADS, u32 VECTORS>
__global__ void __launch_bounds__(THREADS) k_pick_blocks(SelectArgs a, u32 held) {
  constexpr u32 WARPS = THREADS / 32;
  extern __shared__ u32 s_keys[];
  __shared__ u32 s_n, s_least[WARPS];
  __shared__ u64 s_key[PICK_CAP];
  __shared__ u32 s_bits[THREADS], s_count[WARPS];        // VECTORS: a bit per block that is taken
  __shared__ u8 taken[PICK_CAP];         // else: whether a candidate is among the m largest
  const u32 tid = threadIdx.x, H = a.n_kv_heads, t = a.slab_begin + blockIdx.x / H, h = blockIdx.x % H;
  const Where w = find_token<false>(a.b, t, a.err);
  asm volatile("griddepcontrol.wait;" ::: "memory");     // the scores; the batch's arrays are older than the kernel before this one
  if (w.seq >= a.b.n_seqs) return;                       // behind the last sequence
  int32_t *const out = a.out + ((u64)t * H + h) * a.n_blocks;
  const u32 own = w.index / BT;
  if (!w.ok || own < a.n_blocks) {                       // all there are
    for (u32 i = tid; i < a.n_blocks; i += THREADS) out[i] = w.ok && i <= own ? (int32_t)i : -1;
    return;
  }
  // of the blocks [first, end) m are taken
  const u32 end = own + 1 - a.last, n = end - a.first, m = a.n_blocks - a.first - a.last;
  const u32 *const scores = a.scores + ((u64)(t - a.slab_begin) * H + h) * a.scores_stride;
  for (u32 i = tid; i < a.first + a.last; i += THREADS) out[i < a.first ? i : i + m] = i < a.first ? (int32_t)i : (int32_t)(end + i - a.first);
  if (!m) return;
  u32 most = 0;
  constexpr u32 VN = VECTORS ? VECTORS : 1;
  uint4 v[VN] = {};
  auto mine = [&](u32 y, u32 z) { return z == 0 ? v[y].x : z == 1 ? v[y].y : z == 2 ? v[y].z : v[y].w; };
  if constexpr (VECTORS > 0) {
#pragma unroll
    for (u32 y = 0; y < VN; ++y) {
      const u32 i = 4 * (tid + y * THREADS);
      v[y] = i < end ? *(const uint4 *)(scores + i) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (u32 y = 0; y < VN; ++y) {
      const u32 i = 4 * (tid + y * THREADS);
      if (i < a.first || i + 4 > end) {                  // what is not to be chosen counts as 0, and is known by its place
        if (i < a.first || i >= end) v[y].x = 0;
        if (i + 1 < a.first || i + 1 >= end) v[y].y = 0;
        if (i + 2 < a.first || i + 2 >= end) v[y].z = 0;
        if (i + 3 < a.first || i + 3 >= end) v[y].w = 0;
      }
      most = max(max(most, max(v[y].x, v[y].y)), max(v[y].z, v[y].w));
    }
  } else {
    for (u32 i = tid; i < n; i += THREADS) {
      const u32 x = scores[a.first + i];
      if (n <= held) s_keys[i] = x;
      most = max(most, x);
    }
  }
  // Few of many. With k = m / warps, rounded up, every warp has k threads whose largest is not below the k-th largest of these; the least
  // of the warps' k-th is below at least m scores, then, and above nearly all others. What it leaves is put in order by counting.
  const u32 k = (m + WARPS - 1) / WARPS;
  if (k <= 16 && n >= 4 * THREADS) {
    u32 x = most, kth = 0;
    for (u32 y = 0; y < k; ++y) {
      kth = __reduce_max_sync(~0u, x);
      if (tid % 32 == __ffs(__ballot_sync(~0u, x == kth)) - 1) x = 0;
    }
    if (tid % 32 == 0) s_least[tid / 32] = kth;
    if (tid == 0) s_n = 0;
    s_bits[tid] = 0;
    __syncthreads();
    u32 least = s_least[tid % WARPS];
    least = __reduce_min_sync(~0u, least);
    auto candidate = [&](u32 x, u32 i) {                 // i: number of the block; of equal scores the lower one is the larger key
      const u32 at = atomicAdd(&s_n, 1u);
      if (at < PICK_CAP) s_key[at] = (u64)x << 32 | (u32)~i;
    };
    if (most >= least) {
      if constexpr (VECTORS > 0) {       // few threads have more than one: a mask, then the scores once more from the cache
        u32 mask = 0;
#pragma unroll
        for (u32 y = 0; y < VN; ++y)
#pragma unroll
          for (u32 z = 0; z < 4; ++z) mask |= mine(y, z) >= least ? 1u << (4 * y + z) : 0u;
        for (; mask; mask &= mask - 1) {
          const u32 at = __ffs(mask) - 1, i = 4 * (tid + at / 4 * THREADS) + at % 4;
          if (i >= a.first && i < end) candidate(scores[i], i);
        }
      } else {
        for (u32 i = tid; i < n; i += THREADS) {
          const u32 x = n <= held ? s_keys[i] : scores[a.first + i];
          if (x >= least) candidate(x, a.first + i);
        }
      }
    }
    __syncthreads();
    const u32 c = s_n;
    if (c <= PICK_CAP) {
      for (u32 i = tid; i < c; i += THREADS) {
        const u64 x = s_key[i];
        u32 before = 0;
#pragma unroll 4
        for (u32 y = 0; y < c; ++y) before += s_key[y] > x;
        if constexpr (VECTORS > 0) { if (before < m) atomicOr(&s_bits[~(u32)x / 32], 1u << (~(u32)x % 32)); }
        else taken[i] = before < m;
      }
      __syncthreads();
      if constexpr (VECTORS > 0) {       // in order: a word of 32 blocks per thread
        static_assert(VECTORS <= 8, "a bit for every block");
        u32 word = s_bits[tid], incl = __popc(word);
#pragma unroll
        for (u32 o = 1; o < 32; o *= 2) { const u32 z = __shfl_up_sync(~0u, incl, o); if (tid % 32 >= o) incl += z; }
        if (tid % 32 == 31) s_count[tid / 32] = incl;
        __syncthreads();
        u32 at = a.first + incl - __popc(word);
        for (u32 y = 0; y < tid / 32; ++y) at += s_count[y];
        for (; word; word &= word - 1) out[at++] = (int32_t)(tid * 32 + __ffs(word) - 1);
      } else for (u32 i = tid; i < c; i += THREADS) {
        if (!taken[i]) continue;
        const u32 x = (u32)s_key[i];     // the larger, the lower the number
        u32 before = 0;
#pragma unroll 4
        for (u32 y = 0; y < c; ++y) before += taken[y] && (u32)s_key[y] > x;
        out[a.first + before] = (int32_t)~x;
      }
      return;
    }
  }
  __syncthreads();
  const u32 *const keys = VECTORS == 0 && n <= held ? s_keys : scores + a.first;
  const Kth kth = kth_largest<THREADS>([&](auto f) { for (u32 i = tid; i < n; i += THREADS) f(keys[i]); }, n, m);
  __syncthreads();
  // keys equal to the last one that is taken: the first `ties` of them. Both lists in one go where all of them are taken.
  if (kth.ties == ~0u) {
    deal<THREADS>(n, [&](u32 i) { return keys[i] >= kth.at ? 1u : 0u; }, [&](u32 i, u32, u32 at) { out[a.first + at] = (int32_t)(a.first + i); });
    return;
  }
  __shared__ u32 s_border;                               // number of the last tie that is taken
  deal<THREADS>(n, [&](u32 i) { return keys[i] == kth.at ? 1u : 0u; }, [&](u32 i, u32, u32 at) { if (at == kth.ties - 1) s_border = i; });
  __syncthreads();
  const u32 border = s_border;
  deal<THREADS>(n, [&](u32 i) { return keys[i] > kth.at || (keys[i] == kth.at && i <= border) ? 1u : 0u; },
                [&](u32 i, u32, u32 at) { out[a.first + at] = (int32_t)(a.first + i); });
}

// Short rows: a warp per token and KV head, KEYS scores in a row per lane; the m-th largest is found by halving the range it lies in.
template <u32 KEYS>
__global__ void __launch_bounds__(128) k_pick_short(SelectArgs a, u32 rows) {
  const u32 lane = threadIdx.x & 31, row = blockIdx.x * 4 + threadIdx.x / 32, H = a.n_kv_heads, t = a.slab_begin + row / H;
  const bool any = row < rows;
  Where w{~0u, 0, false};
  if (any) w = find_token<true>(a.b, t, a.err);
  asm volatile("griddepcontrol.wait;" ::: "memory");     // the scores; the batch's arrays are older than the kernel before this one
  if (!any || w.seq >= a.b.n_seqs) return;               // behind the last sequence
  int32_t *const out = a.out + ((u64)a.slab_begin * H + row) * a.n_blocks;
  const u32 own = w.index / BT;
  if (!w.ok || own < a.n_blocks) {                       // all there are
    for (u32 i = lane; i < a.n_blocks; i += 32) out[i] = w.ok && i <= own ? (int32_t)i : -1;
    return;
  }
  const u32 end = own + 1 - a.last, m = a.n_blocks - a.first - a.last;
  for (u32 i = lane; i < a.first + a.last; i += 32) out[i < a.first ? i : i + m] = i < a.first ? (int32_t)i : (int32_t)(end + i - a.first);
  if (!m) return;
  const u32 *const scores = a.scores + (u64)row * a.scores_stride;
  u32 x[KEYS], valid = 0, lo = ~0u, hi = 0;
#pragma unroll
  for (u32 y = 0; y < KEYS; y += 4) {
    const u32 i = lane * KEYS + y;
    const uint4 v = i < end ? *(const uint4 *)(scores + i) : make_uint4(0, 0, 0, 0);
    x[y] = v.x; x[y + 1] = v.y; x[y + 2] = v.z; x[y + 3] = v.w;
  }
#pragma unroll
  for (u32 y = 0; y < KEYS; ++y) {
    const u32 i = lane * KEYS + y;
    if (i >= a.first && i < end) { valid |= 1u << y; lo = min(lo, x[y]); hi = max(hi, x[y]); }
  }
  lo = __reduce_min_sync(~0u, lo); hi = __reduce_max_sync(~0u, hi);
  auto at_least = [&](u32 least) {                       // a bit for each
    u32 mask = 0;
#pragma unroll
    for (u32 y = 0; y < KEYS; ++y) mask |= x[y] >= least ? 1u << y : 0u;
    return mask & valid;
  };
  // lo: a score that m or more reach; hi: the largest that may be it
  u32 mask = valid, c = end - a.first;
  while (lo < hi && c != m) {
    const u32 mid = lo + (hi - lo) / 2 + 1, some = at_least(mid), n = __reduce_add_sync(~0u, __popc(some));
    if (n >= m) { lo = mid; mask = some; c = n; } else hi = mid - 1;
  }
  auto before = [&](u32 n) {                             // sum over the lanes in front
    u32 incl = n;
#pragma unroll
    for (u32 o = 1; o < 32; o *= 2) { const u32 z = __shfl_up_sync(~0u, incl, o); if (lane >= o) incl += z; }
    return incl - n;
  };
  if (c != m) {                          // more scores are lo than are taken: the first of them
    u32 ties = 0;
#pragma unroll
    for (u32 y = 0; y < KEYS; ++y) ties |= x[y] == lo ? 1u << y : 0u;
    ties &= valid;
    mask &= ~ties;
    const u32 take = m - __reduce_add_sync(~0u, __popc(mask));
    for (u32 at = before(__popc(ties)); ties && at < take; ++at, ties &= ties - 1) mask |= ties & (0u - ties);
  }
  for (u32 at = a.first + before(__popc(mask)); mask; mask &= mask - 1) out[at++] = (int32_t)(lane * KEYS + __ffs(mask) - 1);
}

// Scores that are in hand together: about as many as L2 holds (126 MB), and parts of a long batch alike, since a short one fills the GPU as
// badly as a small batch. 32 chunks of 64 to 5000 tokens on 20,000 to 258,000, 8 KV heads, against all scores at once (up to 2.6 GB of them): parts of
// up to 16 MB take 1.40 times as long on average, 32 MB 1.15, 64 MB 1.03, 96 MB 1.02, 128 MB 1.004 (at most 1.14), 192 MB 1.01, 256 MB 0.995. 600 tokens on
// 130,500, 160 MB of scores: 243 us as 155 + 5 MB, 209 in two halves.
constexpr u64 SLAB_BYTES = 128ull << 20;
SelectPlan plan_select(const SelectArgs &a, int sm_count) {
  SelectPlan p{};
  p.sms = sm_count;
  p.slab = a.b.n_tokens;
  if (a.b.max_blocks <= a.n_blocks) return p;            // every list has all there are: no scores
  p.scores_stride = ((u64)a.b.max_blocks + 7) / 8 * 8;
  const u64 token = p.scores_stride * a.n_kv_heads * 4;
  const u32 most = (u32)std::min<u64>(a.b.n_tokens, std::max<u64>(1, SLAB_BYTES / token)), parts = (a.b.n_tokens + most - 1) / most;
  p.slab = std::min(most, ((a.b.n_tokens + parts - 1) / parts + 31) / 32 * 32);          // equal parts, of whole tiles of tokens
  p.scratch_bytes = p.slab * token;
  return p;
}

template <class T, u32 G, u32 M>
static cudaError_t score_blocks(const SelectArgs &a, dim3 grid, u32 shares, u32 which, cudaStream_t s, u64 *allowed) {
  const cudaError_t r = allow_smem(k_score_blocks<T, G, M>, which + 24, ScoreRing<G>::SMEM, allowed + 1);
  if (r != cudaSuccess) return r;
  k_score_blocks<T, G, M><<<grid, 256, ScoreRing<G>::SMEM, s>>>(a, shares);
  return cudaGetLastError();
}
template <class T>
static cudaError_t score_blocks(const SelectArgs &a, dim3 grid, u32 shares, bool wide, cudaStream_t s, u64 *allowed) {
  constexpr u32 F = __is_same(T, __half) * 8;
  if (wide && a.k.width <= 64) return score_blocks<T, 2, 2>(a, grid, shares, F + 0, s, allowed);
  if (wide) return score_blocks<T, 4, 2>(a, grid, shares, F + 1, s, allowed);
  if (a.k.width <= 64) return score_blocks<T, 2, 1>(a, grid, shares, F + 2, s, allowed);
  if (a.k.width <= 128) return score_blocks<T, 4, 1>(a, grid, shares, F + 3, s, allowed);
  return score_blocks<T, 8, 1>(a, grid, shares, F + 4, s, allowed);
}
template <class Kernel>
static cudaError_t launch_pick(Kernel kern, const SelectArgs &a, u32 ctas, u32 threads, u32 smem, u32 arg, bool scored, cudaStream_t s) {
  cudaLaunchConfig_t c{};
  c.gridDim = dim3(ctas); c.blockDim = dim3(threads); c.dynamicSmemBytes = smem; c.stream = s;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  c.attrs = &at; c.numAttrs = scored;    // behind a kernel of this call only: the batch's arrays may be of the kernel before that
  return cudaLaunchKernelEx(&c, kern, a, arg);
}
template <u32 THREADS, u32 VECTORS>
static cudaError_t pick_blocks(const SelectArgs &a, u32 rows, u32 held, bool scored, cudaStream_t s) {
  return launch_pick(k_pick_blocks<THREADS, VECTORS>, a, rows, THREADS, held * 4, held, scored, s);
}
static cudaError_t pick_blocks(const SelectArgs &a, u32 rows, bool scored, cudaStream_t s, u64 *allowed) {
  if (a.b.max_blocks <= 512) return launch_pick(k_pick_short<16>, a, (rows + 3) / 4, 128, 0, rows, scored, s);
  if (a.b.max_blocks <= 1024) return launch_pick(k_pick_short<32>, a, (rows + 3) / 4, 128, 0, rows, scored, s);
  if (a.b.max_blocks <= 2048) return pick_blocks<256, 2>(a, rows, 0, scored, s);
  if (a.b.max_blocks <= 4096) return pick_blocks<256, 4>(a, rows, 0, scored, s);
  if (a.b.max_blocks <= 8192) return pick_blocks<256, 8>(a, rows, 0, scored, s);
  if (a.b.max_blocks <= 16384) return pick_blocks<512, 8>(a, rows, 0, scored, s);
  if (a.b.max_blocks <= 32768) return pick_blocks<1024, 8>(a, rows, 0, scored, s);
  const cudaError_t r = allow_smem(k_pick_blocks<1024, 0>, 0, 180 * 1024, allowed);
  if (r != cudaSuccess) return r;
  return pick_blocks<1024, 0>(a, rows, std::min(a.b.max_blocks, 45u * 1024), scored, s);         // scores in shared memory
}
cudaError_t launch_select(SelectArgs a, const SelectPlan &p, cudaStream_t s, u64 *allowed, u32 *launches) {
  a.scores_stride = p.scores_stride;
  for (u32 t = 0; t < a.b.n_tokens; t += p.slab) {
    a.slab_begin = t; a.slab_end = std::min(a.b.n_tokens, t + p.slab);
    const u32 n = a.slab_end - t;
    // tiles of 32 tokens where the sequences bring as many on average: half the codes are read
    const bool wide = a.k.width <= 128 && n / a.b.n_seqs >= 24;
    const u32 rows_of = wide ? 32 : 16, tiles = (u32)(((u64)n + (rows_of - 1ull) * std::min(a.b.n_seqs, n)) / rows_of);
    if (a.b.max_blocks > a.n_blocks) {
      const u32 shares = std::max(1u, std::min((a.b.max_blocks + 63) / 64, 2 * p.sms / std::max(1u, tiles * a.n_kv_heads)));
      const dim3 grid(tiles, a.n_kv_heads, shares);
      const cudaError_t r = a.fp16 ? score_blocks<__half>(a, grid, shares, wide, s, allowed) : score_blocks<__nv_bfloat16>(a, grid, shares, wide, s, allowed);
      ++*launches;
      if (r != cudaSuccess) return r;
    }
    const cudaError_t r = pick_blocks(a, n * a.n_kv_heads, a.b.max_blocks > a.n_blocks, s, allowed);
    ++*launches;
    if (r != cudaSuccess) return r;
  }
  return cudaSuccess;
}

// ======================================================================================================
// Attention over listed blocks: softmax(scale q k^T) v of one token's group of query heads over the keys up to its own in the blocks
// its list names. A unit is a token and KV head (and 8 or 16 query heads); its blocks are dealt out to the four warps of a CTA, or
// of a cluster of them, each with a ring of loads of its own, and joined like the parts of a longer sequence.
// The queries are the narrow side of the products, 8 columns: S^T = K Q^T has the block's 16 keys as rows, O^T = V^T P^T 16 channels. That
// takes half the matrix instructions that 16 rows of queries would, where groups are of 8 heads and less, and a quarter for 4 and less.
// Measured in a captured graph, 8 KV heads of 128, bf16: one token, lists of 64, groups of 4 6.6 us (launch, three dependent loads before the
// first block, join through the cluster); 32 tokens, lists of 256, groups of 12 (538 MB) 90 us, 92 % of the measured copy bandwidth.
// ======================================================================================================
constexpr u32 LIST_WARPS = 4, LIST_THREADS = LIST_WARPS * 32;
template <u32 D, u32 PARTS = 3 /* of 8 KB of a warp's ring */> struct ListShape {
  static constexpr u32 BLOCK = BT * D * 2, STAGES = D == 64 ? 2 * PARTS : PARTS, RING = STAGES * 2 * BLOCK, SMEM = LIST_WARPS * RING + 1024, LD = D + 4;
};
__device__ __forceinline__ u32 transposed(u32 x) {       // an 8 x 8 matrix of 16-bit numbers, two per lane
  u32 y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// The blocks at list places part, part + parts, ... below n for the columns of a unit, into o, m, l (see k_attend_blocks). `it`: stages used
// so far. A lane has
// columns n * 8 + 2 (lane % 4) and the next, keys / channels lane / 4 and 8 further. DOUBLE: columns 4 to 7 are those 0 to 3 once
// more and take the second numbers of the powers.
template <class T, u32 D, u32 NT, bool DOUBLE, bool ANY, class S = ListShape<D>>
__device__ __forceinline__ bool list_keys(const AttendListArgs &x, const KvMaps &maps, const u32 *table, const int32_t *list, u32 n, u32 index, u32 h,
                                          const u16 *const (&q)[NT], u32 part, u32 parts, u32 ring, u32 bar0, u32 *s_block, u32 &it,
                                          float (&o)[D / 16][NT][4], float (&m)[NT][2], float (&l)[NT][2]) {
  const AttendArgs &a = x.a;
  const u32 lane = threadIdx.x & 31, own = index / BT;
  const u32 n_mine = part < n ? (n - part + parts - 1) / parts : 0;
  u32 held_slot = 0, held_block = 0;
  auto load = [&](u32 i) {
    if (i % 32 == 0) {
      held_block = i + lane < n_mine ? (u32)list[part + (i + lane) * parts] : ~0u;
      held_slot = ~0u;
      if (held_block <= own) {
        held_slot = table[held_block];
        if (held_slot >= a.p.n_slots && held_slot - a.p.n_slots >= a.p.n_tail) kv_err(a.err, KVERR_RANGE);
      }
    }
    const u32 slot = __shfl_sync(~0u, held_slot, i % 32), block = __shfl_sync(~0u, held_block, i % 32);
    const u32 st = (it + i) % S::STAGES, dst = ring + st * 2 * S::BLOCK;
    if (lane == 0) s_block[st] = block;
    if (ANY) {
      copy_block<D>(a, a.p.k, slot, h, dst);
      copy_block<D>(a, a.p.v, slot, h, dst + S::BLOCK);
    } else if (lane == 0) {
      const u32 bar = bar0 + st * 8;
      bar_expect(bar, 2 * S::BLOCK);
      load_block(a, maps, dst, bar, slot, 2 * a.layer, h, D / 64);
      load_block(a, maps, dst + S::BLOCK, bar, slot, 2 * a.layer + 1, h, D / 64);
    }
  };
  if (ANY) {
    const u32 c = (a.p.head_dim + 7) / 8;
    if (c < D / 8)
      for (u32 i = lane; i < S::STAGES * 2 * BT * (D / 8 - c); i += 32) {
        const u32 r = i / (D / 8 - c);
        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(ring + r / BT * S::BLOCK + block_off<D>(r % BT, c + i % (D / 8 - c))), "r"(0) : "memory");
      }
  }
#pragma unroll 1
  for (u32 i = 0; i < S::STAGES; ++i) {
    if (i < n_mine) load(i);
    if (ANY) asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // queries: column lane / 4 of every eight, the second operand
  u32 qf[NT][D / 16][2];
#pragma unroll
  for (u32 c = 0; c < NT; ++c) {
    const u16 *const src = q[c] + lane % 4 * 2;
    const bool even = ((uintptr_t)src & 3) == 0;
#pragma unroll
    for (u32 k = 0; k < D / 16; ++k)
#pragma unroll
      for (u32 z = 0; z < 2; ++z) {
        const u16 *const p = src + k * 16 + z * 8;
        if (ANY) {
          const u32 d = lane % 4 * 2 + k * 16 + z * 8;
          qf[c][k][z] = (d < a.p.head_dim ? (u32)p[0] : 0u) | (d + 1 < a.p.head_dim ? (u32)p[1] << 16 : 0u);
        } else {
          qf[c][k][z] = even ? *(const u32 *)p : (u32)p[0] | (u32)p[1] << 16;
        }
      }
  }
#pragma unroll
  for (u32 c = 0; c < NT; ++c) {
    m[c][0] = m[c][1] = -INFINITY; l[c][0] = l[c][1] = 0.0f;
#pragma unroll
    for (u32 k = 0; k < D / 16; ++k)
#pragma unroll
      for (u32 y = 0; y < 4; ++y) o[k][c][y] = 0.0f;
  }
  bool ok = true;
  for (u32 i = 0; i < n_mine; ++i) {
    const u32 st = (it + i) % S::STAGES, kb = ring + st * 2 * S::BLOCK, vb = kb + S::BLOCK;
    if (ANY) {
      asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 1) : "memory");
      __syncwarp();
    } else if (!(ok = __all_sync(~0u, bar_wait(bar0 + st * 8, (it + i) / S::STAGES & 1)))) break;
    const u32 block = s_block[st];
    float s[NT][4];
#pragma unroll
    for (u32 c = 0; c < NT; ++c)
#pragma unroll
      for (u32 y = 0; y < 4; ++y) s[c][y] = 0.0f;
#pragma unroll
    for (u32 k = 0; k < D / 16; ++k) {
      u32 f[4];
      ldm4(f, kb + block_off<D>(lane % 16, 2 * k + lane / 16));
#pragma unroll
      for (u32 c = 0; c < NT; ++c) mma16816<T>(s[c], f, qf[c][k][0], qf[c][k][1]);
    }
#pragma unroll
    for (u32 c = 0; c < NT; ++c)
#pragma unroll
      for (u32 y = 0; y < 4; ++y) s[c][y] *= a.scale_log2;
    if (block >= own) {                  // the token's own block, or no block of its
      const u32 seen = block == own ? index % BT + 1 : 0;
#pragma unroll
      for (u32 c = 0; c < NT; ++c)
#pragma unroll
        for (u32 y = 0; y < 4; ++y) if (lane / 4 + 8 * (y / 2) >= seen) s[c][y] = -INFINITY;
      // values behind the token: weight 0 must not meet an Inf or a NaN
      const u32 r = lane / 2;
      if (r >= seen)
#pragma unroll
        for (u32 c = 0; c < D / 16; ++c)
          asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vb + block_off<D>(r, (lane % 2) * (D / 16) + c)), "r"(0) : "memory");
      if (!ANY) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // a load writes here next
      __syncwarp();
    }
    float top[NT][2];
    bool move = false;
#pragma unroll
    for (u32 c = 0; c < NT; ++c)
#pragma unroll
      for (u32 y = 0; y < 2; ++y) {
        top[c][y] = fmaxf(s[c][y], s[c][y + 2]);
        if (Elem<T>::LOW > -INFINITY) {  // the largest may be too small, too: all of the column's keys have to be looked at
#pragma unroll
          for (u32 z = 4; z < 32; z *= 2) top[c][y] = fmaxf(top[c][y], __shfl_xor_sync(~0u, top[c][y], z));
        }
        move |= must_move<T>(m[c][y], top[c][y]);
      }
    if (__any_sync(~0u, move)) {
#pragma unroll
      for (u32 c = 0; c < NT; ++c)
#pragma unroll
        for (u32 y = 0; y < 2; ++y) {
          float all = l[c][y];
#pragma unroll
          for (u32 z = 4; z < 32; z *= 2) {
            if (!(Elem<T>::LOW > -INFINITY)) top[c][y] = fmaxf(top[c][y], __shfl_xor_sync(~0u, top[c][y], z));
            all = fmaxf(all, __shfl_xor_sync(~0u, all, z));
          }
          const float f = raise_or_lower<T>(m[c][y], top[c][y], all);
          l[c][y] *= f;
#pragma unroll
          for (u32 k = 0; k < D / 16; ++k) { o[k][c][y] *= f; o[k][c][y + 2] *= f; }
        }
    }
    // powers, as the sum of two numbers of the element type (see k_attend_split)
    u32 p[NT][2], rest[NT][2];
#pragma unroll
    for (u32 c = 0; c < NT; ++c) {
      const float ref[2] = {m[c][0] == -INFINITY ? 0.0f : m[c][0], m[c][1] == -INFINITY ? 0.0f : m[c][1]};
#pragma unroll
      for (u32 y = 0; y < 4; ++y) { s[c][y] = ex2(s[c][y] - ref[y & 1]); l[c][y & 1] += s[c][y]; }
#pragma unroll
      for (u32 z = 0; z < 2; ++z) {
        const u32 first = Elem<T>::down(s[c][2 * z], s[c][2 * z + 1]);
        const float2 w = Elem<T>::up(first);
        const u32 second = Elem<T>::down(s[c][2 * z] - w.x, s[c][2 * z + 1] - w.y);
        p[c][z] = transposed(DOUBLE && lane % 4 >= 2 ? second : first);
        rest[c][z] = DOUBLE ? 0 : transposed(second);
      }
    }
#pragma unroll
    for (u32 k = 0; k < D / 16; k += 2) {
      u32 f[2][4];
#pragma unroll
      for (u32 y = 0; y < 2; ++y) ldm4t(f[y], vb + block_off<D>((lane / 16) * 8 + lane % 8, 2 * (k + y) + lane / 8 % 2));
#pragma unroll
      for (u32 y = 0; y < 2; ++y)
#pragma unroll
        for (u32 c = 0; c < NT; ++c) mma16816<T>(o[k + y][c], f[y], p[c][0], p[c][1]);
      if (!DOUBLE)
#pragma unroll
        for (u32 y = 0; y < 2; ++y)
#pragma unroll
          for (u32 c = 0; c < NT; ++c) mma16816<T>(o[k + y][c], f[y], rest[c][0], rest[c][1]);
    }
    __syncwarp();                        // the stage is read: refill it
    if (i + S::STAGES < n_mine) load(i + S::STAGES);
    if (ANY) asm volatile("cp.async.commit_group;" ::: "memory");
  }
  it += n_mine;
  return ok;
}

template <class T, u32 D, u32 NT, bool DOUBLE, u32 CLUSTER, bool ANY>
__global__ void __launch_bounds__(LIST_THREADS, D > 128 ? 1 : 2)
k_attend_blocks(const __grid_constant__ AttendListArgs x, const __grid_constant__ KvMaps maps, u32 col_tiles) {
  typedef ListShape<D> S;
  constexpr u32 COLS = NT * 8, REAL = DOUBLE ? 4 : COLS;       // columns; those that are query heads
  extern __shared__ u8 smem_raw[];
  __shared__ __align__(8) u64 bars[LIST_WARPS * S::STAGES];
  __shared__ u32 s_block[LIST_WARPS][S::STAGES];
  __shared__ float s_ml[LIST_WARPS][COLS][2], s_part_ml[REAL][2];
  __shared__ u32 s_lost;
  const AttendArgs &a = x.a;
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = a.p.n_kv_heads;
  const u32 rank = blockIdx.x % CLUSTER, unit = blockIdx.x / CLUSTER, ct = unit % col_tiles, th = unit / col_tiles, t = th / H, h = th - t * H;
  const u32 bar0 = smem_addr(bars) + warp * S::STAGES * 8;
  if (lane == 0) {
    for (u32 i = 0; i < S::STAGES; ++i) bar_init(bar0 + i * 8, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (!ANY && tid < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(tid ? &maps.tail : &maps.pool) : "memory");
  const Where w = find_token<false>(a.b, t, a.err);
  if (w.seq >= a.b.n_seqs) return;       // behind the last sequence: the whole cluster
  __syncwarp();
  const u32 ring0 = (smem_addr(smem_raw) + 1023) & ~1023u, ring = ring0 + warp * S::RING;
  const int32_t *const list = x.blocks + (u64)th * x.n_blocks;
  u32 n = 0;                             // places up to the last that names a block with keys to see
  if (w.ok) for (u32 i = 0; i < x.n_blocks; i += 32) {
    const u32 have = __ballot_sync(~0u, i + lane < x.n_blocks && (u32)list[i + lane] <= w.index / BT);
    if (have) n = i + 32 - __clz(have);
  }
  const u32 rows = min(a.group - ct * REAL, REAL);             // query heads of this unit
  const u16 *q[NT];
#pragma unroll
  for (u32 c = 0; c < NT; ++c) {
    const u32 r = min((c * 8 + lane / 4) % REAL, rows - 1);    // columns behind the last repeat it
    q[c] = (const u16 *)a.q + (u64)t * a.q_ts + (u64)(h * a.group + ct * REAL + r) * a.q_hs;
  }
  float o[D / 16][NT][4], m[NT][2], l[NT][2];
  u32 it = 0;
  const bool ok = list_keys<T, D, NT, DOUBLE, ANY>(x, maps, a.b.table + w.seq * a.b.table_stride, list, n, w.index, h, q, rank * LIST_WARPS + warp,
                                                   CLUSTER * LIST_WARPS, ring, bar0, s_block[warp], it, o, m, l);
  // each warp's sums into its ring, [column][channel]
  float *const so = (float *)(smem_raw + (ring - smem_addr(smem_raw)));
  static_assert(2 * COLS * S::LD * 4 <= S::RING, "the sums, and the CTA's part behind warp 0's, fit a ring");
#pragma unroll
  for (u32 c = 0; c < NT; ++c)
#pragma unroll
    for (u32 y = 0; y < 2; ++y) {
#pragma unroll
      for (u32 z = 4; z < 32; z *= 2) l[c][y] += __shfl_xor_sync(~0u, l[c][y], z);
      const u32 col = c * 8 + lane % 4 * 2 + y;
      if (lane < 4) { s_ml[warp][col][0] = m[c][y]; s_ml[warp][col][1] = l[c][y]; }
#pragma unroll
      for (u32 k = 0; k < D / 16; ++k) {
        so[col * S::LD + k * 16 + lane / 4] = o[k][c][y];
        so[col * S::LD + k * 16 + lane / 4 + 8] = o[k][c][y + 2];
      }
    }
  const bool lost = __syncthreads_or(!ok);
  float *const sums = (float *)(smem_raw + (ring0 - smem_addr(smem_raw))), *const mine = sums + COLS * S::LD;
  auto write = [&](u32 r, u32 c, float4 v, float mm, float ll) {         // four channels of a query head
    const float inv = ll > 0.0f ? 1.0f / ll : ll;
    const u32 hq = h * a.group + ct * REAL + r, d = ANY ? a.p.head_dim : D;
    u16 *const dst = (u16 *)a.out + (u64)t * a.o_ts + (u64)hq * a.o_hs + c;
    const u32 p0 = Elem<T>::down(v.x * inv, v.y * inv), p1 = Elem<T>::down(v.z * inv, v.w * inv);
    if (((uintptr_t)dst & 7) == 0 && c + 4 <= d) *(uint2 *)dst = make_uint2(p0, p1);
    else {
      if (c < d) dst[0] = (u16)p0;
      if (c + 1 < d) dst[1] = (u16)(p0 >> 16);
      if (c + 2 < d) dst[2] = (u16)p1;
      if (c + 3 < d) dst[3] = (u16)(p1 >> 16);
    }
    if (a.lse && c == 0) a.lse[(u64)t * a.n_q_heads + hq] = (mm + log2f(ll)) * 0.69314718055994531f;
  };
  for (u32 i = tid; i < REAL * D / 4; i += LIST_THREADS) {
    const u32 r = i / (D / 4), c = i % (D / 4) * 4;
    float mm = -INFINITY, ll = 0.0f;
#pragma unroll
    for (u32 y = 0; y < LIST_WARPS; ++y) mm = fmaxf(mm, s_ml[y][r][0]);
    const float ref = mm == -INFINITY ? 0.0f : mm;
    float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
    for (u32 y = 0; y < LIST_WARPS; ++y) {
      const float f = ex2(s_ml[y][r][0] - ref);
      ll += f * s_ml[y][r][1];
#pragma unroll
      for (u32 k = 0; k < (DOUBLE ? 2 : 1); ++k) {
        const float4 z = *(const float4 *)(sums + y * (S::RING / 4) + (r + 4 * k) * S::LD + c);
        v.x += f * z.x; v.y += f * z.y; v.z += f * z.z; v.w += f * z.w;
      }
    }
    if (CLUSTER == 1) {
      if (r < rows && !lost) write(r, c, v, mm, ll);
    } else {
      *(float4 *)(mine + r * S::LD + c) = v;
      if (c == 0) { s_part_ml[r][0] = mm; s_part_ml[r][1] = ll; }
    }
  }
  u32 any_lost = lost;
  if (CLUSTER > 1) {
    if (tid == 0) s_lost = lost;
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    auto there = [&](const void *p, u32 cta) {
      u32 r;
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr(p)), "r"(cta));
      return r;
    };
    for (u32 first = 0; first < REAL * D / 4; first += CLUSTER * LIST_THREADS) {
      const u32 at = first + rank * LIST_THREADS + tid;
      const bool here = at < REAL * D / 4;
      const u32 r = here ? at / (D / 4) : 0, c = here ? at % (D / 4) * 4 : 0;
      float mm[CLUSTER], ll[CLUSTER], top = -INFINITY, sum = 0.0f;
      float4 v = make_float4(0, 0, 0, 0), z[CLUSTER];
#pragma unroll
      for (u32 y = 0; y < CLUSTER; ++y) {
        u32 gone;
        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(mm[y]), "=f"(ll[y]) : "r"(there(&s_part_ml[r][0], y)) : "memory");
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(z[y].x), "=f"(z[y].y), "=f"(z[y].z), "=f"(z[y].w) : "r"(there(mine + r * S::LD + c, y)) : "memory");
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(gone) : "r"(there(&s_lost, y)) : "memory");
        any_lost |= gone;
        top = fmaxf(top, mm[y]);
      }
      const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
      for (u32 y = 0; y < CLUSTER; ++y) {
        const float f = ex2(mm[y] - ref);
        sum += f * ll[y];
        v.x += f * z[y].x; v.y += f * z[y].y; v.z += f * z[y].z; v.w += f * z[y].w;
      }
      if (here && r < rows && !any_lost) write(r, c, v, top, sum);
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");    // nobody reads here any more
  }
  if (any_lost) {
    if (tid == 0) kv_err(a.err, KVERR_WAIT);
    if (!ok && !ANY) for (u32 i = 0; i < S::STAGES; ++i) for (u32 y = 0; y < 2; ++y) bar_wait(bar0 + i * 8, y);     // copies in flight
  }
}

// Many units (chunks and prompts): a warp per unit, one after the other, without a word to the others; what a unit takes besides its blocks
// is hidden by the other warps of the SM.
// Bound by the chain of a block's own steps, so more warps do more than a longer ring: with 4 CTAs per SM and one stage (heads of 128; 64:
// two) 792 tokens, 8 KV heads, groups of 4, lists of 64 take 203 us (64: 150), with 3 CTAs and two stages 218 (178), with 2 and three 277
// (240). Two tiles of columns have more registers: groups of 12 with 3 CTAs 323 us, with 2 378, with 4 351.
template <u32 NT> constexpr u32 MANY_PARTS = NT == 1 ? 1 : 2;
template <u32 D, u32 NT> constexpr u32 MANY_CTAS = NT == 1 ? 4 : 3;
template <class T, u32 D, u32 NT, bool DOUBLE>
__global__ void __launch_bounds__(LIST_THREADS, MANY_CTAS<D, NT>)
k_attend_lists(const __grid_constant__ AttendListArgs x, const __grid_constant__ KvMaps maps, u32 col_tiles, u32 n_units) {
  typedef ListShape<D, MANY_PARTS<NT>> S;
  constexpr u32 COLS = NT * 8, REAL = DOUBLE ? 4 : COLS;
  extern __shared__ u8 smem_raw[];
  __shared__ __align__(8) u64 bars[LIST_WARPS * S::STAGES];
  __shared__ u32 s_block[LIST_WARPS][S::STAGES];
  const AttendArgs &a = x.a;
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = a.p.n_kv_heads;
  const u32 bar0 = smem_addr(bars) + warp * S::STAGES * 8, ring = ((smem_addr(smem_raw) + 1023) & ~1023u) + warp * S::RING;
  if (lane == 0) {
    for (u32 i = 0; i < S::STAGES; ++i) bar_init(bar0 + i * 8, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (tid < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(tid ? &maps.tail : &maps.pool) : "memory");
  __syncwarp();
  u32 it = 0;
  for (u32 unit = blockIdx.x * LIST_WARPS + warp; unit < n_units; unit += gridDim.x * LIST_WARPS) {
    const u32 ct = unit % col_tiles, th = unit / col_tiles, t = th / H, h = th - t * H;
    const Where w = find_token<true>(a.b, t, a.err);
    if (w.seq >= a.b.n_seqs) continue;   // behind the last sequence
    const int32_t *const list = x.blocks + (u64)th * x.n_blocks;
    u32 n = 0;                           // places up to the last that names a block with keys to see
    if (w.ok) for (u32 i = 0; i < x.n_blocks; i += 32) {
      const u32 have = __ballot_sync(~0u, i + lane < x.n_blocks && (u32)list[i + lane] <= w.index / BT);
      if (have) n = i + 32 - __clz(have);
    }
    const u32 rows = min(a.group - ct * REAL, REAL);
    const u16 *q[NT];
#pragma unroll
    for (u32 c = 0; c < NT; ++c) {
      const u32 r = min((c * 8 + lane / 4) % REAL, rows - 1);
      q[c] = (const u16 *)a.q + (u64)t * a.q_ts + (u64)(h * a.group + ct * REAL + r) * a.q_hs;
    }
    float o[D / 16][NT][4], m[NT][2], l[NT][2];
    if (!list_keys<T, D, NT, DOUBLE, false, S>(x, maps, a.b.table + w.seq * a.b.table_stride, list, n, w.index, h, q, 0, 1, ring, bar0, s_block[warp], it, o, m, l)) {
      if (lane == 0) kv_err(a.err, KVERR_WAIT);          // let the copies in flight land, for a while, before the warp ends
      for (u32 i = 0; i < S::STAGES; ++i) for (u32 y = 0; y < 2; ++y) bar_wait(bar0 + i * 8, y);
      return;
    }
    // results from the registers: pairs of channels of a query head, put together by turning each 8 x 8 part over
#pragma unroll
    for (u32 c = 0; c < NT; ++c) {
      float inv[2];
#pragma unroll
      for (u32 y = 0; y < 2; ++y) {
#pragma unroll
        for (u32 z = 4; z < 32; z *= 2) l[c][y] += __shfl_xor_sync(~0u, l[c][y], z);
        inv[y] = l[c][y] > 0.0f ? 1.0f / l[c][y] : l[c][y];
        const u32 r = c * 8 + lane % 4 * 2 + y;
        if (a.lse && lane < 4 && r < rows) a.lse[(u64)t * a.n_q_heads + h * a.group + ct * REAL + r] = (m[c][y] + log2f(l[c][y])) * 0.69314718055994531f;
      }
      const u32 r = c * 8 + lane / 4;
      u16 *const dst = (u16 *)a.out + (u64)t * a.o_ts + (u64)(h * a.group + ct * REAL + min(r, rows - 1)) * a.o_hs + lane % 4 * 2;
      const bool even = ((uintptr_t)dst & 3) == 0;
#pragma unroll
      for (u32 k = 0; k < D / 16; ++k)
#pragma unroll
        for (u32 z = 0; z < 2; ++z) {
          float v0 = o[k][c][2 * z], v1 = o[k][c][2 * z + 1];
          if (DOUBLE) { v0 += __shfl_xor_sync(~0u, v0, 2); v1 += __shfl_xor_sync(~0u, v1, 2); }
          const u32 e = transposed(Elem<T>::down(v0 * inv[0], v1 * inv[1]));
          u16 *const p = dst + k * 16 + z * 8;
          if (r >= rows) continue;
          if (even) *(u32 *)p = e; else { p[0] = (u16)e; p[1] = (u16)(e >> 16); }
        }
    }
    __syncwarp();
  }
}

template <class T, u32 D, u32 NT, bool DOUBLE, u32 CLUSTER, bool ANY>
static cudaError_t launch_list(const AttendListArgs &x, const KvMaps &m, u32 units, u32 col_tiles, cudaStream_t s, u64 *allowed) {
  constexpr u32 size = CLUSTER == 8 ? 3 : CLUSTER == 4 ? 2 : CLUSTER == 2 ? 1 : 0, kind = DOUBLE ? 0 : NT;
  constexpr u32 which = 7 + (ANY ? (D == 256 ? 2 : D == 128) + (CLUSTER > 1 ? 3 : 0) : 6 + (D == 128 ? 12 : 0) + size * 3 + kind);      // 7 .. 36
  auto const kern = k_attend_blocks<T, D, NT, DOUBLE, CLUSTER, ANY>;
  cudaError_t r = allow_smem(kern, which, ListShape<D>::SMEM, allowed + (__is_same(T, __half) ? 2 : 0));
  if (r != cudaSuccess) return r;
  cudaLaunchConfig_t c{};
  c.gridDim = dim3(units * CLUSTER); c.blockDim = dim3(LIST_THREADS); c.dynamicSmemBytes = ListShape<D>::SMEM; c.stream = s;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = CLUSTER; at.val.clusterDim.y = at.val.clusterDim.z = 1;
  c.attrs = &at; c.numAttrs = CLUSTER > 1;
  return cudaLaunchKernelEx(&c, kern, x, m, col_tiles);
}
template <class T, u32 D, u32 NT, bool DOUBLE>
static cudaError_t launch_list(const AttendListArgs &x, const KvMaps &m, u32 units, u32 col_tiles, u32 cluster, u32 sms, cudaStream_t s, u64 *allowed) {
  switch (cluster) {
    case 0: {                            // a warp per unit
      constexpr u32 SMEM = ListShape<D, MANY_PARTS<NT>>::SMEM;
      const cudaError_t r = allow_smem(k_attend_lists<T, D, NT, DOUBLE>, 12 + ((D == 128) * 2 + __is_same(T, __half)) * 3 + (DOUBLE ? 0 : NT), SMEM, allowed + 1);
      if (r != cudaSuccess) return r;
      k_attend_lists<T, D, NT, DOUBLE><<<std::min((units + LIST_WARPS - 1) / LIST_WARPS, MANY_CTAS<D, NT> * sms), LIST_THREADS, SMEM, s>>>(x, m, col_tiles, units);
      return cudaGetLastError();
    }
    case 1: return launch_list<T, D, NT, DOUBLE, 1, false>(x, m, units, col_tiles, s, allowed);
    case 2: return launch_list<T, D, NT, DOUBLE, 2, false>(x, m, units, col_tiles, s, allowed);
    case 4: return launch_list<T, D, NT, DOUBLE, 4, false>(x, m, units, col_tiles, s, allowed);
    default: return launch_list<T, D, NT, DOUBLE, 8, false>(x, m, units, col_tiles, s, allowed);
  }
}
template <class T>
static cudaError_t launch_list(const AttendListArgs &x, const KvMaps &m, u32 sms, cudaStream_t s, u64 *allowed) {
  const u32 g = x.a.group, d = x.a.p.head_dim, th = x.a.b.n_tokens * x.a.p.n_kv_heads;
  if (d != 64 && d != 128) {             // heads of every other size: 16 columns
    const u32 tiles = (g + 15) / 16;
    const u64 units = (u64)th * tiles;
    const bool few = units * 8 <= (d > 128 ? 1ull : 2ull) * sms && x.n_blocks >= 32;
    if (d < 64) return few ? launch_list<T, 64, 2, false, 8, true>(x, m, units, tiles, s, allowed) : launch_list<T, 64, 2, false, 1, true>(x, m, units, tiles, s, allowed);
    if (d < 128) return few ? launch_list<T, 128, 2, false, 8, true>(x, m, units, tiles, s, allowed) : launch_list<T, 128, 2, false, 1, true>(x, m, units, tiles, s, allowed);
    return few ? launch_list<T, 256, 2, false, 8, true>(x, m, units, tiles, s, allowed) : launch_list<T, 256, 2, false, 1, true>(x, m, units, tiles, s, allowed);
  }
  const u32 cols = g <= 4 ? 4 : g <= 8 ? 8 : 16, tiles = (g + cols - 1) / cols;
  const u64 units = (u64)th * tiles;
  // a warp per unit where there is one for each that runs at once, else CTAs or clusters of them per unit
  u32 cluster = units >= 8ull * sms ? 0 : 1;
  while (cluster && cluster < 8 && units * cluster * 2 <= 2ull * sms && x.n_blocks >= 16 * cluster) cluster *= 2;
  if (d == 64) return cols == 4 ? launch_list<T, 64, 1, true>(x, m, units, tiles, cluster, sms, s, allowed)
                   : cols == 8 ? launch_list<T, 64, 1, false>(x, m, units, tiles, cluster, sms, s, allowed)
                               : launch_list<T, 64, 2, false>(x, m, units, tiles, cluster, sms, s, allowed);
  return cols == 4 ? launch_list<T, 128, 1, true>(x, m, units, tiles, cluster, sms, s, allowed)
       : cols == 8 ? launch_list<T, 128, 1, false>(x, m, units, tiles, cluster, sms, s, allowed)
                   : launch_list<T, 128, 2, false>(x, m, units, tiles, cluster, sms, s, allowed);
}
cudaError_t launch_attend_blocks(const AttendListArgs &x, const KvMaps &m, int sm_count, cudaStream_t s, u64 *allowed, u32 *launches) {
  ++*launches;
  return x.a.fp16 ? launch_list<__half>(x, m, sm_count, s, allowed) : launch_list<__nv_bfloat16>(x, m, sm_count, s, allowed);
}

// ======================================================================================================
// Attention weight of blocks: w_b = keep w_b + sum over the new tokens, query heads and keys j of block b of exp(scale q.k_j - lse), with the
// logarithms lse of the sums of exponentials that the attention left. K is read, V is not.
// ======================================================================================================
// Powers relative to a row's lse: both the scale and lse / ln 2 are taken as two 32-bit numbers, since an error of 2^-24 of either
// would be one of some 10^-6 of the power where scores are large.
struct Lse { float high, low; };
__device__ __forceinline__ Lse lse_log2(float lse) {
  constexpr float L1 = 1.44269502f, L2 = 1.92596300e-8f;       // 1 / ln 2
  Lse r;
  r.high = lse * L1;
  r.low = fmaf(lse, L1, -r.high) + lse * L2;
  if (!(fabsf(lse) <= 1e30f)) { r.high = lse == -INFINITY ? INFINITY : lse; r.low = 0.0f; }     // a row that sees no key: no weight
  return r;
}

// First block that any new token of a sequence sees: those in front of the window are not read and need no valid slot.
__device__ __forceinline__ u32 first_seen(const AttendArgs &a, const Seq &q) {
  const long long lo = a.window ? (long long)q.kv - q.n + 1 - (long long)a.window : 0;
  return lo > 0 ? (u32)(lo / BT) : 0u;
}

// 16 bytes from 8 elements at p, of which n_left exist.
__device__ __forceinline__ uint4 load8(const u16 *p, int n_left, bool vec) {
  if (n_left >= 8 && vec) return *(const uint4 *)p;
  u32 x[4] = {0, 0, 0, 0};
#pragma unroll
  for (int y = 0; y < 8; ++y) if (y < n_left) x[y / 2] |= (u32)p[y] << (y % 2 * 16);
  return make_uint4(x[0], x[1], x[2], x[3]);
}

// Few rows (a new token per sequence), heads of 64 and 128: bound by reading K once. A CTA of four warps takes a tile of up to 32 blocks of one
// sequence, each warp every fourth head of it, with a ring of TMA loads of its own (a block's keys of one head per stage). The block's 16
// keys are the rows of the matrix instruction, eight (token, head) rows the columns, which stay in registers for all blocks of a head.
// Lane i holds the sum of block i. Two CTAs per SM keep 192 KB of loads in flight. Measured in a captured graph, 8 KV heads of 128: 32 tokens on
// 2,000 to 130,000 each, groups of 12 (3.0 GB) 469 us, 99 % of the measured copy bandwidth; one token on 258,047 90 us (89 %), on 1000 4.6 us.
// (K straight into registers, the next block's while one is worked on, took 1370 us where this takes 469.)
constexpr u32 WEIGH_TILE = 32, WS_WARPS = 4, WS_THREADS = WS_WARPS * 32;
template <u32 D> struct WeighRing { static constexpr u32 BLOCK = BT * D * 2, STAGES = D == 64 ? 12 : 6, RING = STAGES * BLOCK, SMEM = WS_WARPS * RING + 1024; };
template <class T, u32 D, u32 NT>
__global__ void __launch_bounds__(WS_THREADS, 2) k_weigh_split(const __grid_constant__ WeighArgs x, const __grid_constant__ KvMaps maps, u32 n_tile) {
  typedef WeighRing<D> S;
  extern __shared__ u8 smem_raw[];
  __shared__ __align__(8) u64 bars[WS_WARPS * S::STAGES];
  __shared__ float s_sum[WS_WARPS][WEIGH_TILE];
  const AttendArgs &a = x.a;
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = a.p.n_kv_heads, g = a.group;
  const u32 tiles = (a.b.max_blocks + n_tile - 1) / n_tile, seq = blockIdx.x / tiles, b_tile = (blockIdx.x - seq * tiles) * n_tile;
  const Seq q = load_seq(a.b, seq, a.err);
  const u32 n_held = (q.kv + BT - 1) / BT, b0 = max(b_tile, first_seen(a, q)), b1 = min(b_tile + n_tile, n_held), nb = b1 > b0 && q.n ? b1 - b0 : 0;
  bool ok = true;
  if (nb) {
    const u32 bar0 = smem_addr(bars) + warp * S::STAGES * 8, ring = ((smem_addr(smem_raw) + 1023) & ~1023u) + warp * S::RING;
    u32 held = ~0u;                      // lane i: slot of block i
    if (lane < nb) {
      held = a.b.table[seq * a.b.table_stride + b0 + lane];
      if (held >= a.p.n_slots && held - a.p.n_slots >= a.p.n_tail) kv_err(a.err, KVERR_RANGE);
    }
    if (lane == 0) {
      for (u32 i = 0; i < S::STAGES; ++i) bar_init(bar0 + i * 8, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncwarp();
    const u32 rows = q.n * g, n_rounds = (rows + NT * 8 - 1) / (NT * 8), n_heads = warp < H ? (H - warp + WS_WARPS - 1) / WS_WARPS : 0, n_items = n_rounds * n_heads * nb;
    const int shift = (int)q.kv - (int)q.n;                      // index of the first new token
    u32 load_b = 0, load_h = warp, load_st = 0;                  // the next item to load
    auto load = [&]() {
      const u32 slot = __shfl_sync(~0u, held, load_b);
      if (lane == 0) {
        bar_expect(bar0 + load_st * 8, S::BLOCK);
        load_block(a, maps, ring + load_st * S::BLOCK, bar0 + load_st * 8, slot, 2 * a.layer, load_h, D / 64);
      }
      if (++load_st == S::STAGES) load_st = 0;
      if (++load_b == nb) { load_b = 0; load_h += WS_WARPS; if (load_h >= H) load_h = warp; }
    };
    for (u32 i = 0; i < min(S::STAGES, n_items); ++i) load();
    double acc = 0.0;                    // (a long prompt adds thousands of sums up: 32 bits would lose some 10^-5)
    u32 it = 0, st = 0, phase = 0;
    for (u32 r0 = 0; ok && r0 < rows; r0 += NT * 8)
      for (u32 h = warp; ok && h < H; h += WS_WARPS) {
        u32 qf[NT][D / 16][2];
        Lse L[NT][2];
        int lo[NT][2], hi[NT][2];        // keys that columns 2 (lane % 4) and the next see
#pragma unroll
        for (u32 c = 0; c < NT; ++c) {
          const u32 r = min(r0 + c * 8 + lane / 4, rows - 1), tok = r / g;
          const u16 *const src = (const u16 *)a.q + (u64)(q.t0 + tok) * a.q_ts + (u64)(h * g + r - tok * g) * a.q_hs + lane % 4 * 2;
          const bool even = ((uintptr_t)src & 3) == 0;
#pragma unroll
          for (u32 k = 0; k < D / 16; ++k)
#pragma unroll
            for (u32 z = 0; z < 2; ++z) {
              const u16 *const p = src + k * 16 + z * 8;
              qf[c][k][z] = even ? *(const u32 *)p : (u32)p[0] | (u32)p[1] << 16;
            }
#pragma unroll
          for (u32 z = 0; z < 2; ++z) {
            const u32 rr = r0 + c * 8 + lane % 4 * 2 + z, tk = min(rr, rows - 1) / g;
            L[c][z] = lse_log2(a.lse[(u64)(q.t0 + tk) * a.n_q_heads + h * g + min(rr, rows - 1) - tk * g]);
            hi[c][z] = rr >= rows ? 0 : a.full ? (int)q.kv : max(0, shift + (int)tk + 1);
            lo[c][z] = a.window ? hi[c][z] - (int)min(a.window, 0x7FFFFFFFu) : 0;
          }
        }
        for (u32 b = 0; b < nb; ++b, ++it) {
          if (!(ok = __all_sync(~0u, bar_wait(bar0 + st * 8, phase)))) break;
          const u32 kb = ring + st * S::BLOCK;
          float s[NT][4];
#pragma unroll
          for (u32 c = 0; c < NT; ++c)
#pragma unroll
            for (u32 y = 0; y < 4; ++y) s[c][y] = 0.0f;
#pragma unroll
          for (u32 k = 0; k < D / 16; ++k) {
            u32 f[4];
            ldm4(f, kb + block_off<D>(lane % 16, 2 * k + lane / 16));
#pragma unroll
            for (u32 c = 0; c < NT; ++c) mma16816<T>(s[c], f, qf[c][k][0], qf[c][k][1]);
          }
          __syncwarp();                  // the stage is read
          if (it + S::STAGES < n_items) load();
          if (++st == S::STAGES) { st = 0; phase ^= 1; }
          const int key0 = (int)((b0 + b) * BT + lane / 4);
          float sum = 0.0f;
#pragma unroll
          for (u32 c = 0; c < NT; ++c)
#pragma unroll
            for (u32 y = 0; y < 4; ++y) {
              const int key = key0 + (int)(y / 2) * 8;
              const float e = ex2(fmaf(s[c][y], a.scale_log2, -L[c][y & 1].high) + fmaf(s[c][y], x.scale_low, -L[c][y & 1].low));
              sum += key < hi[c][y & 1] && key >= lo[c][y & 1] ? e : 0.0f;
            }
          sum = sum_over_warp(sum);
          if (lane == b) acc += sum;
        }
      }
    s_sum[warp][lane] = (float)acc;
    if (__syncthreads_or(!ok)) {         // let the copies in flight land, for a while, before the CTA ends; nothing is written
      if (lane == 0) kv_err(a.err, KVERR_WAIT);
      for (u32 i = 0; i < S::STAGES; ++i) for (u32 y = 0; y < 2; ++y) bar_wait(bar0 + i * 8, y);
      return;
    }
  }
  if (tid < n_tile && b_tile + tid < a.b.max_blocks) {
    const u32 b = b_tile + tid;
    float sum = 0.0f;
    if (b >= b0 && b < b0 + nb) for (u32 w = 0; w < WS_WARPS; ++w) sum += s_sum[w][b - b0];
    if (x.weights) sum += x.keep * x.weights[seq * x.w_stride + b];
    x.out[seq * x.o_stride + b] = b < n_held ? sum : 0.0f;
  }
}

// Heads of every other size, any number of rows. `share` warps, no more than there are KV heads, work on a block, each on every so many-th head; a lane's 16 bytes of a key and
// of a query are operands of the matrix instruction if channels are counted in that order on both sides, so both go from memory to
// registers. The next (block, head)'s keys are on their way while one is worked on. Heads of 96: one token on 100,000 61 us (floor 24), 1000
// tokens 620 us (floor 2: rows go by eight, and a block's rows are not divided).
constexpr u32 WEIGH_LSE = 512;
template <class T, u32 G>      // G: 64-byte parts of a head
__global__ void __launch_bounds__(256, G > 4 ? 1 : 2) k_weigh(WeighArgs x, u32 n_tile, u32 share) {
  __shared__ float s_sum[8][WEIGH_TILE];
  __shared__ Lse s_lse[WEIGH_LSE];
  const AttendArgs &a = x.a;
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = a.p.n_kv_heads, g = a.group;
  const u32 tiles = (a.b.max_blocks + n_tile - 1) / n_tile, seq = blockIdx.x / tiles, b_tile = (blockIdx.x - seq * tiles) * n_tile;
  const Seq q = load_seq(a.b, seq, a.err);
  const u32 n_held = (q.kv + BT - 1) / BT;
  if (b_tile < n_held && q.n) {
    const bool staged = (u64)q.n * a.n_q_heads <= WEIGH_LSE;
    if (staged) {
      for (u32 i = tid; i < q.n * a.n_q_heads; i += 256) s_lse[i] = lse_log2(a.lse[(u64)q.t0 * a.n_q_heads + i]);
      __syncthreads();
    }
    const int shift = (int)q.kv - (int)q.n;                      // index of the first new token
    const u32 j = lane % 4, r8 = lane / 4, d = a.p.head_dim;
    // this warp's blocks b_tile + first + step * i and heads sub + share * k
    const u32 first = warp / share, step = 8 / share, sub = warp % share;
    const u32 n_blocks = min(n_tile, n_held - b_tile) > first ? (min(n_tile, n_held - b_tile) - first + step - 1) / step : 0, n_heads = (H - sub + share - 1) / share;
    u32 held = ~0u;                      // lane i: slot of block i
    if (lane < n_blocks && b_tile + first + step * lane >= first_seen(a, q)) {
      held = a.b.table[seq * a.b.table_stride + b_tile + first + step * lane];
      if (held >= a.p.n_slots && held - a.p.n_slots >= a.p.n_tail) kv_err(a.err, KVERR_RANGE);
    }
    struct Keys { uint4 v[G][2]; };
    auto load = [&](u32 i, u32 k) {
      Keys x;
      const u16 *const src = (const u16 *)slot_ptr(a.p, a.p.k, __shfl_sync(~0u, held, i));
      const bool vec = d % 8 == 0 && ((uintptr_t)src & 15) == 0;
#pragma unroll
      for (u32 y = 0; y < G; ++y)
#pragma unroll
        for (u32 z = 0; z < 2; ++z) {
          const u32 c = y * 32 + j * 8;
          x.v[y][z] = src && c < d ? load8(src + ((u64)(r8 + 8 * z) * H + sub + share * k) * d + c, (int)d - (int)c, vec) : make_uint4(0, 0, 0, 0);
        }
      return x;
    };
    double total = 0.0;                  // of the block, over the heads
    // of one block and head
    auto work = [&](const Keys &keys, u32 i, u32 k) {
      const u32 h = sub + share * k, b = b_tile + first + step * i;
      // rows that see any of the block's keys: tokens with index >= first key, and inside the window
      const int key0 = (int)(b * BT);
      const u32 tok0 = a.full ? 0 : (u32)max(0, key0 - shift);
      const u32 tok1 = a.window ? (u32)max(0ll, min((long long)q.n, (long long)key0 + BT - 1 + a.window - shift)) : q.n;
      double sum = 0.0;
      float part = 0.0f;
      u32 count = 0;
      for (u32 r0 = tok0 * g; r0 < tok1 * g; r0 += 8) {
        const u32 r = min(r0 + r8, tok1 * g - 1), tok = r / g;
        const u16 *const qs = (const u16 *)a.q + (u64)(q.t0 + tok) * a.q_ts + (u64)(h * g + r - tok * g) * a.q_hs;
        const bool qvec = d % 8 == 0 && ((uintptr_t)qs & 15) == 0;
        float s[4] = {0, 0, 0, 0};
#pragma unroll
        for (u32 y = 0; y < G; ++y) {
          const u32 c = y * 32 + j * 8;
          const uint4 v = c < d ? load8(qs + c, (int)d - (int)c, qvec) : make_uint4(0, 0, 0, 0);
          const u32 f0[4] = {keys.v[y][0].x, keys.v[y][1].x, keys.v[y][0].y, keys.v[y][1].y}, f1[4] = {keys.v[y][0].z, keys.v[y][1].z, keys.v[y][0].w, keys.v[y][1].w};
          mma16816<T>(s, f0, v.x, v.y);
          mma16816<T>(s, f1, v.z, v.w);
        }
#pragma unroll
        for (u32 z = 0; z < 2; ++z) {
          const u32 rr = r0 + 2 * j + z;
          if (rr >= tok1 * g) continue;
          const u32 tk = rr / g, at = tk * a.n_q_heads + h * g + rr - tk * g;
          const Lse L = staged ? s_lse[at] : lse_log2(a.lse[(u64)q.t0 * a.n_q_heads + at]);
          const int own = shift + (int)tk, hi = a.full ? (int)q.kv : own + 1, lo = a.window ? hi - (int)min(a.window, 0x7FFFFFFFu) : 0;
#pragma unroll
          for (u32 w = 0; w < 2; ++w) {
            const int key = key0 + (int)r8 + 8 * (int)w;
            const float v = s[2 * w + z], e = ex2(fmaf(v, a.scale_log2, -L.high) + fmaf(v, x.scale_low, -L.low));
            part += key < hi && key >= lo ? e : 0.0f;
          }
        }
        if (++count % 16 == 0) { sum += part; part = 0.0f; }   // sums of few in 32 bits, of those in 64
      }
      total += sum + part;
      if (k + 1 == n_heads) {            // the block is through
        const float all = sum_over_warp((float)total);
        if (lane == 0) s_sum[warp][first + step * i] = all;
        total = 0.0;
      }
    };
    const u32 n_items = n_blocks * n_heads;
    u32 i = 0, k = 0;                    // the item in hand
    auto after = [&](u32 &i, u32 &k) { if (++k == n_heads) { k = 0; ++i; } };
    if (n_items) {
      Keys one = load(0, 0), two;
      for (u32 it = 0; it < n_items; it += 2) {
        u32 i1 = i, k1 = k;
        after(i1, k1);
        if (it + 1 < n_items) two = load(i1, k1);
        work(one, i, k);
        if (it + 1 >= n_items) break;
        i = i1; k = k1;
        after(i, k);
        if (it + 2 < n_items) one = load(i, k);
        work(two, i1, k1);
      }
    }
    __syncthreads();
  }
  if (tid < n_tile && b_tile + tid < a.b.max_blocks) {
    const u32 b = b_tile + tid;
    float sum = 0.0f;
    if (b < n_held && q.n) for (u32 w = tid % (8 / share) * share, y = 0; y < share; ++y) sum += s_sum[w + y][tid];
    if (x.weights) sum += x.keep * x.weights[seq * x.w_stride + b];
    x.out[seq * x.o_stride + b] = b < n_held ? sum : 0.0f;
  }
}

// Many rows (prompts, chunks). Here the keys are the rows of the matrix instruction as well: S^T = K Q^T for 256 keys, two tiles of
// 128, by 128 (token, head) rows, so that a thread owns a key and adds up what its row of S^T gives in a register, with no
// exchange between threads and no masks but at the diagonal. The row's lse comes off in the product itself: with 16 channels more,
// constants on the side of K and the parts of -lse / scale in bf16 on the side of Q, S^T is (s - lse / scale) in 32 bits,
// and a power is one multiplication and ex2. (With lse from shared memory and a fused multiply-add it was bound by shared memory, which
// the products alone keep busy half of the time: 8192 tokens, 8 x 4 heads of 128, 352 us.)
// 256 keys by 128 rows take 2600 cycles. The special-function units need 1792 of them (2048 for all powers; every eighth pair is made on the
// FMA pipes: 341 -> 331 us; every fourth 331, three of eight 343), the tensor cores 1160, so neither is the limit: without the powers a step takes 1710
// cycles, without most of the products 2470. What is left is each thread's chain from tensor memory to the sum, four warps per scheduler. In a
// captured graph: 8192 tokens, 8 KV heads of 128, groups of 4 324 us (0.275 TFLOP: 849 TFLOP/s, half of the measured matrix rate), 500 tokens on 130,500
// 601 us, the last 32 of 32,000 26 us. One thread per key instead of two 410 us, K in stages of 256 keys and two stages of queries 339, lse in parts
// by 64-bit arithmetic 339, 32 columns of S at a time 375.
//   warps 0-15   two threads per key, each for half of the rows: powers and their sum
//   warp 16      issues the products, S^T in tensor memory, held twice: 2 x 2 x 128 columns
//   warp 17      works out what this CTA does
//   warp 18      loads K (TMA, a box per block), 128 keys of a head per stage, three stages: two in use, one ahead
//   warps 19-22  bring queries, up to 128 rows per stage (TMA where they lie as it wants them), and their lse; two warps for every other stage
// A tile of rows is as many tokens as fit 128 / group: rows are the same (token, head of the group) in every tile, and one box of TMA.
// Work: for each 256 keys of each sequence ("a pair" of tiles) the tiles of rows that see any of them, head by head. All of it,
// one tile after the other, is dealt out in equal stretches, one per CTA; a pair that several CTAs work on is put together from
// their sums by the kernel behind, always in the same order.
constexpr u32 WTC_KEYS = 256, WTC_KB = WTC_KEYS / BT, WTC_THREADS = 736, WTC_JOBS = 4, WTC_Q = 3, WTC_K = 3;
template <u32 D> struct WeighShape {
  static constexpr u32 BLOCK = BT * D * 2, K = TC_TILE * D * 2, Q = TC_TILE * D * 2, EXTRA = TC_TILE * 32, SMEM = WTC_K * K + WTC_Q * Q + (WTC_Q + 1) * EXTRA + 1024;
};
// The 16 channels more, [row / 8][channel / 8][row % 8][channel % 8] without swizzle (lbo = 128: next 8 channels, sbo = 256: next 8 rows).
// Channels 0 to 3 carry parts of -lse / scale over ALPHA = 2^-e, where the scale (of powers of two) is 2^e to 2^(e+1). They are bf16 in either
// type of pool, an instruction of its own on the same sums: fp16 numbers end at 2^16, and lse / scale of fp16 scores at 2^40.
__device__ __forceinline__ u64 plain_desc(u32 addr) { return (u64)((addr & 0x3FFFF) >> 4) | (u64)(128 >> 4) << 16 | (u64)(256 >> 4) << 32 | 1ull << 46; }
__device__ __forceinline__ float extra_alpha(float scale_log2) { return __uint_as_float((254u - (__float_as_uint(scale_log2) >> 23)) << 23); }
// -1 / scale as two numbers (the scale that scores are multiplied by is the one of powers of two): lse times it is -lse / scale. (32-bit arithmetic in two parts: with 64 bits the warps that make the
// parts were what the others waited for.)
struct PerScale { float high, low; };
__device__ __forceinline__ PerScale per_scale(const WeighArgs &x) {
  const double k = -1.4426950408889634 / ((double)x.a.scale_log2 + (double)x.scale_low);
  PerScale p;
  p.high = (float)k; p.low = (float)(k - (double)p.high);
  return p;
}
__device__ __forceinline__ uint4 extra_parts(float lse, const PerScale &k, float per_alpha) {
  typedef Elem<__nv_bfloat16> E;
  float e[4] = {0, 0, 0, 0};
  if (fabsf(lse) <= 1e30f) {
    float high = lse * k.high, low = fmaf(lse, k.high, -high) + lse * k.low;
    high *= per_alpha; low *= per_alpha;
#pragma unroll
    for (u32 y = 0; y < 4; ++y) {
      e[y] = E::up1(E::down1(high));
      high -= e[y];
      if (y == 0) high += low;           // (what is left of the first part is far smaller, so nothing of either is lost)
    }
  } else e[0] = lse != lse ? lse : lse > 0.0f || lse == -INFINITY ? -INFINITY : INFINITY;      // -inf: a row without keys, no weight
  return make_uint4(E::down(e[0], e[1]), E::down(e[2], e[3]), 0u, 0u);
}

// 2^t of two numbers without the special-function units: t = n + f with n the nearest whole number, 2^f on [-1/2, 1/2] by the polynomial of
// degree 5 with the least relative error (fitted by reweighted least squares: 7.5e-8; 2.0e-7 with the roundings of its steps), times
// 2^n put together from n's bits. Below 2^-127 it gives 0, above 2^128 Inf, and NaN for NaN.
__device__ __forceinline__ u64 mul2(u64 a, u64 b) { u64 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float within(float t) {
  float r;
  asm("{\n\t.reg .f32 x;\n\tmax.NaN.f32 x, %1, 0fC2FE0000;\n\tmin.NaN.f32 %0, x, 0f43000000;\n\t}" : "=f"(r) : "f"(t));     // [-127, 128]
  return r;
}
__device__ __forceinline__ u64 twice(float x) { return pack2(x, x); }
__device__ __forceinline__ u64 ex2_fma(float t0, float t1) {
  const u64 t = pack2(within(t0), within(t1));
  const u64 m = add2(t, twice(12582912.0f));               // 1.5 * 2^23: n in the lowest bits
  const u64 f = fma2(add2(m, twice(-12582912.0f)), twice(-1.0f), t);
  u64 p = fma2(twice(0.0013276472454890609f), f, twice(0.009675540961325169f));
  p = fma2(p, f, twice(0.05550713092088699f));
  p = fma2(p, f, twice(0.24022120237350464f));
  p = fma2(p, f, twice(0.6931469440460205f));
  p = fma2(p, f, twice(1.0000001192092896f));
  const float2 z = unpack2(m);
  return mul2(p, pack2(__uint_as_float((__float_as_uint(z.x) << 23) + 0x3F800000u), __uint_as_float((__float_as_uint(z.y) << 23) + 0x3F800000u)));
}

// Waits for the loads from tensor memory. What was added up from the numbers before is done first, and nothing is done with the new ones
// before: the compiler sees neither in the instruction.
__device__ __forceinline__ void tc_wait_ld16(u32 *r, u64 (&done)[2]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
               "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+l"(done[0]), "+l"(done[1]) :: "memory");
}

// Rows of a sequence that see any of the keys [key0, key0 + 256): tokens [lo, hi) of the new ones.
struct Seen { u32 lo, hi; };
__device__ __forceinline__ Seen seen_by(const AttendArgs &a, const Seq &q, u32 key0) {
  const long long shift = (long long)q.kv - q.n, last = min((long long)key0 + WTC_KEYS, (long long)q.kv) - 1;
  Seen s;
  s.lo = a.full ? 0u : (u32)max(0ll, min((long long)q.n, (long long)key0 - shift));
  s.hi = a.window ? (u32)max(0ll, min((long long)q.n, last + (long long)a.window - shift)) : q.n;
  s.hi = max(s.hi, s.lo);
  return s;
}
__device__ __forceinline__ u32 row_tiles(const Seen &s, u32 tokens) { return (s.hi - s.lo + tokens - 1) / tokens; }

// Scratch: a header {tiles per stretch, tiles}, the place of each pair in the work (and the end), a word per CTA (1: it has given up a
// wait, and its sums are not to be used), then 16 sums, one per block, for each (pair, CTA): the one of pair p and CTA c is number p + c,
// as each next one has a greater p or c. All but the sums are written whatever the waits come to, so what the kernel behind
// reads by them is in bounds.
struct WeighScratch { u64 *per, *place; u32 *lost; float *sums; };
__host__ __device__ __forceinline__ u64 weigh_pairs(u32 n_seqs, u32 max_blocks) { return (u64)n_seqs * ((max_blocks + WTC_KB - 1) / WTC_KB); }
__host__ __device__ __forceinline__ u64 weigh_header(u64 pairs, u32 n_ctas) { return (16 + 8 * (pairs + 1) + 4ull * n_ctas + 15) & ~15ull; }
__device__ __forceinline__ WeighScratch weigh_scratch(u8 *p, u32 n_seqs, u32 max_blocks, u32 n_ctas) {
  const u64 pairs = weigh_pairs(n_seqs, max_blocks);
  WeighScratch s;
  s.per = (u64 *)p;
  s.place = s.per + 2;
  s.lost = (u32 *)(s.place + pairs + 1);
  s.sums = (float *)(p + weigh_header(pairs, n_ctas));
  return s;
}

struct WeighJob {
  u32 t0, tokens, index0;      // first token, tokens that see any of the keys, index of the first one in its sequence
  u32 kv, key0, seq, first;    // first: block that is seen at all
  u32 tiles, x0, x1;           // row tiles of a head; tiles [x0, x1) of all heads
  u64 sum;                     // place of the sums
  u32 last;
};

template <class T, u32 D>
__global__ void __launch_bounds__(WTC_THREADS, 1)
k_weigh_tc(const __grid_constant__ WeighArgs x, const __grid_constant__ KvMaps maps, const __grid_constant__ CUtensorMap queries, u32 mapped) {
  typedef WeighShape<D> S;
  constexpr bool FP16 = !__is_same(T, __nv_bfloat16);
  extern __shared__ u8 smem_raw[];
  __shared__ __align__(8) u64 s_kfull[WTC_K], s_kempty[WTC_K], s_qfull[WTC_Q], s_qempty[WTC_Q], s_sfull[2], s_sempty[2], s_hfull[2 * WTC_JOBS], s_drain, s_jfull[WTC_JOBS], s_jempty[WTC_JOBS];
  __shared__ float s_half[WTC_JOBS][WTC_KEYS];
  __shared__ u32 s_tmem;
  __shared__ volatile u32 s_lost;
  __shared__ WeighJob s_job[WTC_JOBS];
  const AttendArgs &a = x.a;
  asm volatile("griddepcontrol.launch_dependents;");
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = a.p.n_kv_heads, g = a.group;
  const u32 kfull = smem_addr(s_kfull), kempty = smem_addr(s_kempty), qfull = smem_addr(s_qfull), qempty = smem_addr(s_qempty),
            sfull = smem_addr(s_sfull), sempty = smem_addr(s_sempty), hfull = smem_addr(s_hfull), drain = smem_addr(&s_drain), jfull = smem_addr(s_jfull), jempty = smem_addr(s_jempty);
  if (tid == 0) {
    for (u32 i = 0; i < 2 * WTC_JOBS; ++i) bar_init(hfull + i * 8, 4);
    for (u32 i = 0; i < 2; ++i) { bar_init(sfull + i * 8, 1); bar_init(sempty + i * 8, 16); }
    for (u32 i = 0; i < WTC_K; ++i) { bar_init(kfull + i * 8, 1); bar_init(kempty + i * 8, 1); }
    for (u32 i = 0; i < WTC_Q; ++i) { bar_init(qfull + i * 8, 3); bar_init(qempty + i * 8, 1); }
    for (u32 i = 0; i < WTC_JOBS; ++i) { bar_init(jfull + i * 8, 1); bar_init(jempty + i * 8, 22); }
    bar_init(drain, 1);
    s_lost = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (warp == 18 && lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(lane ? &maps.tail : &maps.pool) : "memory");
  tc_before();
  __syncthreads();
  tc_after();
  const u32 tmem = s_tmem;
  const u32 sk = (smem_addr(smem_raw) + 1023) & ~1023u, sq = sk + WTC_K * S::K, extra = sq + WTC_Q * S::Q;       // extra: K's constants, then a stage's parts of lse each
  const u32 TOK = TC_TILE / g, ROWS = TOK * g;           // tokens and rows of a tile
  volatile u32 *const lost = &s_lost;
  // Waits last as long as a job of another warp may: a tile of 128 rows takes a microsecond, and a job has no more than x0 .. x1 of
  // them; 32 for each of the longest that can be.
  const u64 most = (u64)H * ((a.b.n_tokens + TOK - 1) / TOK) * 8;
  const u32 patience = (u32)min(most, (u64)0x7FFFFFFF);
  u32 jobs = 0;
  auto next_job = [&](WeighJob &j) {
    const u32 at = jobs % WTC_JOBS;
    if (!tc_wait(jfull + at * 8, (jobs / WTC_JOBS) & 1, lost, patience)) return false;
    j = s_job[at];
    __syncwarp();
    if (lane == 0) bar_arrive(jempty + at * 8);
    ++jobs;
    return j.last == 0;
  };

  if (warp == 17) {
    // ---- what this CTA does. A lane per pair, 32 pairs of a sequence at a time; twice: for the sum of the work (and CTA 0 for the places,
    // before anything is waited for), then for its share.
    const WeighScratch sc = weigh_scratch(a.scratch, a.b.n_seqs, a.b.max_blocks, gridDim.x);
    u64 total = 0, per = 0, tokens = 0;
    u32 made = 0;
    bool ok = true;
    for (u32 pass = 0; pass < 2 && ok; ++pass) {
      const u64 begin = per * blockIdx.x, end = min(begin + per, total);
      u64 base = 0, pair = 0;
      for (u32 s0 = 0; s0 < a.b.n_seqs && ok; s0 += 32) {
        Seq mine{0, 0, 0};
        if (s0 + lane < a.b.n_seqs) mine = load_seq(a.b, s0 + lane, a.err);
        if (pass == 0) tokens += mine.n;
        const u32 n_here = min(32u, a.b.n_seqs - s0);
        for (u32 y = 0; y < n_here && ok; ++y) {
          Seq q;
          q.t0 = __shfl_sync(~0u, mine.t0, y); q.n = __shfl_sync(~0u, mine.n, y); q.kv = __shfl_sync(~0u, mine.kv, y);
          const u32 pairs = (q.kv + WTC_KEYS - 1) / WTC_KEYS;
          for (u32 k0 = 0; k0 < pairs && ok; k0 += 32) {
            const u32 k = k0 + lane;
            Seen seen{0, 0};
            if (k < pairs) seen = seen_by(a, q, k * WTC_KEYS);
            const u32 tiles = row_tiles(seen, TOK);
            const u64 work = (u64)tiles * H;
            u64 incl = work;
#pragma unroll
            for (u32 o = 1; o < 32; o *= 2) { const u64 z = __shfl_up_sync(~0u, incl, o); if (lane >= o) incl += z; }
            const u64 from = base + incl - work, to = base + incl;
            if (pass == 0) {
              if (blockIdx.x == 0 && k < pairs) sc.place[pair + k] = from;
            } else {
              const u64 f = max(from, begin), t = min(to, end);
              for (u32 mask = __ballot_sync(~0u, f < t); mask && ok; mask &= mask - 1) {
                const u32 at = made % WTC_JOBS;
                if (made >= WTC_JOBS && !(ok = !a.lose && tc_wait(jempty + at * 8, (made / WTC_JOBS - 1) & 1, lost, patience))) { *lost = 1; break; }
                if (lane == __ffs(mask) - 1) {
                  WeighJob j;
                  j.t0 = q.t0 + seen.lo; j.tokens = seen.hi - seen.lo; j.index0 = q.kv - q.n + seen.lo;
                  j.kv = q.kv; j.key0 = k * WTC_KEYS; j.seq = s0 + y; j.first = first_seen(a, q);
                  j.tiles = tiles; j.x0 = (u32)(f - from); j.x1 = (u32)(t - from);
                  j.sum = pair + k + blockIdx.x;
                  j.last = 0;
                  s_job[at] = j;
                }
                __syncwarp();
                if (lane == 0) bar_arrive(jfull + at * 8);
                ++made;
              }
            }
            base += __shfl_sync(~0u, incl, 31);
            if (pass && base >= end) { k0 = pairs; y = n_here; s0 = a.b.n_seqs; break; }
          }
          pair += pairs;
        }
      }
      if (pass == 0) {
#pragma unroll
        for (u32 o = 16; o; o /= 2) tokens += __shfl_xor_sync(~0u, tokens, o);
        // starts that go up and down make the same tokens count again and again: then nothing is added (load_seq has set the error word)
        total = tokens > a.b.n_tokens ? 0 : base;
        per = (total + gridDim.x - 1) / gridDim.x;
        if (blockIdx.x == 0 && lane == 0) { sc.per[0] = per; sc.per[1] = total; sc.place[pair] = base; }
      }
    }
    const u32 at = made % WTC_JOBS;
    if (ok && made >= WTC_JOBS) ok = tc_wait(jempty + at * 8, (made / WTC_JOBS - 1) & 1, lost, patience);
    if (ok && lane == 0) { s_job[at].last = 1; bar_arrive(jfull + at * 8); }
  } else if (warp == 18) {
    // ---- K: blocks in front of the window and behind the sequence's last read as zeros
    u32 it = 0;
    bool ok = true;
    for (WeighJob j; ok && next_job(j);) {
      const u32 b = j.key0 / BT + lane, held = (j.kv + BT - 1) / BT;
      u32 slot = ~0u;
      if (lane < WTC_KB && b < held && b >= j.first) {
        slot = a.b.table[j.seq * a.b.table_stride + b];
        if (slot >= a.p.n_slots && slot - a.p.n_slots >= a.p.n_tail) kv_err(a.err, KVERR_RANGE);
      }
      for (u32 h = j.x0 / j.tiles; ok && h <= (j.x1 - 1) / j.tiles; ++h)
        for (u32 tile = 0; tile < 2; ++tile, ++it) {
          const u32 st = it % WTC_K;
          if (it >= WTC_K && !(ok = tc_wait(kempty + st * 8, (it / WTC_K - 1) & 1, lost, patience))) break;
          if (lane == 0) bar_expect(kfull + st * 8, S::K);
          __syncwarp();
          if (lane / (WTC_KB / 2) == tile) load_block(a, maps, sk + st * S::K + lane % (WTC_KB / 2) * S::BLOCK, kfull + st * 8, slot, 2 * a.layer, h, D / 64);
          __syncwarp();
        }
    }
    for (u32 i = it > WTC_K ? it - WTC_K : 0; i < it; ++i) bar_wait(kfull + (i % WTC_K) * 8, (i / WTC_K) & 1);     // landed before the CTA ends
  } else if (warp == 16) {
    // ---- products
    if (elect_one()) {
      const u32 id = tc_idesc(FP16, TC_TILE, false), id_extra = tc_idesc(false, TC_TILE, false);
      const u64 dk0 = tc_desc(sk, 16, D * 16), dq0 = tc_desc(sq, 16, 1024), de = plain_desc(extra);
      u32 n = 0, it = 0;
      bool ok = true;
      for (; ok;) {
        const u32 at = jobs % WTC_JOBS;
        if (!(ok = tc_wait1(jfull + at * 8, (jobs / WTC_JOBS) & 1, lost, patience))) break;
        ++jobs;
        const u32 tiles = s_job[at].tiles, x0 = s_job[at].x0, x1 = s_job[at].x1, end = s_job[at].last;
        bar_arrive(jempty + at * 8);
        if (end) break;
        u32 r = x0 % tiles;
        bool fresh = true;
        for (u32 i = x0; i < x1; ++i, ++n) {
          const u32 st = n % WTC_Q, buf = n % 2, ks[2] = {it % WTC_K, (it + 1) % WTC_K};
          if (!(ok = tc_wait1(qfull + st * 8, (n / WTC_Q) & 1, lost, patience))) break;
          if (n >= 2 && !(ok = tc_wait1(sempty + buf * 8, (n / 2 - 1) & 1, lost, patience))) break;
          tc_after();
          const u64 dq = dq0 + st * (S::Q / 16);
#pragma unroll
          for (u32 tile = 0; tile < 2; ++tile) {
            if (fresh && !(ok = tc_wait1(kfull + ks[tile] * 8, ((it + tile) / WTC_K) & 1, lost, patience))) break;
            const u64 dk = dk0 + ks[tile] * (S::K / 16);
#pragma unroll
            for (u32 k = 0; k < D / 16; ++k)
              tc_mma_ss(tmem + buf * 256 + tile * 128, dk + ((k / 4) * 1024 + (k % 4) * 32) / 16, dq + ((k / 4) * (TC_TILE * 128) + (k % 4) * 32) / 16, id, k > 0);
            tc_mma_ss(tmem + buf * 256 + tile * 128, de, de + (1 + st) * (S::EXTRA / 16), id_extra, 1);
          }
          if (!ok) break;
          tc_commit(sfull + buf * 8);
          tc_commit(qempty + st * 8);
          fresh = ++r == tiles || i + 1 == x1;
          if (fresh) { r = 0; tc_commit(kempty + ks[0] * 8); tc_commit(kempty + ks[1] * 8); it += 2; }
        }
      }
      tc_commit(drain);                  // all products and their arrivals are done before the CTA ends
      bar_wait(drain, 0);
    }
    __syncwarp();
  } else if (warp >= 19) {
    // ---- queries: warps 19, 20 bring the even tiles, 21, 22 the odd ones
    const u32 side = (warp - 19) / 2, mine = (warp - 19) % 2 * 32 + lane;      // 64 threads
    constexpr u32 PER = D / 8, STEP = 64 / PER;                                // 16-byte parts of a row; rows per round
    const PerScale k = per_scale(x);
    const float per_alpha = 1.0f / extra_alpha(a.scale_log2);
    const u32 my_tok[2] = {mine / g, (mine + 64) / g};                         // tokens of the rows whose lse this thread brings
    u32 n = 0, brought = ~0u;
    // rows that no tile has, and that none has had yet: no NaN in them. The second 8 channels more are 0.
    auto zero = [](u32 at) { asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory"); };
    for (u32 i = side * 64 + mine; i < WTC_Q * S::Q / 16; i += 128) zero(sq + i * 16);
    for (u32 i = side * 64 + mine; i < WTC_Q * S::EXTRA / 16; i += 128) zero(extra + S::EXTRA + i * 16);
    if (side == 0) {                     // K's constants, before the first tile is handed over
      const float alpha = extra_alpha(a.scale_log2);
      const u32 c = Elem<__nv_bfloat16>::down(alpha, alpha);
      for (u32 row = mine; row < TC_TILE; row += 64) {
        const u32 at = extra + row / 8 * 256 + row % 8 * 16;
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(c), "r"(c), "r"(0), "r"(0) : "memory");
        zero(at + 128);
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("bar.sync 1, 128;" ::: "memory");
    bool ok = true;
    for (WeighJob j; ok && next_job(j);) {
      u32 h = j.x0 / j.tiles, r = j.x0 - h * j.tiles;
      for (u32 i = j.x0; i < j.x1; ++i, ++n) {
        if (n % 2 == side) {
          const u32 st = n % WTC_Q;
          const u32 left = min(TOK, j.tokens - r * TOK) * g, t = j.t0 + r * TOK;       // rows of this tile, its first token
          uint4 parts[2];                // while the stage is still in use
#pragma unroll
          for (u32 y = 0; y < 2; ++y) {
            const u32 row = mine + 64 * y;
            parts[y] = extra_parts(row < left ? a.lse[(u64)(t + my_tok[y]) * a.n_q_heads + h * g + row - my_tok[y] * g] : -INFINITY, k, per_alpha);
          }
          if (n >= WTC_Q && !(ok = tc_wait(qempty + st * 8, (n / WTC_Q - 1) & 1, lost, patience))) break;
          brought = n;
          if (mapped) {
            if (mine == 0) {
              bar_expect(qfull + st * 8, ROWS * D * 2);
#pragma unroll
              for (u32 y = 0; y < D / 64; ++y)
                asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                             ::"r"(sq + st * S::Q + y * (TC_TILE * 128)), "l"(&queries), "r"(64 * y), "r"(h * g), "r"(t), "r"(qfull + st * 8) : "memory");
            }
          } else {
            const u32 c = mine % PER;
#pragma unroll 4
            for (u32 y = 0; y < TC_TILE / STEP; ++y) {
              const u32 row = y * STEP + mine / PER, tok = row / g;
              const u32 dst = sq + st * S::Q + (c / 8) * (TC_TILE * 128) + row * 128 + (((c % 8) ^ (row % 8)) * 16);
              if (row < left) {
                const u16 *const src = (const u16 *)a.q + (u64)(t + tok) * a.q_ts + (u64)(h * g + row - tok * g) * a.q_hs + c * 8;
                u32 v[4];
#pragma unroll
                for (u32 z = 0; z < 4; ++z) v[z] = (u32)src[2 * z] | (u32)src[2 * z + 1] << 16;
                asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
              }
            }
            if (mine == 0) bar_arrive(qfull + st * 8);
          }
#pragma unroll
          for (u32 y = 0; y < 2; ++y) {
            const u32 row = mine + 64 * y;
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(extra + (1 + st) * S::EXTRA + row / 8 * 256 + row % 8 * 16),
                         "r"(parts[y].x), "r"(parts[y].y), "r"(parts[y].z), "r"(parts[y].w) : "memory");
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) bar_arrive(qfull + st * 8);
        }
        if (++r == j.tiles) { r = 0; ++h; }
      }
    }
    if (mapped && mine == 0 && brought != ~0u) {         // landed before the CTA ends: this side's last tile, and where it may not have been used the one before
      if (*lost && brought >= 2) bar_wait(qfull + ((brought - 2) % WTC_Q) * 8, ((brought - 2) / WTC_Q) & 1);
      bar_wait(qfull + (brought % WTC_Q) * 8, (brought / WTC_Q) & 1);
    }
  } else {
    // ---- powers and their sums: a key per thread, half of the columns
    const u32 tile = warp / 8, half = warp / 4 % 2, key_t = tid % TC_TILE, from = tmem + ((warp % 4) << 21) + tile * 128 + half * 64;
    const WeighScratch sc = weigh_scratch(a.scratch, a.b.n_seqs, a.b.max_blocks, gridDim.x);
    const u64 scale2 = pack2(a.scale_log2, a.scale_log2);
    u32 n = 0;
    bool ok = true;
    u32 v[2][16];
    auto begin = [&](u32 n) {            // the first columns of tile n
      if (!tc_wait(sfull + n % 2 * 8, (n / 2) & 1, lost, patience)) return false;
      tc_after();
      tc_ld16(v[0], from + n % 2 * 256);
      return true;
    };
    for (WeighJob j; ok && next_job(j);) {
      const u32 key = j.key0 + tile * TC_TILE + key_t;
      float sum = 0.0f, rest = 0.0f;     // rest: what rounding took from the sum, since a long prompt has thousands of tiles
      u32 r = j.x0 % j.tiles;
      if (!(ok = begin(n))) break;
      for (u32 i = j.x0; i < j.x1; ++i, ++n) {
        const u32 buf = n % 2;
        const u32 toks = min(TOK, j.tokens - r * TOK), cols = toks * g;
        const u32 index0 = j.index0 + r * TOK, index1 = index0 + toks - 1;        // of the tile's first and last token
        const u32 k0 = j.key0 + tile * TC_TILE, k1 = min(k0 + TC_TILE, j.kv);       // this tile's keys
        const bool whole = cols >= half * 64 + 64 && (a.full || k1 <= index0 + 1) && (!a.window || (u64)k0 + a.window > index1);
        u64 part[2] = {0, 0};
        // columns that see this thread's key: tokens from its own on, while it is inside the window; index0 is negative only with `full`
        u64 see = ~0ull;
        if (!whole) {
          const int behind = (int)key - (int)index0;
          const u32 lo = a.full ? 0u : (u32)max(behind, 0), hi = a.window ? (u32)max(0ll, min((long long)toks, (long long)behind + a.window)) : toks;
          const int lo_col = (int)(min(lo, toks) * g) - (int)half * 64, hi_col = (int)(hi * g) - (int)half * 64;
          see = (lo_col >= 64 ? 0ull : lo_col > 0 ? ~0ull << lo_col : ~0ull) & (hi_col >= 64 ? ~0ull : hi_col > 0 ? ~(~0ull << hi_col) : 0ull);
        }
#pragma unroll
        for (u32 c = 0; c < 4; ++c) {
          tc_wait_ld16(v[c & 1], part);
          if (c < 3) tc_ld16(v[(c + 1) & 1], from + buf * 256 + 16 * (c + 1));
          else {                         // S is read: on with the next tile's before the last powers of this one
            tc_before();
            __syncwarp();
            if (lane == 0) bar_arrive(sempty + buf * 8);
            if (i + 1 < j.x1 && !(ok = begin(n + 1))) break;
          }
          const float *const s = reinterpret_cast<const float *>(v[c & 1]);
          if (whole) {
#pragma unroll
            for (u32 y = 0; y < 16; y += 2) {
              const float2 p = unpack2(mul2(pack2(s[y], s[y + 1]), scale2));
              part[y / 2 % 2] = add2(part[y / 2 % 2], y == 4 ? ex2_fma(p.x, p.y) : pack2(ex2(p.x), ex2(p.y)));
            }
          } else {
            const u32 mask = (u32)(see >> (16 * c));
            if (__any_sync(~0u, mask & 0xFFFF)) {
#pragma unroll
              for (u32 y = 0; y < 16; y += 2) {
                auto power = [&](u32 i) { return mask >> i & 1 ? ex2(s[i] * a.scale_log2) : 0.0f; };
                part[y / 2 % 2] = add2(part[y / 2 % 2], pack2(power(y), power(y + 1)));
              }
            }
          }
        }
        if (!ok) break;
        const float2 all = unpack2(add2(part[0], part[1]));
        const float y = all.x + all.y, t = sum + y;
        rest += y - (t - sum);
        sum = t;                         // (nothing is negative, so the sum is nearly always the greater of the two)
        if (++r == j.tiles) r = 0;
      }
      if (!ok) break;
      if (sum < INFINITY) sum += rest;   // Inf stays Inf
      // The halves together. Four places in turn: the second half can be no more than two tiles of rows ahead of the first.
      const u32 at = (jobs - 1) % WTC_JOBS, bar = hfull + (tile * WTC_JOBS + at) * 8;
      if (half) {
        s_half[at][tile * TC_TILE + key_t] = sum;
        __syncwarp();
        if (lane == 0) bar_arrive(bar);
      } else {
        if (!(ok = tc_wait(bar, ((jobs - 1) / WTC_JOBS) & 1, lost, patience))) break;
        sum += s_half[at][tile * TC_TILE + key_t];
        if (key >= j.kv) sum = 0.0f;
#pragma unroll
        for (u32 o = 8; o; o /= 2) sum += __shfl_xor_sync(~0u, sum, o);
        if (lane % 16 == 0) sc.sums[j.sum * WTC_KB + key_t / BT + tile * (TC_TILE / BT)] = sum;
      }
    }
  }
  tc_before();
  __syncthreads();
  tc_after();
  if (warp == 16) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  if (tid == 0) {
    weigh_scratch(a.scratch, a.b.n_seqs, a.b.max_blocks, gridDim.x).lost[blockIdx.x] = s_lost;
    if (s_lost) kv_err(a.err, KVERR_WAIT);
  }
}

// Puts the sums of the kernel before, of n_ctas CTAs, together: a thread per block. Where one of them has given up nothing is written.
__global__ void __launch_bounds__(256) k_weigh_join(WeighArgs x, u32 n_ctas) {
  const AttendArgs &a = x.a;
  const u32 chunks = (a.b.max_blocks + 255) / 256, seq = blockIdx.x / chunks, b = (blockIdx.x - seq * chunks) * 256 + threadIdx.x;
  // the sequence's first pair
  u32 before = 0;
  for (u32 s0 = 0; s0 < seq; s0 += 256) {
    u32 n = 0;
    if (s0 + threadIdx.x < seq) n = (load_seq(a.b, s0 + threadIdx.x, a.err).kv + WTC_KEYS - 1) / WTC_KEYS;
    n = __reduce_add_sync(~0u, n);
    __shared__ u32 s_n[8];
    __syncthreads();
    if (threadIdx.x % 32 == 0) s_n[threadIdx.x / 32] = n;
    __syncthreads();
    for (u32 w = 0; w < 8; ++w) before += s_n[w];
  }
  const Seq q = load_seq(a.b, seq, a.err);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const WeighScratch sc = weigh_scratch(a.scratch, a.b.n_seqs, a.b.max_blocks, n_ctas);
  const u64 per = sc.per[0], total = sc.per[1];
  bool lost = false;
  for (u32 c = threadIdx.x; c < n_ctas; c += 256) lost |= sc.lost[c] != 0;
  if (__syncthreads_or(lost) || b >= a.b.max_blocks) return;
  double sum = 0.0;
  const bool held = b < (q.kv + BT - 1) / BT;
  if (held) {
    const u32 pair = before + b / WTC_KB;
    if (total) {
      const u64 from = sc.place[pair], to = sc.place[pair + 1];
      if (from < to) for (u64 c = from / per; c <= (to - 1) / per; ++c) sum += sc.sums[(pair + c) * WTC_KB + b % WTC_KB];
    }
    if (x.weights) sum += x.keep * x.weights[seq * x.w_stride + b];
  }
  x.out[seq * x.o_stride + b] = held ? (float)sum : 0.0f;
}

// Few rows or many. (One tile of 128 rows costs the second kernel as much as one row.)
constexpr u32 WEIGH_FEW = 32;
WeighPlan plan_weigh(const WeighArgs &x, u32 max_q_len, int sm_count) {
  WeighPlan p{};
  const u32 d = x.a.p.head_dim;
  const u64 rows = (u64)(max_q_len && max_q_len < x.a.b.n_tokens ? max_q_len : x.a.b.n_tokens) * x.a.group;
  // (the parts of lse / scale are bf16 numbers, over a power of two that is one as well: scales far from 1 are left to the first kernel)
  p.many = (d == 64 || d == 128) && rows > WEIGH_FEW && x.a.group <= TC_TILE && x.a.scale_log2 > 0x1p-13f && x.a.scale_log2 < 0x1p13f;
  p.grid = sm_count;
  const u64 blocks = (u64)x.a.b.n_seqs * x.a.b.max_blocks;
  if (d == 64 || d == 128) {             // four CTAs per slot, as long as a tile has a block
    p.share = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
    p.tile = (u32)std::max<u64>(1, std::min<u64>(WEIGH_TILE, blocks / (8ull * sm_count)));
  } else {                               // one warp per block and 32 blocks per CTA where there are enough of them, else the heads of a block over several warps
    p.share = 1;                         // (never more than KV heads)
    while (p.share < 8 && p.share * 2 <= x.a.p.n_kv_heads && blocks * p.share < 32ull * sm_count) p.share *= 2;
    p.tile = p.share == 1 && blocks >= 128ull * sm_count ? WEIGH_TILE : (u32)std::max<u64>(1, std::min<u64>(8, blocks / (2ull * sm_count)));
  }
  if (p.many) {
    const u64 pairs = weigh_pairs(x.a.b.n_seqs, x.a.b.max_blocks);
    p.scratch_bytes = weigh_header(pairs, p.grid) + (pairs + p.grid) * WTC_KB * 4;
  }
  return p;
}

template <class T, u32 D>
static cudaError_t launch_weigh_tc(const WeighArgs &x, const WeighPlan &p, const KvMaps &m, cudaStream_t s, u64 *allowed, u32 *launches) {
  cudaError_t r = allow_smem(k_weigh_tc<T, D>, 3 + (D == 128) * 2 + __is_same(T, __half), WeighShape<D>::SMEM, allowed);
  if (r != cudaSuccess) return r;
  CUtensorMap queries{};
  const u32 mapped = make_row_map(&queries, x.a.q, D, x.a.n_q_heads, x.a.b.n_tokens, x.a.q_hs, x.a.q_ts, x.a.group, TC_TILE / x.a.group);
  k_weigh_tc<T, D><<<p.grid, WTC_THREADS, WeighShape<D>::SMEM, s>>>(x, m, queries, mapped);
  ++*launches;
  if ((r = cudaGetLastError()) != cudaSuccess) return r;
  cudaLaunchConfig_t c{};
  c.gridDim = dim3(x.a.b.n_seqs * ((x.a.b.max_blocks + 255) / 256)); c.blockDim = dim3(256); c.stream = s;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  c.attrs = &at; c.numAttrs = 1;
  ++*launches;
  return cudaLaunchKernelEx(&c, k_weigh_join, x, p.grid);
}
template <class T, u32 D, u32 NT>
static cudaError_t launch_weigh_split(const WeighArgs &x, const WeighPlan &p, const KvMaps &m, cudaStream_t s, u64 *allowed) {
  constexpr u32 SMALL = WeighRing<D>::SMEM;
  const cudaError_t r = allow_smem(k_weigh_split<T, D, NT>, ((D == 128) * 2 + __is_same(T, __half)) * 3 + (NT == 4 ? 2 : NT - 1), SMALL, allowed + 1);
  if (r != cudaSuccess) return r;
  k_weigh_split<T, D, NT><<<x.a.b.n_seqs * ((x.a.b.max_blocks + p.tile - 1) / p.tile), WS_THREADS, SMALL, s>>>(x, m, p.tile);
  return cudaGetLastError();
}
template <class T, u32 D>
static cudaError_t launch_weigh_split(const WeighArgs &x, const WeighPlan &p, const KvMaps &m, cudaStream_t s, u64 *allowed, u32 *launches) {
  ++*launches;
  if (p.share == 1) return launch_weigh_split<T, D, 1>(x, p, m, s, allowed);
  if (p.share == 2) return launch_weigh_split<T, D, 2>(x, p, m, s, allowed);
  return launch_weigh_split<T, D, 4>(x, p, m, s, allowed);
}
cudaError_t launch_weigh(const WeighArgs &x, const WeighPlan &p, const KvMaps &m, cudaStream_t s, u64 *allowed, u32 *launches) {
  const u32 d = x.a.p.head_dim;
  if (p.many) {
    if (d == 64) return x.a.fp16 ? launch_weigh_tc<__half, 64>(x, p, m, s, allowed, launches) : launch_weigh_tc<__nv_bfloat16, 64>(x, p, m, s, allowed, launches);
    return x.a.fp16 ? launch_weigh_tc<__half, 128>(x, p, m, s, allowed, launches) : launch_weigh_tc<__nv_bfloat16, 128>(x, p, m, s, allowed, launches);
  }
  if (d == 64) return x.a.fp16 ? launch_weigh_split<__half, 64>(x, p, m, s, allowed, launches) : launch_weigh_split<__nv_bfloat16, 64>(x, p, m, s, allowed, launches);
  if (d == 128) return x.a.fp16 ? launch_weigh_split<__half, 128>(x, p, m, s, allowed, launches) : launch_weigh_split<__nv_bfloat16, 128>(x, p, m, s, allowed, launches);
  const u32 ctas = x.a.b.n_seqs * ((x.a.b.max_blocks + p.tile - 1) / p.tile);
  ++*launches;
  if (x.a.fp16) {
    if (d <= 64) k_weigh<__half, 2><<<ctas, 256, 0, s>>>(x, p.tile, p.share);
    else if (d <= 128) k_weigh<__half, 4><<<ctas, 256, 0, s>>>(x, p.tile, p.share);
    else k_weigh<__half, 8><<<ctas, 256, 0, s>>>(x, p.tile, p.share);
  } else {
    if (d <= 64) k_weigh<__nv_bfloat16, 2><<<ctas, 256, 0, s>>>(x, p.tile, p.share);
    else if (d <= 128) k_weigh<__nv_bfloat16, 4><<<ctas, 256, 0, s>>>(x, p.tile, p.share);
    else k_weigh<__nv_bfloat16, 8><<<ctas, 256, 0, s>>>(x, p.tile, p.share);
  }
  return cudaGetLastError();
}

// ======================================================================================================
// Eviction by weight: of a sequence's blocks the first, the last and the heaviest stay. A CTA per sequence. Bound by latency, three rounds of
// loads and some thirty barriers, and for long rows by the instructions of one SM: 1001 blocks 7.6 us, 32 sequences of up to 15,600 19 us, one of
// 62,501 115 us, in a captured graph.
// ======================================================================================================
constexpr u32 EVICT_THREADS = 1024;
__device__ __forceinline__ u32 weight_order(float w) { return ordered(w == w ? w + 0.0f : INFINITY); }       // a NaN weighs most

// R: the row in registers, so many blocks per thread, all of it read before anything is written, wherever the outputs are.
template <u32 R>
__global__ void __launch_bounds__(EVICT_THREADS) k_evict_blocks(EvictArgs a) {
  __shared__ u32 s_n[R * 32], s_all[R];
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, seq = blockIdx.x;
  u32 slot[R];
  float w[R];
#pragma unroll
  for (u32 k = 0; k < R; ++k) {
    const u32 i = tid + k * EVICT_THREADS;
    if (i < a.max_blocks) { slot[k] = a.table[seq * a.table_stride + i]; w[k] = a.weights[seq * a.w_stride + i]; }
  }
  const u32 room = a.max_blocks * BT;
  u32 kv = a.kv_len[seq];
  if (kv > room) { if (tid == 0) kv_err(a.err, KVERR_RANGE); kv = room; }
  const u32 had = (kv + BT - 1) / BT, gone = had > a.n_blocks ? had - a.n_blocks : 0, end = had - a.last;       // [first, end): those to choose from
  // flags: a bit per block of this thread; at: how many flagged blocks of the sequence come before each
  auto places = [&](u32 flags, u32 (&at)[R]) {
#pragma unroll
    for (u32 k = 0; k < R; ++k) {
      const u32 b = __ballot_sync(~0u, flags >> k & 1);
      at[k] = __popc(b & ((1u << lane) - 1));
      if (lane == 0) s_n[k * 32 + warp] = __popc(b);
    }
    __syncthreads();
    if (warp < R) {
      const u32 mine = s_n[warp * 32 + lane];
      u32 incl = mine;
#pragma unroll
      for (u32 o = 1; o < 32; o *= 2) { const u32 z = __shfl_up_sync(~0u, incl, o); if (lane >= o) incl += z; }
      s_n[warp * 32 + lane] = incl - mine;
      if (lane == 31) s_all[warp] = incl;
    }
    __syncthreads();
    u32 before = 0;
#pragma unroll
    for (u32 k = 0; k < R; ++k) { at[k] += before + s_n[k * 32 + warp]; before += s_all[k]; }
    __syncthreads();
  };
  u32 stays = 0, at[R];
#pragma unroll
  for (u32 k = 0; k < R; ++k) {
    const u32 i = tid + k * EVICT_THREADS;
    if (i < had && (!gone || i < a.first || i >= end)) stays |= 1u << k;
  }
  const u32 m = gone ? end - a.first - gone : 0;       // to be kept of those to choose from
  if (m) {
    const Kth kth = kth_largest<EVICT_THREADS>([&](auto f) {
#pragma unroll
      for (u32 k = 0; k < R; ++k) { const u32 i = tid + k * EVICT_THREADS; if (i >= a.first && i < end) f(weight_order(w[k])); }
    }, end - a.first, m);
    u32 ties = 0;
#pragma unroll
    for (u32 k = 0; k < R; ++k) {
      const u32 i = tid + k * EVICT_THREADS;
      if (i < a.first || i >= end) continue;
      const u32 x = weight_order(w[k]);
      if (x > kth.at || (x == kth.at && kth.ties == ~0u)) stays |= 1u << k;
      else if (x == kth.at) ties |= 1u << k;
    }
    if (kth.ties != ~0u) {               // of those that weigh the same the first ones
      places(ties, at);
#pragma unroll
      for (u32 k = 0; k < R; ++k) if ((ties >> k & 1) && at[k] < kth.ties) stays |= 1u << k;
    }
  }
  places(stays, at);
  u32 *const table_out = a.table_out + seq * a.table_out_stride, *const evicted = a.evicted + seq * a.evicted_stride;
  float *const weights_out = a.weights_out + seq * a.w_out_stride;
  const u32 kept = had - gone;
#pragma unroll
  for (u32 k = 0; k < R; ++k) {
    const u32 i = tid + k * EVICT_THREADS;
    if (i < had) {
      if (stays >> k & 1) { table_out[at[k]] = slot[k]; weights_out[at[k]] = w[k]; }
      else evicted[i - at[k]] = slot[k];
    }
    if (i >= kept && i < a.max_blocks) { table_out[i] = ~0u; weights_out[i] = 0.0f; }
    if (i >= gone && i < a.max_blocks) evicted[i] = ~0u;
  }
  if (tid == 0) a.kv_len_out[seq] = kv - gone * BT;
}

// Rows of any length, 4 K blocks at a time: read, then written at or in front of where they were.
__global__ void __launch_bounds__(EVICT_THREADS) k_evict_long(EvictArgs a, u32 held) {
  extern __shared__ u32 s_keys[];
  __shared__ u32 s_border, s_n[EVICT_THREADS / 32];
  const u32 tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, seq = blockIdx.x;
  const u32 *const table = a.table + seq * a.table_stride;
  const float *const weights = a.weights + seq * a.w_stride;
  u32 *const table_out = a.table_out + seq * a.table_out_stride, *const evicted = a.evicted + seq * a.evicted_stride;
  float *const weights_out = a.weights_out + seq * a.w_out_stride;
  const u32 room = a.max_blocks * BT;
  u32 kv = a.kv_len[seq];
  if (kv > room) { if (tid == 0) kv_err(a.err, KVERR_RANGE); kv = room; }
  const u32 had = (kv + BT - 1) / BT, gone = had > a.n_blocks ? had - a.n_blocks : 0;
  auto order = [&](float w) { return weight_order(w); };
  Kth kth{0, ~0u};
  u32 border = 0;
  if (gone) {                            // of the n blocks between the first and the last ones m stay
    const u32 n = had - a.first - a.last, m = n - gone;
    const float *const w = weights + a.first;
    if (n <= held) for (u32 i = tid; i < n; i += EVICT_THREADS) s_keys[i] = order(w[i]);
    __syncthreads();
    auto key = [&](u32 i) { return n <= held ? s_keys[i] : order(w[i]); };
    if (m) kth = kth_largest<EVICT_THREADS>([&](auto f) { for (u32 i = tid; i < n; i += EVICT_THREADS) f(key(i)); }, n, m); else kth = Kth{~0u, 0};
    __syncthreads();
    if (kth.ties != ~0u && kth.ties) {
      deal<EVICT_THREADS>(n, [&](u32 i) { return key(i) == kth.at ? 1u : 0u; }, [&](u32 i, u32, u32 at) { if (at == kth.ties - 1) s_border = i; });
      __syncthreads();
      border = s_border;
    }
  }
  // in order, 4 blocks of each thread at a time: read, then written at or in front of where they were
  u32 at[2] = {0, 0};
  for (u32 i0 = 0; i0 < had; i0 += 4 * EVICT_THREADS) {
    u32 slot[4], stays = 0, n[2] = {0, 0};
    float w[4];
#pragma unroll
    for (u32 y = 0; y < 4; ++y) {
      const u32 i = i0 + 4 * tid + y;
      if (i >= had) continue;
      slot[y] = table[i]; w[y] = weights[i];
      const u32 x = order(w[y]);
      const bool stay = !gone || i < a.first || i >= had - a.last || x > kth.at || (x == kth.at && (kth.ties == ~0u || (kth.ties && i - a.first <= border)));
      stays |= (u32)stay << y;
      ++n[stay ? 0 : 1];
    }
    u32 incl = n[0] | n[1] << 16;        // at most 4096 each
    const u32 here = incl;
#pragma unroll
    for (u32 o = 1; o < 32; o *= 2) { const u32 z = __shfl_up_sync(~0u, incl, o); if (lane >= o) incl += z; }
    __syncthreads();                     // everything is read; the sums of the round before too
    if (lane == 31) s_n[warp] = incl;
    __syncthreads();
    u32 before = 0, all = 0;
#pragma unroll
    for (u32 v = 0; v < EVICT_THREADS / 32; ++v) { if (v < warp) before += s_n[v]; all += s_n[v]; }
    before += incl - here;
    u32 to[2] = {at[0] + (before & 0xFFFF), at[1] + (before >> 16)};
#pragma unroll
    for (u32 y = 0; y < 4; ++y) {
      if (i0 + 4 * tid + y >= had) continue;
      if (stays >> y & 1) { table_out[to[0]] = slot[y]; weights_out[to[0]++] = w[y]; }
      else evicted[to[1]++] = slot[y];
    }
    at[0] += all & 0xFFFF; at[1] += all >> 16;
  }
  __syncthreads();
  for (u32 i = at[0] + tid; i < a.max_blocks; i += EVICT_THREADS) { table_out[i] = ~0u; weights_out[i] = 0.0f; }
  for (u32 i = at[1] + tid; i < a.max_blocks; i += EVICT_THREADS) evicted[i] = ~0u;
  if (tid == 0) a.kv_len_out[seq] = kv - gone * BT;
}

cudaError_t launch_evict(const EvictArgs &a, cudaStream_t s, u64 *allowed, u32 *launches) {
  if (a.max_blocks <= 4096) k_evict_blocks<4><<<a.n_seqs, EVICT_THREADS, 0, s>>>(a);
  else if (a.max_blocks <= 8192) k_evict_blocks<8><<<a.n_seqs, EVICT_THREADS, 0, s>>>(a);
  else if (a.max_blocks <= 16384) k_evict_blocks<16><<<a.n_seqs, EVICT_THREADS, 0, s>>>(a);
  else {
    const u32 held = std::min(a.max_blocks, 45u * 1024);         // keys in shared memory
    const cudaError_t r = allow_smem(k_evict_long, 2, 180 * 1024, allowed);
    if (r != cudaSuccess) return r;
    k_evict_long<<<a.n_seqs, EVICT_THREADS, held * 4, s>>>(a, held);
  }
  ++*launches;
  return cudaGetLastError();
}

}  // namespace kvt
