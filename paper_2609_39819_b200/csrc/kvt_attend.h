// kvt_attend.h — what the entry points in kvt_engine.cu hand to the kernels in kvt_attend.cu.
#pragma once
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

namespace kvt {

// bits of the sticky error word of the model-side operators
enum : uint32_t { KVERR_RANGE = 1, KVERR_WAIT = 2 };

// One chunk row (layer, K or V) of the pools: slot s < n_slots lies at base + s * slot_stride, slot n_slots + i is tail
// block i at tail + i * tail_stride. Inside a block: [16 tokens][n_kv_heads][head_dim].
struct KvRow { uint8_t *base, *tail; };
struct KvPools {
  KvRow k, v;
  uint64_t slot_stride, tail_stride;
  uint32_t n_slots, n_tail;
  uint32_t n_kv_heads, head_dim;
};

struct KvBatch {
  const uint32_t *q_start, *kv_len, *table;
  uint64_t table_stride;
  uint32_t n_seqs, n_tokens, max_blocks;
};

struct AppendArgs {
  KvBatch b; KvPools p;
  const void *q, *k, *v; void *q_out;
  uint64_t q_ts, q_hs, k_ts, k_hs, v_ts, v_hs, qo_ts, qo_hs;
  const double *freqs; const uint8_t *axis_of; const int32_t *positions; uint64_t pos_stride;
  uint32_t n_q_heads, rot_dim, n_axes, interleaved, fp16;
  uint32_t *err;
};

struct AttendArgs {
  KvBatch b; KvPools p;
  const void *q; void *out; float *lse;
  uint64_t q_ts, q_hs, o_ts, o_hs;
  uint32_t n_q_heads, group, window, full, fp16;
  uint32_t layer, layer_major;
  uint8_t *scratch;
  float scale_log2;                 // scale / ln 2: scores in powers of two
  uint32_t *err;
};

// Tensor maps of the pool and of the tail blocks (tail = pool where there are none), for head sizes of 64 and 128: a box
// is one head of a block's 16 tokens, and lands in shared memory as [2][head_dim / 64][8 tokens][64] with 128-byte
// swizzle, the operand layout of the matrix instructions. A coordinate behind the last slot reads as zeros.
struct KvMaps { CUtensorMap pool, tail; };
bool make_kv_map(CUtensorMap *m, void *base, bool layer_major, uint64_t n_slots, uint64_t n_chunks, uint64_t n_kv_heads,
                 uint64_t head_dim);

// What kvt_attend does, decided from sizes alone.
struct AttendPlan {
  uint32_t kind;             // 0 any other head size, 1 few rows (warp-level matrix instructions), 2 many rows (tcgen05),
                             // 3 few rows of few and moderately long units (clusters)
  uint32_t rows;             // rows of a tile
  uint32_t sms, grid, cluster;
  uint32_t parts;            // partial results there is room for; 0: nothing can be cut
  uint64_t most;             // kind 1: work, kind 2: tiles that sequences which do not overlap can bring
  uint64_t scratch_bytes;
};
AttendPlan plan_attend(const AttendArgs &a, uint32_t max_q_len, int sm_count);

// out = *err, *err = 0, in one step: a bit that a kernel on another stream sets meanwhile is in `out` or stays for the next time.
cudaError_t launch_take_error(uint32_t *err, uint32_t *out, cudaStream_t s);
cudaError_t launch_append(const AppendArgs &a, cudaStream_t s, uint32_t *launches);
// allowed: bits of the kernels whose shared memory has been asked for on this engine's device
cudaError_t launch_attend(const AttendArgs &a, const AttendPlan &p, const KvMaps &m, cudaStream_t s, uint64_t *allowed, uint32_t *launches);

}  // namespace kvt
