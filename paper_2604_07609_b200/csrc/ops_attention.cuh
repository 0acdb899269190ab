// What the kernels of blink_window_attention share.
#pragma once
#include <cuda_bf16.h>

#include "ops.h"

namespace blink {

struct AttnArgs {
  OpsPool pool;
  const void* q;
  void* out;
  long long q_stride, out_stride;   // elements between rows
  const int32_t *row_start, *kv_len, *table;
  int n, rows, stride;              // requests, rows of q, block ids of a table row
  int window, sinks;                // window 0: no window
  int few;                          // requests of up to so many rows go to attn_few, longer ones to the tiles
  float qscale;                     // 1 / sqrt(hd) * log2(e)
  int near_ctas, near_groups;       // > 0: a cluster of so many CTAs per unit; clusters per (request, kv head)
  bool out_32;                      // rows of out begin on 32-byte boundaries
  char* ws;
};

// A request as the kernels see it: lengths that would reach behind its table row or the rows are cut.
struct AttnReq {
  int start, rows, ctx;   // first row, rows, position of the first row
};
__device__ __forceinline__ AttnReq attn_req(const AttnArgs& a, int start, int end, int kv_len) {
  AttnReq r;
  r.start = min(max(start, 0), a.rows);
  r.rows = min(max(end, r.start), a.rows) - r.start;
  r.ctx = (int)min((long long)max(kv_len, 0), (long long)a.stride * OPS_BLOCK) - r.rows;
  return r;
}

// The blocks that rows at positions first .. last see: the first `sinks` of the table, and from block `from` on, `n` in all.
struct AttnSpan {
  int sinks, from, n;
};
__device__ __forceinline__ AttnSpan attn_span(const AttnArgs& a, int first, int last) {
  AttnSpan s;
  if (last < 0) return {0, 0, 1};   // nothing is seen; a unit has one tile at least, so that its zeros are written
  s.from = a.window > 0 ? max(0, first - a.window + 1) / OPS_BLOCK : 0;
  s.sinks = min((a.sinks + OPS_BLOCK - 1) / OPS_BLOCK, s.from);
  s.n = s.sinks + last / OPS_BLOCK - s.from + 1;
  return s;
}
__device__ __forceinline__ bool attn_sees(const AttnArgs& a, int key, int pos) {
  return key <= pos && (a.window == 0 || key > pos - a.window || key < a.sinks);
}

// The workspace begins with a word that is 0, or BLINK_ETIMEDOUT when a wait inside the kernels ran out (rows that are not done are then NaN).
constexpr size_t ATTN_STATUS_BYTES = 256;
// Requests of more than a.few rows on tcgen05 (ops_attn_tiles.cu); the others are in the stream before it.
int attn_tiles(const AttnArgs& a, int sms, void* stream);
// The same in 32 bits (ops_attn_block.cu).
int attn_blocks(const AttnArgs& a, int sms, void* stream);

__device__ __forceinline__ float attn_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

}  // namespace blink
