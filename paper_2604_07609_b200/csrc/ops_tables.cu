// Block tables and slot maps of a step, from the requests' lengths: blink_build_tables.
//
//   need[r] = max(0, ceil((ctx[r] + new[r]) / 16) - held[r]),  first[r] = sum of need before r,  row_start[r] = sum of new before r
//   block_table[r][held[r] + j] = free[F - 1 - first[r] - j]            (the order in which the serving loop pops its stack)
//   row i of request r: position ctx[r] + i, slot = its block * 16 + position % 16
//
// What bounds it: latency (8 requests 4 us, 256 requests with 110 thousand rows 5.3, of which some 3 are a launch's).  A few KB are read, 8 bytes a row
// written; a step has hundreds to some ten thousand rows.  So one launch,
// and no memory between CTAs: every CTA of a cluster adds up the lengths for itself (two loads a request and one scan), then
// takes its share of the requests' blocks and of the rows.  A row finds its request by a search in shared memory and reads a
// new block from the stack itself, so that nobody waits for the tables.  The barrier of the cluster stands between the last read and the
// first write of what may be the same memory (held, count).
#include <cooperative_groups.h>

#include "ops.h"

namespace blink {

constexpr int TAB_THREADS = 1024;
constexpr int TAB_MAX_BLOCK = (1 << 27) - 1;   // a slot of it still fits 31 bits

struct TablesArgs {
  const int32_t *ctx_len, *new_len, *held, *free_blocks, *free_count;
  int n, free_capacity, stride, max_rows;
  int32_t *block_table, *held_out, *free_count_out, *row_start, *kv_len, *positions, *slot_map, *status;
};

__global__ void __launch_bounds__(TAB_THREADS) blink_tables_kernel(const TablesArgs a) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  extern __shared__ int s_dyn[];
  int* s_row = s_dyn;                 // [n + 1] first row of a request
  int* s_need = s_dyn + (a.n + 1);    // [n + 1] blocks handed out before it
  int* s_ctx = s_need + (a.n + 1);    // [n]
  int* s_held = s_ctx + a.n;          // [n]
  __shared__ long long s_warp[2][32];
  __shared__ int s_err;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
  ops_begin();
  if (tid == 0) s_err = 0;
  __syncthreads();

  // lengths, a run of requests per thread
  const int per = (a.n + TAB_THREADS - 1) / TAB_THREADS;
  const int r0 = min(a.n, tid * per), r1 = min(a.n, r0 + per);
  long long rows = 0, need = 0;
  int err = 0;
  for (int r = r0; r < r1; ++r) {
    const int ctx = a.ctx_len[r], add = a.new_len[r], held = a.held[r];
    const long long end = (long long)ctx + add;
    const long long want = (end + OPS_BLOCK - 1) / OPS_BLOCK - held;
    if (ctx < 0 || add < 0 || held < 0) err = max(err, 3);
    else if (held > a.stride || (end + OPS_BLOCK - 1) / OPS_BLOCK > a.stride || end > 0x7fffffff - OPS_BLOCK) err = max(err, 2);
    s_ctx[r] = ctx;
    s_held[r] = held;
    s_row[r] = (int)rows;   // (within the thread's run; its start is added below)
    s_need[r] = (int)need;
    rows += max(add, 0);
    need += max(want, 0ll);
  }
  const int count = *a.free_count;
  if (count < 0 || count > a.free_capacity) err = max(err, 3);
  long long x = rows, y = need;   // inclusive sums over the threads
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, x, d), v = __shfl_up_sync(0xffffffffu, y, d);
    if (lane >= d) { x += u; y += v; }
  }
  if (lane == 31) { s_warp[0][warp] = x; s_warp[1][warp] = y; }
  if (err) atomicMax(&s_err, err);
  __syncthreads();
  if (warp == 0) {
    long long u = s_warp[0][lane], v = s_warp[1][lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long p = __shfl_up_sync(0xffffffffu, u, d), q = __shfl_up_sync(0xffffffffu, v, d);
      if (lane >= d) { u += p; v += q; }
    }
    s_warp[0][lane] = u;
    s_warp[1][lane] = v;
  }
  __syncthreads();
  const long long tot_rows = s_warp[0][31], tot_need = s_warp[1][31];
  const long long row_base = x - rows + (warp ? s_warp[0][warp - 1] : 0), need_base = y - need + (warp ? s_warp[1][warp - 1] : 0);
  // all of it or nothing; bad lengths before sizes before an empty stack
  const int bad = s_err;
  const int status = bad == 3 ? BLINK_EINVAL : bad == 2 || tot_rows > a.max_rows ? BLINK_ETOOBIG : tot_need > count ? BLINK_ENOMEM : BLINK_OK;
  const bool ok = status == BLINK_OK;
  if (ok)
    for (int r = r0; r < r1; ++r) {
      s_row[r] += (int)row_base;
      s_need[r] += (int)need_base;
    }
  if (tid == 0) {
    s_row[a.n] = (int)tot_rows;
    s_need[a.n] = (int)tot_need;
  }
  __syncthreads();
  if (ctas > 1) cluster.sync();   // every CTA has read held and count

  for (int r = rank * TAB_THREADS + tid; r <= a.n; r += ctas * TAB_THREADS) {
    a.row_start[r] = ok ? s_row[r] : 0;
    if (r < a.n) {
      const int add = ok ? s_row[r + 1] - s_row[r] : 0, more = ok ? s_need[r + 1] - s_need[r] : 0;
      a.kv_len[r] = ok ? s_ctx[r] + add : 0;
      a.held_out[r] = s_held[r] + more;
    }
  }
  if (rank == 0 && tid == 0) {
    *a.free_count_out = ok ? count - (int)tot_need : count;
    *a.status = status;
  }
  if (ok) {
    // new blocks into the tables, one each
    for (int i = rank * TAB_THREADS + tid; i < (int)tot_need; i += ctas * TAB_THREADS) {
      int lo = 0, hi = a.n;   // last request with s_need <= i (of equal ones the last: those before it need nothing)
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_need[mid] <= i) lo = mid; else hi = mid;
      }
      a.block_table[(size_t)lo * a.stride + s_held[lo] + (i - s_need[lo])] = a.free_blocks[count - 1 - i];
    }
  }
  const int live = ok ? (int)tot_rows : 0;
  // rows, four in a row per thread: one search, the four blocks on their way together, 16 bytes a store
  const bool vec = ((reinterpret_cast<uintptr_t>(a.positions) | reinterpret_cast<uintptr_t>(a.slot_map)) & 15) == 0;
  for (int i0 = 4 * (rank * TAB_THREADS + tid); i0 < a.max_rows; i0 += 4 * ctas * TAB_THREADS) {
    int lo = 0;
    if (i0 < live) {
      int hi = a.n;   // the last request that begins at or before the row
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_row[mid] <= i0) lo = mid; else hi = mid;
      }
    }
    int pos[4], slot[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = i0 + j;
      pos[j] = slot[j] = -1;
      if (i < live) {
        while (s_row[lo + 1] <= i) ++lo;
        pos[j] = s_ctx[lo] + (i - s_row[lo]);
        const int b = pos[j] / OPS_BLOCK, fresh = b - s_held[lo];
        slot[j] = fresh >= 0 ? a.free_blocks[count - 1 - (s_need[lo] + fresh)] : a.block_table[(size_t)lo * a.stride + b];
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) slot[j] = slot[j] >= 0 && slot[j] <= TAB_MAX_BLOCK ? slot[j] * OPS_BLOCK + pos[j] % OPS_BLOCK : -1;
    if (vec && i0 + 4 <= a.max_rows) {
      *reinterpret_cast<int4*>(a.positions + i0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
      *reinterpret_cast<int4*>(a.slot_map + i0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i0 + j < a.max_rows) {
          a.positions[i0 + j] = pos[j];
          a.slot_map[i0 + j] = slot[j];
        }
    }
  }
}

}  // namespace blink

extern "C" int blink_build_tables(const int32_t* ctx_len, const int32_t* new_len, const int32_t* blocks_held, int n_requests,
                                  const int32_t* free_blocks, int free_capacity, const int32_t* free_count, int32_t* block_table,
                                  int table_stride, int max_rows, int32_t* blocks_held_out, int32_t* free_count_out, int32_t* row_start,
                                  int32_t* kv_len, int32_t* positions, int32_t* slot_map, int32_t* status, void* stream) {
  using namespace blink;
  const void* must[] = {ctx_len, new_len, blocks_held, free_blocks, free_count, block_table, blocks_held_out, free_count_out,
                        row_start, kv_len, positions, slot_map, status};
  for (const void* p : must)
    if (!ops_aligned(p, 4)) return BLINK_EINVAL;
  if (n_requests < 1 || free_capacity < 0 || table_stride < 1 || max_rows < 1) return BLINK_EINVAL;
  if (n_requests > OPS_MAX_REQUESTS || max_rows > 0x3fffffff) return BLINK_ETOOBIG;
  const TablesArgs a = {ctx_len, new_len, blocks_held, free_blocks, free_count, n_requests, free_capacity, table_stride, max_rows,
                        block_table, blocks_held_out, free_count_out, row_start, kv_len, positions, slot_map, status};
  // (four rows a thread: 110 thousand rows of 256 requests 6.9 us with eight CTAs, 5.3 with 16)
  const int cluster = max_rows > 32 * TAB_THREADS ? 16 : max_rows > 4 * TAB_THREADS || n_requests > TAB_THREADS ? 8 : 1;
  const OpsShared smem((size_t)(4 * n_requests + 2) * 4, (size_t)(4 * OPS_MAX_REQUESTS + 2) * 4);
  return ops_launch(blink_tables_kernel, cluster, TAB_THREADS, smem, stream, cluster, a);
}
