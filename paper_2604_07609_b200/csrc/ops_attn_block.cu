// blink_window_attention in 32 bits for requests of more than a few rows, on the CUDA cores: there is no matrix instruction of that precision.
//
// A unit is a request, a kv head and 32 or 16 (query row, head) rows, a CTA each.  Keys come in tiles of 64, the visible blocks of the unit, sinks first,
// four to a tile; keys and values through shared memory by asynchronous copies, the next keys on their way while the output is formed
// and the next values during the scores.  A thread has R rows (4 or 2) x 4 keys of the scores and R rows x HD / 16 dims of the output: with four, 12 wavefronts of
// shared memory for 64 multiply-adds a warp, which then take as long.  The 16 threads of a row are half a warp, so maxima and sums are shuffles.
//
// What bounds it: multiply-adds, and in small calls the cold instructions: the loops are not unrolled further than that.  (As units of 8 rows
// in registers, with everything unrolled, the small configuration's batch took 22.5 us, 12.6 here; a prompt of 1000 rows of the 8B shape
// 1024 us, 336 here: 25 of 74 TFLOP/s that the multiply-adds could do.)
#include <cmath>

#include "ops_attention.cuh"

namespace blink {

constexpr int BLK_THREADS = 128, BLK_KEYS = 64, BLK_BLOCKS = BLK_KEYS / OPS_BLOCK;
constexpr int BLK_IDS = 128;   // block ids of a unit that are read at once

template <int HD, int R>   // R: rows of a thread
struct BlkShape {
  static constexpr int ROWS = 8 * R, PITCH = HD + 4, P_PITCH = BLK_KEYS + 4;   // floats
  static constexpr int Q = 0, K = ROWS * PITCH, V = K + BLK_KEYS * PITCH, P = V + BLK_KEYS * PITCH, END = P + ROWS * P_PITCH;
};

template <int HD, int R>
__global__ void __launch_bounds__(BLK_THREADS) blink_attn_block_kernel(const __grid_constant__ AttnArgs a) {
  using S = BlkShape<HD, R>;
  constexpr int BLK_ROWS = S::ROWS;
  extern __shared__ __align__(16) float s_f[];
  __shared__ int s_ids[BLK_IDS];   // of the list's first blocks
  __shared__ int s_warp[BLK_THREADS / 32], s_unit[5];   // of the unit: request; its first row, rows and first position; rows (of a head) before it
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rep = a.pool.rep;
  ops_begin();
  if (a.few == 0 && blockIdx.x == 0 && tid == 0) *reinterpret_cast<int*>(a.ws) = 0;   // (else the kernels behind this one do)
  // the unit: the CTA's place in the sequence of all of them, found by the thread whose run of requests holds it
  const int h = (int)blockIdx.x % a.pool.Hkv, place = (int)blockIdx.x / a.pool.Hkv;
  const int each = (a.n + BLK_THREADS - 1) / BLK_THREADS, r0 = min(a.n, tid * each), r1 = min(a.n, r0 + each);
  auto groups_of = [&](const AttnReq& q) { return q.rows > a.few ? (q.rows * rep + BLK_ROWS - 1) / BLK_ROWS : 0; };
  int mine = 0;
  for (int r = r0; r < r1; ++r) mine += groups_of(attn_req(a, a.row_start[r], a.row_start[r + 1], a.kv_len[r]));
  int x = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) s_warp[warp] = x;
  if (tid == 0) s_unit[0] = -1;
  __syncthreads();
  for (int i = 0; i < warp; ++i) x += s_warp[i];
  if (place >= x - mine && place < x) {
    int at = x - mine;
    for (int r = r0; r < r1; ++r) {
      const AttnReq q = attn_req(a, a.row_start[r], a.row_start[r + 1], a.kv_len[r]);
      const int g = groups_of(q);
      if (place < at + g) {
        s_unit[0] = r;
        s_unit[1] = q.start;
        s_unit[2] = q.rows;
        s_unit[3] = q.ctx;
        s_unit[4] = (at + g - 1 - place) * BLK_ROWS;   // later rows, which see more, first
        break;
      }
      at += g;
    }
  }
  __syncthreads();
  const int r = s_unit[0];
  if (r < 0) return;   // (the grid is as large as it can have to be)
  const int start = s_unit[1], ctx = s_unit[3], m0 = s_unit[4], m1 = min(s_unit[2] * rep, m0 + BLK_ROWS);
  const int first = ctx + m0 / rep, last = ctx + (m1 - 1) / rep;
  const AttnSpan span = attn_span(a, first, last);
  const int32_t* table = a.table + (long long)r * a.stride;
  const int tiles = (span.n + BLK_BLOCKS - 1) / BLK_BLOCKS;
  auto at_of = [&](int i) { return (i < span.sinks ? i : span.from + i - span.sinks) * OPS_BLOCK; };   // first position of the list's block i

  s_ids[tid] = tid < span.n && last >= 0 ? table[at_of(tid) / OPS_BLOCK] : -1;
  static_assert(BLK_IDS == BLK_THREADS, "an id per thread");
  for (int k = tid; k < BLK_ROWS * (HD / 4); k += BLK_THREADS) {
    const int m = m0 + k / (HD / 4), d = k % (HD / 4) * 4;
    float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m < m1) q = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + (start + m / rep) * a.q_stride + (h * rep + m % rep) * HD + d);
    *reinterpret_cast<float4*>(s_f + S::Q + (k / (HD / 4)) * S::PITCH + d) = q;
  }
  __syncthreads();
  // a tile's keys or values; blocks behind the list, and those that are none, as zeros
  auto copy = [&](int to, const char* base, int j) {
    constexpr int CH = HD / 4;   // 16-byte pieces of a row
#pragma unroll 4
    for (int k = tid; k < BLK_KEYS * CH; k += BLK_THREADS) {
      const int key = k / CH, c = k % CH, i = j * BLK_BLOCKS + key / OPS_BLOCK;
      const int id = i < BLK_IDS ? s_ids[i] : i < span.n && last >= 0 ? table[at_of(i) / OPS_BLOCK] : -1;
      const bool there = (unsigned)id < (unsigned)a.pool.n_blocks;
      const char* src = base + (((long long)(there ? id : 0) * a.pool.Hkv + h) * OPS_BLOCK + key % OPS_BLOCK) * (HD * 4) + c * 16;
      const uint32_t dst = (uint32_t)__cvta_generic_to_shared(s_f + to + key * S::PITCH + c * 4);
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16u : 0u) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  copy(S::K, a.pool.k, 0);
  copy(S::V, a.pool.v, 0);

  const int rg = tid >> 4, c16 = tid & 15;   // rows R rg .. R rg + R - 1; keys c16 + 16 i, dims 4 c16 + 64 i
  constexpr int D = HD / 64;
  float m[R], l[R];
  float4 acc[R][D];
  int pos[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int mr = m0 + rg * R + i;
    pos[i] = mr < m1 ? ctx + mr / rep : -1;
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int d = 0; d < D; ++d) acc[i][d] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll 1
  for (int j = 0; j < tiles; ++j) {
    asm volatile("cp.async.wait_group 1;" ::: "memory");   // the keys (the values came after them)
    __syncthreads();
    float s[R][4];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[i][k] = 0.f;
#pragma unroll 2
    for (int d = 0; d < HD; d += 4) {
      float4 q[R], kk[4];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        q[i] = *reinterpret_cast<const float4*>(s_f + S::Q + (rg * R + i) * S::PITCH + d);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) kk[k] = *reinterpret_cast<const float4*>(s_f + S::K + (c16 + 16 * k) * S::PITCH + d);
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[i][k] = fmaf(q[i].x, kk[k].x, fmaf(q[i].y, kk[k].y, fmaf(q[i].z, kk[k].z, fmaf(q[i].w, kk[k].w, s[i][k]))));
    }
    __syncthreads();
    if (j + 1 < tiles) copy(S::K, a.pool.k, j + 1);
    else asm volatile("cp.async.commit_group;" ::: "memory");
    // softmax; a tile that some row does not see all of is masked
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float top = m[i];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        s[i][k] = attn_sees(a, at_of(j * BLK_BLOCKS + k) + c16, pos[i]) ? s[i][k] * a.qscale : -INFINITY;
        top = fmaxf(top, s[i][k]);
      }
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float base = top == -INFINITY ? 0.f : top, f = m[i] == -INFINITY ? 0.f : exp2f(m[i] - base);
      m[i] = top;
      l[i] *= f;
#pragma unroll
      for (int d = 0; d < D; ++d) { acc[i][d].x *= f; acc[i][d].y *= f; acc[i][d].z *= f; acc[i][d].w *= f; }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float p = exp2f(s[i][k] - base);
        l[i] += p;
        s_f[S::P + (rg * R + i) * S::P_PITCH + c16 + 16 * k] = p;
      }
    }
    asm volatile("cp.async.wait_group 1;" ::: "memory");   // the values (the next keys came after them)
    __syncthreads();
    const int p0 = at_of(j * BLK_BLOCKS), p3 = at_of(j * BLK_BLOCKS + BLK_BLOCKS - 1) + OPS_BLOCK - 1;
    if (p3 > last || (a.window > 0 && (p0 <= first - a.window || a.sinks > 0))) {   // what no row sees may be anything, and 0 x NaN is not 0
      for (int k = warp; k < BLK_KEYS; k += BLK_THREADS / 32) {
        const int at = at_of(j * BLK_BLOCKS + k / OPS_BLOCK) + k % OPS_BLOCK;
        if (at <= last && (a.window == 0 || at > first - a.window || at < a.sinks)) continue;
        for (int d = lane * 4; d < HD; d += 128) *reinterpret_cast<float4*>(s_f + S::V + k * S::PITCH + d) = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      __syncthreads();
    }
#pragma unroll 1
    for (int k = 0; k < BLK_KEYS; k += 4) {
      float4 p[R];
#pragma unroll
      for (int i = 0; i < R; ++i) p[i] = *reinterpret_cast<const float4*>(s_f + S::P + (rg * R + i) * S::P_PITCH + k);
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int d = 0; d < D; ++d) {
          const float4 v = *reinterpret_cast<const float4*>(s_f + S::V + (k + y) * S::PITCH + d * 64 + c16 * 4);
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const float w = y == 0 ? p[i].x : y == 1 ? p[i].y : y == 2 ? p[i].z : p[i].w;
            acc[i][d].x = fmaf(w, v.x, acc[i][d].x);
            acc[i][d].y = fmaf(w, v.y, acc[i][d].y);
            acc[i][d].z = fmaf(w, v.z, acc[i][d].z);
            acc[i][d].w = fmaf(w, v.w, acc[i][d].w);
          }
        }
    }
    __syncthreads();
    if (j + 1 < tiles) copy(S::V, a.pool.v, j + 1);
    else asm volatile("cp.async.commit_group;" ::: "memory");
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int i = 0; i < R; ++i) {
    float sum = l[i];
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    const int mr = m0 + rg * R + i;
    if (mr >= m1) continue;
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    float* dst = static_cast<float*>(a.out) + (start + mr / rep) * a.out_stride + (h * rep + mr % rep) * HD + c16 * 4;
#pragma unroll
    for (int d = 0; d < D; ++d) *reinterpret_cast<float4*>(dst + d * 64) = make_float4(acc[i][d].x * inv, acc[i][d].y * inv, acc[i][d].z * inv, acc[i][d].w * inv);
  }
}

template <int HD, int R>
static int blocks_run(const AttnArgs& a, void* stream) {
  const int64_t grid = ((int64_t)a.rows * a.pool.rep / (8 * R) + a.n) * a.pool.Hkv;
  return ops_launch(blink_attn_block_kernel<HD, R>, grid, BLK_THREADS, BlkShape<HD, R>::END * 4, stream, 0, a);
}

int attn_blocks(const AttnArgs& a, int sms, void* stream) {
  // 32 rows a CTA read the keys half as often as 16, but leave SMs without one where there are few rows
  const bool many = (int64_t)a.rows * a.pool.rep / 32 * a.pool.Hkv >= 2 * sms;
  if (a.pool.hd == 128) return many ? blocks_run<128, 4>(a, stream) : blocks_run<128, 2>(a, stream);
  return many ? blocks_run<64, 4>(a, stream) : blocks_run<64, 2>(a, stream);
}

}  // namespace blink
