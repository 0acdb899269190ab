// Attention over the paged cache through a sliding window and a few first tokens that stay visible: blink_window_attention.
//
//   row at position p sees key j <= p when j > p - window (window 0: every j) or j < sinks
//   o = sum_j softmax_j(q . k_j / sqrt(hd)) v_j,  zeros where nothing is seen
//
// Four ways: the two kernels here (attn_few with its join, attn_near), tiles on the tensor cores (ops_attn_tiles.cu) and 32-bit blocks
// (ops_attn_block.cu); which requests and calls take which stands at the entry point, with both sides measured.
//
// attn_few: requests of few rows (a token, a few drafts).  What bounds it: HBM, every visible key and value once.  (8B shape, a row each: 64 requests
// behind 5000 keys 196 us, 6.7 TB/s; 256 754 us, 7.0; one behind 120000 keys 82 us, 6.0.)  With more rows, instructions: 48 requests of 4 rows behind
// 2500 keys 92 us, 5.3 TB/s, of 8 rows 133.  (Tiles copied ahead into shared memory, which leaves registers to more rows, cost time at every number of rows:
// 5 rows 103 us, 127 so; it is not the loads that a warp waits for.)
// A unit is a request, a kv head and up to MR (query row, head) rows, its tiles are the visible blocks of 16 keys.  All tiles of all units
// stand in one sequence that is cut into equal runs, one per CTA, whatever the lengths; lengths are read on the device, so that a
// captured graph serves growing contexts.  A CTA's warps take its tiles in turn, straight from memory to registers in the layout of the
// matrix instructions: no shared memory and no barrier on the way, 8 KB in flight per warp.  A unit that a cut divides leaves one
// record (maximum, sum, weighted values) per CTA; a second kernel joins them in order, without atomics.
//
// bf16 with keys and values in the roles of the wide operand (m16n8k16: 16 keys x 8 rows for the scores, 16 dims x 8 rows
// for the output): eight rows fill an instruction, where rows as the wide operand would leave half to three quarters of it empty.
//   scores: lane (g, c) = (lane / 4, lane % 4) holds 16-byte pieces of keys g and g + 8; the order of the dims within a product is free,
//           so a piece of 8 dims serves two instructions, and the same piece of a query row is the other operand
//   output: probabilities become an operand with one movmatrix per 8 keys; values are read as rows and paired by key with byte permutes
// Probabilities are rounded to bf16 for the product with the values (as large an error as that of the output's own rounding);
// scores, maxima, sums and outputs are in 32 bits.  The maximum in use follows the largest score only when that has grown by more than 2^8.
#include <cooperative_groups.h>

#include <algorithm>
#include <cmath>

#include "ops_attention.cuh"

namespace blink {

constexpr int FEW_WARPS = 4, FEW_THREADS = FEW_WARPS * 32;
constexpr int FEW_MAX_CTAS = 640;    // of a launch; the records are laid out for so many
constexpr int FEW_MIN_TILES = 4;     // of a CTA's run, while there are any
constexpr int FEW_UNIT_TILES = 4;    // what a unit costs beside its tiles, in tiles
constexpr int JOIN_THREADS = 256, JOIN_FEW = 4;   // parts that the CTA in whose run a unit begins joins by itself
// Calls that take all requests to the tiles (see the entry point): rows (of a kv head) of the longest, keys that a row sees, at most.
constexpr int ALL_ROWS = 8, ALL_SHORT = 1536, ALL_KEYS = 8192, ALL_KEYS_32 = 256;

// What the join needs of a unit that was cut.  A CTA leaves two: of the unit in which its run begins, and of the one in which it ends.
struct FewCut {
  int first, parts;      // the CTA in whose run it begins; records, that CTA's second and the first of each of the following ones.  0: none
  int row, m0, m1, h;    // first row of the request, rows (of row * rep + head) m0 .. m1 - 1, kv head
};

// workspace: status, cuts [FEW_MAX_CTAS][2], (maximum, sum) [2 * FEW_MAX_CTAS][MR], values [2 * FEW_MAX_CTAS][MR][HD]
__host__ __device__ constexpr size_t few_ml_at() { return ATTN_STATUS_BYTES + (sizeof(FewCut) * 2 * FEW_MAX_CTAS + 255) / 256 * 256; }
__host__ __device__ constexpr size_t few_acc_at(int mr) { return few_ml_at() + (size_t)2 * FEW_MAX_CTAS * mr * 8; }
__host__ __device__ constexpr size_t few_bytes(int mr, int hd) { return few_acc_at(mr) + (size_t)2 * FEW_MAX_CTAS * mr * hd * 4; }

__device__ __forceinline__ uint4 few_ld(const char* p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
  return r;
}
__device__ __forceinline__ void few_mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t few_transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Rows m0 .. m1 - 1 of a unit in one warp: queries, maxima, sums, weighted values.
template <int HD, int NT>
struct FewBf16 {
  static constexpr int MR = 8 * NT, CH = HD / 32, U = HD / 64, PITCH = HD + 4;
  // 32 rows: the queries stay in shared memory, in fragments (a 16-byte read for two instructions), or registers spill (48 requests of 2500 keys, 8 rows each:
  // 157 us with them in registers, 131 so; 24 rows 107 and 110)
  static constexpr bool Q_SHARED = NT >= 4;
  static constexpr int Q_BYTES = Q_SHARED ? NT * CH * 512 : 0;
  uint4 q[Q_SHARED ? 1 : NT][Q_SHARED ? 1 : CH];
  const uint4* q_at;
  float acc[NT][U][4][4], m[NT][2], l[NT][2];
  int pos[NT][2];
  int live;   // instructions' worth of rows in use

  // (Q_SHARED: between two barriers; the warps take a share of the fragments each)
  __device__ __forceinline__ void begin(const AttnArgs& a, const AttnReq& r, int h, int m0, int m1, char* s_q) {
    const int g = (threadIdx.x & 31) >> 2, c = threadIdx.x & 3, rep = a.pool.rep;
    q_at = reinterpret_cast<const uint4*>(s_q) + (threadIdx.x & 31);
    live = (m1 - m0 + 7) / 8;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int mq = m0 + nt * 8 + g;
      const char* src = static_cast<const char*>(a.q) + ((r.start + (mq < m1 ? mq / rep : 0)) * a.q_stride + (h * rep + (mq < m1 ? mq % rep : 0)) * HD + 8 * c) * 2;
#pragma unroll
      for (int k = 0; k < CH; ++k) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if constexpr (Q_SHARED) {
          if (k % FEW_WARPS != (int)(threadIdx.x >> 5)) continue;
          if (mq < m1) x = *reinterpret_cast<const uint4*>(src + k * 64);
          reinterpret_cast<uint4*>(s_q)[(nt * CH + k) * 32 + (threadIdx.x & 31)] = x;
        } else {
          if (mq < m1) x = *reinterpret_cast<const uint4*>(src + k * 64);
          q[nt][k] = x;
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int mr = m0 + nt * 8 + 2 * c + i;
        pos[nt][i] = mr < m1 ? r.ctx + mr / rep : -1;
        m[nt][i] = -INFINITY;
        l[nt][i] = 0.f;
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[nt][u][t][i] = 0.f;
    }
  }

  // Block b of the request; k, v: its keys and values of this head, null: zeros.  edge: some row does not see all of it; first, last: positions
  // of the first and the last row.
  __device__ __forceinline__ void tile(const AttnArgs& a, int b, const char* k, const char* v, bool edge, int first, int last) {
    if constexpr (NT >= 4) {
      if (live == 4) return tile_of<4>(a, b, k, v, edge, first, last);
    }
    if constexpr (NT >= 3) {
      if (live == 3) return tile_of<3>(a, b, k, v, edge, first, last);
    }
    if constexpr (NT >= 2) {
      if (live == 2) return tile_of<2>(a, b, k, v, edge, first, last);
    }
    tile_of<1>(a, b, k, v, edge, first, last);
  }
  // (code of its own for each number of instructions that a unit's rows take: conditions around them cost registers, and spills)
  template <int LIVE>
  __device__ __forceinline__ void tile_of(const AttnArgs& a, int b, const char* k, const char* v, bool edge, int first, int last) {
    const int g = (threadIdx.x & 31) >> 2, c = threadIdx.x & 3;
    uint4 kk[2][CH], vv[U][4];
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int x = 0; x < CH; ++x) kk[i][x] = k ? few_ld(k + (g + 8 * i) * (HD * 2) + x * 64 + c * 16) : zero;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) vv[u][i] = v ? few_ld(v + (2 * c + (i & 1) + 8 * (i >> 1)) * (HD * 2) + u * 128 + g * 16) : zero;
    float s[LIVE][4];
#pragma unroll
    for (int nt = 0; nt < LIVE; ++nt) {
      s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
      for (int x = 0; x < CH; ++x) {
        uint4 y;
        if constexpr (Q_SHARED) y = q_at[(nt * CH + x) * 32];
        else y = q[nt][x];
        few_mma(s[nt], kk[0][x].x, kk[1][x].x, kk[0][x].y, kk[1][x].y, y.x, y.y);
        few_mma(s[nt], kk[0][x].z, kk[1][x].z, kk[0][x].w, kk[1][x].w, y.z, y.w);
      }
    }
    const int key = b * OPS_BLOCK + g;
    bool grown = false;
#pragma unroll
    for (int nt = 0; nt < LIVE; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // i: key g + 8 * (i / 2), row 2 c + i % 2
        s[nt][i] *= a.qscale;
        if (edge && !attn_sees(a, key + 8 * (i >> 1), pos[nt][i & 1])) s[nt][i] = -INFINITY;
        grown |= s[nt][i] > m[nt][i & 1] + 8.f;
      }
    if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
      for (int nt = 0; nt < LIVE; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float x = fmaxf(s[nt][i], s[nt][i + 2]);
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
          x = fmaxf(x, m[nt][i]);
          const float f = x == -INFINITY ? 1.f : attn_ex2(m[nt][i] - x);
          m[nt][i] = x;
          l[nt][i] *= f;
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              acc[nt][u][t][i] *= f;
              acc[nt][u][t][i + 2] *= f;
            }
        }
    }
    uint32_t p[LIVE][2];
#pragma unroll
    for (int nt = 0; nt < LIVE; ++nt) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[nt][i] = attn_ex2(s[nt][i] - (m[nt][i & 1] == -INFINITY ? 0.f : m[nt][i & 1]));
        l[nt][i & 1] += s[nt][i];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const __nv_bfloat162 x = __floats2bfloat162_rn(s[nt][2 * i], s[nt][2 * i + 1]);
        p[nt][i] = few_transposed(*reinterpret_cast<const uint32_t*>(&x));
      }
    }
    if (edge) {   // what no row sees may be anything: 0 x NaN
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = b * OPS_BLOCK + 2 * c + (i & 1) + 8 * (i >> 1);
        const bool seen = at <= last && (a.window == 0 || at > first - a.window || at < a.sinks);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (!seen) vv[u][i] = zero;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t x[4] = {t == 0 ? vv[u][0].x : t == 1 ? vv[u][0].y : t == 2 ? vv[u][0].z : vv[u][0].w,
                               t == 0 ? vv[u][1].x : t == 1 ? vv[u][1].y : t == 2 ? vv[u][1].z : vv[u][1].w,
                               t == 0 ? vv[u][2].x : t == 1 ? vv[u][2].y : t == 2 ? vv[u][2].z : vv[u][2].w,
                               t == 0 ? vv[u][3].x : t == 1 ? vv[u][3].y : t == 2 ? vv[u][3].z : vv[u][3].w};
        const uint32_t a0 = __byte_perm(x[0], x[1], 0x5410), a1 = __byte_perm(x[0], x[1], 0x7632), a2 = __byte_perm(x[2], x[3], 0x5410),
                       a3 = __byte_perm(x[2], x[3], 0x7632);
#pragma unroll
        for (int nt = 0; nt < LIVE; ++nt) few_mma(acc[nt][u][t], a0, a1, a2, a3, p[nt][0], p[nt][1]);
      }
  }

  // To shared memory: values [row][PITCH], (maximum, sum) [row].
  __device__ __forceinline__ void leave(float* to, float2* ml) {
    const int g = (threadIdx.x & 31) >> 2, c = threadIdx.x & 3;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x = l[nt][i];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        const int row = nt * 8 + 2 * c + i;
        if (g == 0) ml[row] = make_float2(m[nt][i], x);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float* dst = to + row * PITCH + u * 64 + g * 8;
          *reinterpret_cast<float4*>(dst) = make_float4(acc[nt][u][0][i], acc[nt][u][0][i + 2], acc[nt][u][1][i], acc[nt][u][1][i + 2]);
          *reinterpret_cast<float4*>(dst + 4) = make_float4(acc[nt][u][2][i], acc[nt][u][2][i + 2], acc[nt][u][3][i], acc[nt][u][3][i + 2]);
        }
      }
  }
};

// The same in 32 bits on the CUDA cores: eight lanes share a key (lane s of them has dims 4 s + 32 j ..), a warp four keys at a time.
template <int HD>
struct FewFp32 {
  static constexpr int MR = HD == 128 ? 4 : 8, J = HD / 32, PITCH = HD + 4;
  static constexpr bool Q_SHARED = false;
  static constexpr int Q_BYTES = 0;
  float4 q[MR][J], acc[MR][J];
  float m[MR], l[MR];
  int pos[MR];

  __device__ __forceinline__ void begin(const AttnArgs& a, const AttnReq& r, int h, int m0, int m1, char*) {
    const int s = threadIdx.x & 7, rep = a.pool.rep;
#pragma unroll
    for (int i = 0; i < MR; ++i) {
      const int mq = m0 + i;
      const float* src = static_cast<const float*>(a.q) + (r.start + (mq < m1 ? mq / rep : 0)) * a.q_stride + (h * rep + (mq < m1 ? mq % rep : 0)) * HD + 4 * s;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        q[i][j] = mq < m1 ? *reinterpret_cast<const float4*>(src + 32 * j) : make_float4(0.f, 0.f, 0.f, 0.f);
        acc[i][j] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      pos[i] = mq < m1 ? r.ctx + mq / rep : -1;
      m[i] = -INFINITY;
      l[i] = 0.f;
    }
  }

  __device__ __forceinline__ void tile(const AttnArgs& a, int b, const char* k, const char* v, bool edge, int first, int last) {
    const int s = threadIdx.x & 7, kg = (threadIdx.x & 31) >> 3;
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    auto ld = [&](const char* p, int key, int j) {
      if (!p) return zero;
      const uint4 x = few_ld(p + (key * HD + 4 * s + 32 * j) * 4);
      return make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w));
    };
    float sc[4][MR];
    bool grown = false;
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      float4 x[J];
#pragma unroll
      for (int j = 0; j < J; ++j) x[j] = ld(k, it * 4 + kg, j);
#pragma unroll
      for (int i = 0; i < MR; ++i) {
        float t = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) t = fmaf(q[i][j].x, x[j].x, fmaf(q[i][j].y, x[j].y, fmaf(q[i][j].z, x[j].z, fmaf(q[i][j].w, x[j].w, t))));
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
        t *= a.qscale;
        if (edge && !attn_sees(a, b * OPS_BLOCK + it * 4 + kg, pos[i])) t = -INFINITY;
        sc[it][i] = t;
        grown |= t > m[i] + 8.f;
      }
    }
    if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
      for (int i = 0; i < MR; ++i) {
        float x = fmaxf(fmaxf(sc[0][i], sc[1][i]), fmaxf(sc[2][i], sc[3][i]));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
        x = fmaxf(fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16)), m[i]);
        const float f = x == -INFINITY ? 1.f : exp2f(m[i] - x);
        m[i] = x;
        l[i] *= f;
#pragma unroll
        for (int j = 0; j < J; ++j) { acc[i][j].x *= f; acc[i][j].y *= f; acc[i][j].z *= f; acc[i][j].w *= f; }
      }
    }
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int at = b * OPS_BLOCK + it * 4 + kg;
      const bool seen = !edge || (at <= last && (a.window == 0 || at > first - a.window || at < a.sinks));   // what no row sees may be anything
      float4 x[J];
#pragma unroll
      for (int j = 0; j < J; ++j) {
        x[j] = ld(v, it * 4 + kg, j);
        if (!seen) x[j] = zero;
      }
#pragma unroll
      for (int i = 0; i < MR; ++i) {
        const float p = exp2f(sc[it][i] - (m[i] == -INFINITY ? 0.f : m[i]));
        l[i] += p;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          acc[i][j].x = fmaf(p, x[j].x, acc[i][j].x);
          acc[i][j].y = fmaf(p, x[j].y, acc[i][j].y);
          acc[i][j].z = fmaf(p, x[j].z, acc[i][j].z);
          acc[i][j].w = fmaf(p, x[j].w, acc[i][j].w);
        }
      }
    }
  }

  __device__ __forceinline__ void leave(float* to, float2* ml) {
    const int lane = threadIdx.x & 31, s = lane & 7;
#pragma unroll
    for (int i = 0; i < MR; ++i) {
      auto both = [&](float x) {
        x += __shfl_xor_sync(0xffffffffu, x, 8);
        return x + __shfl_xor_sync(0xffffffffu, x, 16);
      };
      const float sum = both(l[i]);
      if (lane == 0) ml[i] = make_float2(m[i], sum);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const float4 x = make_float4(both(acc[i][j].x), both(acc[i][j].y), both(acc[i][j].z), both(acc[i][j].w));
        if (lane < 8) *reinterpret_cast<float4*>(to + i * PITCH + 4 * s + 32 * j) = x;
      }
    }
  }
};

__device__ __forceinline__ void few_store(__nv_bfloat16* p, float4 x) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ void few_store(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }

// Groups of MR rows of a request, and tiles of each (the same number for all of them, so that a place in the sequence is found by division;
// a group that has fewer leaves the rest out).  A unit's start and end cost as much as some tiles and count as such, behind its
// tiles: without them CTAs that got many short units were the last (200 rows of 20 to 5000 keys, cold: 148 us, 105 with them).
struct FewShape {
  int groups, tiles;
};
template <int MR>
__device__ __forceinline__ FewShape few_shape(const AttnArgs& a, const AttnReq& r) {
  if (r.rows == 0 || r.rows > a.few) return {0, 0};
  const long long m = (long long)r.rows * a.pool.rep;
  const int groups = (int)((m + MR - 1) / MR), last = r.ctx + r.rows - 1;
  if (groups == 1) return {1, attn_span(a, r.ctx, last).n + FEW_UNIT_TILES};
  int tiles = attn_span(a, r.ctx, last).n;   // every group's are among these
  if (a.window > 0) tiles = min(tiles, (a.sinks + OPS_BLOCK - 1) / OPS_BLOCK + (int)min(0x7ffff000ll, (long long)a.window + MR / a.pool.rep + 1) / OPS_BLOCK + 2);
  return {groups, tiles + FEW_UNIT_TILES};
}

template <typename T, int HD, typename W, int CTAS>
__global__ void __launch_bounds__(FEW_THREADS, CTAS) blink_attn_few_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int MR = W::MR, PITCH = W::PITCH;
  extern __shared__ __align__(16) char s_dyn[];
  float* s_acc = reinterpret_cast<float*>(s_dyn);                                        // [FEW_WARPS][MR][PITCH]
  float2* s_ml = reinterpret_cast<float2*>(s_acc + FEW_WARPS * MR * PITCH);              // [FEW_WARPS][MR]
  char* s_q = reinterpret_cast<char*>(s_ml + FEW_WARPS * MR);
  long long* s_pre = reinterpret_cast<long long*>(s_q + W::Q_BYTES);                     // [n + 1] tiles before a request
  int2* s_len = reinterpret_cast<int2*>(s_pre + a.n + 1);                                // [n] first row, kv_len
  __shared__ long long s_warp[FEW_WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  ops_wait();
  if (blockIdx.x == 0 && tid == 0) {
    reinterpret_cast<int*>(a.ws)[0] = 0;
    reinterpret_cast<int*>(a.ws)[1] = 0;   // units that the tiles' CTAs have taken from the counter
    __threadfence();
  }
  ops_next();

  // the sequence of tiles: a run of requests per thread
  const int each = (a.n + FEW_THREADS - 1) / FEW_THREADS;
  const int r0 = min(a.n, tid * each), r1 = min(a.n, r0 + each);
  long long mine = 0;
  for (int r = r0; r < r1; ++r) {
    const int start = a.row_start[r], kv = a.kv_len[r];
    const FewShape s = few_shape<MR>(a, attn_req(a, start, a.row_start[r + 1], kv));
    s_len[r] = make_int2(start, kv);
    s_pre[r] = mine;
    mine += (long long)s.groups * a.pool.Hkv * s.tiles;
  }
  long long x = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  long long total = 0;
#pragma unroll
  for (int w = 0; w < FEW_WARPS; ++w) {
    if (w < warp) x += s_warp[w];
    total += s_warp[w];
  }
  for (int r = r0; r < r1; ++r) s_pre[r] += x - mine;
  if (tid == 0) s_pre[a.n] = total;
  __syncthreads();

  const long long per = max((total + gridDim.x - 1) / gridDim.x, (long long)FEW_MIN_TILES);
  long long at = blockIdx.x * per;
  const long long end = min(total, at + per);
  FewCut begins = {}, ends = {};
  int r = 0;
  if (at < end) {
    int hi = a.n;
    while (hi - r > 1) {   // the last request that begins at or before it
      const int mid = (r + hi) >> 1;
      if (s_pre[mid] <= at) r = mid; else hi = mid;
    }
  }
  W w;
  while (at < end) {
    while (s_pre[r + 1] <= at) ++r;
    const AttnReq req = attn_req(a, s_len[r].x, r + 1 < a.n ? s_len[r + 1].x : a.row_start[a.n], s_len[r].y);
    const FewShape shape = few_shape<MR>(a, req);
    const long long off = at - s_pre[r];
    const int unit = (int)(off / shape.tiles), t0 = (int)(off - (long long)unit * shape.tiles);
    const int t1 = (int)min((long long)shape.tiles, t0 + (end - at));
    const int group = unit / a.pool.Hkv, h = unit - group * a.pool.Hkv;
    const int m0 = group * MR, m1 = min(req.rows * a.pool.rep, m0 + MR);
    const int first = req.ctx + m0 / a.pool.rep, last = req.ctx + (m1 - 1) / a.pool.rep;
    const AttnSpan span = attn_span(a, first, last);
    const int stop = min(t1, span.n);
    if (t0 >= span.n) {   // nothing of it is left
      at += t1 - t0;
      continue;
    }
    const int32_t* table = a.table + (long long)r * a.stride;

    auto block_of = [&](int t) { return t < span.sinks ? t : span.from + t - span.sinks; };
    int id = -1;   // of the warp's tile number `lane`, of 32 at a time
    if (t0 + warp + FEW_WARPS * lane < stop && last >= 0) id = table[block_of(t0 + warp + FEW_WARPS * lane)];
    w.begin(a, req, h, m0, m1, s_q);   // (the barrier before it: that behind the tiles of the segment before)
    if constexpr (W::Q_SHARED) __syncthreads();
    int i = 0;
    for (int t = t0 + warp; t < stop; t += FEW_WARPS, ++i) {
      if (i == 32) {
        i = 0;
        id = t + FEW_WARPS * lane < stop && last >= 0 ? table[block_of(t + FEW_WARPS * lane)] : -1;
      }
      const int b = block_of(t), block = __shfl_sync(0xffffffffu, id, i);
      const bool there = (unsigned)block < (unsigned)a.pool.n_blocks;
      const long long tile = ((long long)block * a.pool.Hkv + h) * (OPS_BLOCK * HD * (int)sizeof(T));
      const int k0 = b * OPS_BLOCK, k1 = k0 + OPS_BLOCK - 1;
      const bool edge = k1 > first || (a.window > 0 && k0 <= last - a.window && k1 >= a.sinks);
      w.tile(a, b, there ? a.pool.k + tile : nullptr, there ? a.pool.v + tile : nullptr, edge, first, last);
    }
    __syncthreads();   // (what was left there for the segment before has been read)
    w.leave(s_acc + warp * MR * PITCH, s_ml + warp * MR);
    __syncthreads();
    const bool whole = t0 == 0 && t1 >= span.n;
    const size_t rec = 2 * blockIdx.x + (t0 == 0 ? 1 : 0);
    float2* rec_ml = reinterpret_cast<float2*>(a.ws + few_ml_at()) + rec * MR;
    float* rec_acc = reinterpret_cast<float*>(a.ws + few_acc_at(MR)) + rec * MR * HD;
    for (int k = tid; k < (m1 - m0) * (HD / 4); k += FEW_THREADS) {
      const int row = k / (HD / 4), d = (k - row * (HD / 4)) * 4;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int y = 0; y < FEW_WARPS; ++y) M = fmaxf(M, s_ml[y * MR + row].x);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int y = 0; y < FEW_WARPS; ++y) {
        const float2 ml = s_ml[y * MR + row];
        const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M);
        const float4 z = *reinterpret_cast<const float4*>(s_acc + (y * MR + row) * PITCH + d);
        L = fmaf(ml.y, f, L);
        o.x = fmaf(z.x, f, o.x); o.y = fmaf(z.y, f, o.y); o.z = fmaf(z.z, f, o.z); o.w = fmaf(z.w, f, o.w);
      }
      if (whole) {
        const float inv = L > 0.f ? 1.f / L : 0.f;
        const int mr = m0 + row;
        few_store(static_cast<T*>(a.out) + (req.start + mr / a.pool.rep) * a.out_stride + (h * a.pool.rep + mr % a.pool.rep) * HD + d,
                  make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
      } else {
        *reinterpret_cast<float4*>(rec_acc + row * HD + d) = o;
        if (d == 0) rec_ml[row] = make_float2(M, L);
      }
    }
    if (!whole) {
      auto runs = [&](long long x) { return per < (1ll << 30) ? (int)((unsigned)x / (unsigned)per) : (int)(x / per); };   // (x: not much above per, or a unit's tiles)
      const int before = t0 == 0 ? 0 : runs(t0 + per - 1);   // CTAs before this one that have a part
      const FewCut cut = {(int)blockIdx.x - before, before + runs(at - blockIdx.x * per + span.n - t0 - 1) + 1, req.start, m0, m1, h};
      if (t0 == 0) ends = cut; else begins = cut;
    }
    at += t1 - t0;
  }
  if (tid == 0) {
    FewCut* cuts = reinterpret_cast<FewCut*>(a.ws + ATTN_STATUS_BYTES) + 2 * blockIdx.x;
    cuts[0] = begins;
    cuts[1] = ends;
  }
}

// The units that were cut: m = max m_i, l = sum l_i 2^(m_i - m), o = sum o_i 2^(m_i - m) / l over a row's parts.  The rows of a unit are dealt to the CTAs
// whose runs it spans (as many as there are parts; up to JOIN_FEW, which many units have, one CTA has all of them, instead of two units one after the
// other), a row's parts to warps, and these joined in order.  Latency: 2 to 3 us behind a batch.
// (With a CTA per unit: three requests of 2 to 4 rows behind 2000 keys 26.5 us, 14.7 so (a cluster each takes 12); one row behind 30000 keys 33.5 and 28.  All dealt out: 64 rows behind 600 keys
// 33.9, 31.4 so.)
template <typename T, int HD, int MR>
__global__ void __launch_bounds__(JOIN_THREADS) blink_attn_join_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int WARPS = JOIN_THREADS / 32, V = HD / 32;   // values of a row per lane
  __shared__ float s_acc[WARPS][HD];
  __shared__ float2 s_ml[WARPS];
  ops_next();
  ops_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float2* ml = reinterpret_cast<const float2*>(a.ws + few_ml_at());
  const float* acc = reinterpret_cast<const float*>(a.ws + few_acc_at(MR));
  const FewCut* cuts = reinterpret_cast<const FewCut*>(a.ws + ATTN_STATUS_BYTES) + 2 * blockIdx.x;
  const FewCut both[2] = {cuts[0], cuts[1]};
#pragma unroll 1
  for (int e = 0; e < 2; ++e) {
    const FewCut cut = e ? both[1] : both[0];
    if (cut.parts == 0) continue;
    const int hands = cut.parts > JOIN_FEW ? cut.parts : 1, mine_first = (int)blockIdx.x - cut.first;   // rows mine_first, mine_first + hands, ..
    const int rows = hands == 1 ? (mine_first == 0 ? cut.m1 - cut.m0 : 0) : (cut.m1 - cut.m0 - mine_first + hands - 1) / hands;
    if (rows <= 0) continue;
    const int share = rows >= WARPS ? 1 : WARPS / rows;   // warps of a row
    const int at_once = WARPS / share;                     // rows at a time
    for (int r0 = 0; r0 < rows; r0 += at_once) {
      const int r = r0 + warp / share, part = warp % share, row = mine_first + r * hands;
      const bool mine = warp / share < at_once && r < rows;
      float M = -INFINITY, L = 0.f, o[V];
#pragma unroll
      for (int v = 0; v < V; ++v) o[v] = 0.f;
      auto record = [&](int p) { return (size_t)(2 * (cut.first + p) + (p == 0 ? 1 : 0)) * MR + row; };
      if (mine) {
        for (int p = part + share * lane; p < cut.parts; p += share * 32) M = fmaxf(M, ml[record(p)].x);
#pragma unroll
        for (int d = 16; d; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
#pragma unroll 4
        for (int p = part; p < cut.parts; p += share) {
          const float2 x = ml[record(p)];
          const float f = x.x == -INFINITY ? 0.f : exp2f(x.x - M);
          const float* z = acc + record(p) * HD + lane * V;
          L = fmaf(x.y, f, L);
          if constexpr (V == 4) {
            const float4 y = *reinterpret_cast<const float4*>(z);
            o[0] = fmaf(y.x, f, o[0]); o[1] = fmaf(y.y, f, o[1]); o[2] = fmaf(y.z, f, o[2]); o[3] = fmaf(y.w, f, o[3]);
          } else {
            const float2 y = *reinterpret_cast<const float2*>(z);
            o[0] = fmaf(y.x, f, o[0]); o[1] = fmaf(y.y, f, o[1]);
          }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) s_acc[warp][lane * V + v] = o[v];
        if (lane == 0) s_ml[warp] = make_float2(M, L);
      }
      __syncthreads();
      if (mine && part == 0) {
        float top = -INFINITY, sum = 0.f;
        for (int k = 0; k < share; ++k) top = fmaxf(top, s_ml[warp + k].x);
#pragma unroll
        for (int v = 0; v < V; ++v) o[v] = 0.f;
        for (int k = 0; k < share; ++k) {
          const float2 x = s_ml[warp + k];
          const float f = x.x == -INFINITY ? 0.f : exp2f(x.x - top);
          sum = fmaf(x.y, f, sum);
#pragma unroll
          for (int v = 0; v < V; ++v) o[v] = fmaf(s_acc[warp + k][lane * V + v], f, o[v]);
        }
        const float inv = sum > 0.f ? 1.f / sum : 0.f;
        const int mr = cut.m0 + row;
        T* dst = static_cast<T*>(a.out) + (cut.row + mr / a.pool.rep) * a.out_stride + (cut.h * a.pool.rep + mr % a.pool.rep) * HD + lane * V;
        if constexpr (V == 4) few_store(dst, make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv));
        else if constexpr (sizeof(T) == 2) *reinterpret_cast<__nv_bfloat162*>(dst) = __floats2bfloat162_rn(o[0] * inv, o[1] * inv);
        else *reinterpret_cast<float2*>(dst) = make_float2(o[0] * inv, o[1] * inv);
      }
      __syncthreads();
    }
  }
}

// The same for few units and short contexts, where latency is all there is: a cluster of CTAs per unit, which share its tiles and join their records
// through distributed shared memory.  One kernel instead of two, no sequence to be added up first: a row of 1028 keys of the 8B shape
// 7.5 us, 12.3 with the kernels above (some 3 us are the launch, the rest loads that wait for one another: lengths, block ids, keys).
// a.few as there; `groups` clusters per (request, kv head), a group of rows each, or every groups-th where there are more.
template <typename T, int HD, typename W>
__global__ void __launch_bounds__(FEW_THREADS) blink_attn_near_kernel(const __grid_constant__ AttnArgs a, const int groups) {
  namespace cg = cooperative_groups;
  constexpr int MR = W::MR, PITCH = W::PITCH;
  extern __shared__ __align__(16) char s_dyn[];
  float* s_acc = reinterpret_cast<float*>(s_dyn);                             // [FEW_WARPS][MR][PITCH], then this CTA's record in the first of them
  float2* s_ml = reinterpret_cast<float2*>(s_acc + FEW_WARPS * MR * PITCH);   // [FEW_WARPS][MR]
  float2* s_rec = s_ml + FEW_WARPS * MR;                                      // [MR] maxima and sums of the record
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
  ops_wait();
  if (blockIdx.x == 0 && tid == 0) {
    reinterpret_cast<int*>(a.ws)[0] = 0;
    reinterpret_cast<int*>(a.ws)[1] = 0;   // units that the tiles' CTAs have taken from the counter
    __threadfence();
  }
  ops_next();
  const int unit = (int)blockIdx.x / ctas, h = unit % a.pool.Hkv, r = unit / a.pool.Hkv / groups, g0 = unit / a.pool.Hkv % groups;
  const AttnReq req = attn_req(a, a.row_start[r], a.row_start[r + 1], a.kv_len[r]);
  if (req.rows == 0 || req.rows > a.few) return;   // (the whole cluster)
  const int32_t* table = a.table + (long long)r * a.stride;
  W w;
  for (int m0 = g0 * MR; m0 < req.rows * a.pool.rep; m0 += groups * MR) {
    const int m1 = min(req.rows * a.pool.rep, m0 + MR);
    const int first = req.ctx + m0 / a.pool.rep, last = req.ctx + (m1 - 1) / a.pool.rep;
    const AttnSpan span = attn_span(a, first, last);
    auto block_of = [&](int t) { return t < span.sinks ? t : span.from + t - span.sinks; };
    const int t0 = rank * FEW_WARPS + warp, step = ctas * FEW_WARPS;   // the warp's tiles
    int id = -1;   // of its tile number `lane`, of 32 at a time
    if (t0 + step * lane < span.n && last >= 0) id = table[block_of(t0 + step * lane)];
    w.begin(a, req, h, m0, m1, reinterpret_cast<char*>(s_rec + MR));
    if constexpr (W::Q_SHARED) __syncthreads();
    int i = 0;
    for (int t = t0; t < span.n; t += step, ++i) {
      if (i == 32) {
        i = 0;
        id = t + step * lane < span.n && last >= 0 ? table[block_of(t + step * lane)] : -1;
      }
      const int b = block_of(t), block = __shfl_sync(0xffffffffu, id, i);
      const bool there = (unsigned)block < (unsigned)a.pool.n_blocks;
      const long long tile = ((long long)block * a.pool.Hkv + h) * (OPS_BLOCK * HD * (int)sizeof(T));
      const int k0 = b * OPS_BLOCK, k1 = k0 + OPS_BLOCK - 1;
      const bool edge = k1 > first || (a.window > 0 && k0 <= last - a.window && k1 >= a.sinks);
      w.tile(a, b, there ? a.pool.k + tile : nullptr, there ? a.pool.v + tile : nullptr, edge, first, last);
    }
    w.leave(s_acc + warp * MR * PITCH, s_ml + warp * MR);
    __syncthreads();
    // the warps' parts -> the CTA's record, in the place of the first (each thread reads what it writes)
    const int items = (m1 - m0) * (HD / 4);
    for (int k = tid; k < items; k += FEW_THREADS) {
      const int row = k / (HD / 4), d = (k - row * (HD / 4)) * 4;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int y = 0; y < FEW_WARPS; ++y) M = fmaxf(M, s_ml[y * MR + row].x);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int y = 0; y < FEW_WARPS; ++y) {
        const float2 ml = s_ml[y * MR + row];
        const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M);
        const float4 z = *reinterpret_cast<const float4*>(s_acc + (y * MR + row) * PITCH + d);
        L = fmaf(ml.y, f, L);
        o.x = fmaf(z.x, f, o.x); o.y = fmaf(z.y, f, o.y); o.z = fmaf(z.z, f, o.z); o.w = fmaf(z.w, f, o.w);
      }
      *reinterpret_cast<float4*>(s_acc + row * PITCH + d) = o;
      if (d == 0) s_rec[row] = make_float2(M, L);
    }
    cluster.sync();
    // the CTAs' records -> the output, a share of it by each CTA
    for (int k = rank * FEW_THREADS + tid; k < items; k += ctas * FEW_THREADS) {
      const int row = k / (HD / 4), d = (k - row * (HD / 4)) * 4;
      float M = -INFINITY, L = 0.f;
#pragma unroll 4
      for (int c = 0; c < ctas; ++c) M = fmaxf(M, cluster.map_shared_rank(s_rec, c)[row].x);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int c = 0; c < ctas; ++c) {
        const float2 ml = cluster.map_shared_rank(s_rec, c)[row];
        const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M);
        const float4 z = *reinterpret_cast<const float4*>(cluster.map_shared_rank(s_acc, c) + row * PITCH + d);
        L = fmaf(ml.y, f, L);
        o.x = fmaf(z.x, f, o.x); o.y = fmaf(z.y, f, o.y); o.z = fmaf(z.z, f, o.z); o.w = fmaf(z.w, f, o.w);
      }
      const float inv = L > 0.f ? 1.f / L : 0.f;
      const int mr = m0 + row;
      few_store(static_cast<T*>(a.out) + (req.start + mr / a.pool.rep) * a.out_stride + (h * a.pool.rep + mr % a.pool.rep) * HD + d,
                make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    }
    cluster.sync();   // (the records have been read)
  }
}

template <typename T, int HD, typename W, int CTAS>
static int few_run(const AttnArgs& a, int sms, void* stream) {
  if (a.near_ctas > 0) {
    const int64_t ctas = (int64_t)a.n * a.pool.Hkv * a.near_groups * a.near_ctas;
    const size_t need = (size_t)FEW_WARPS * W::MR * (W::PITCH * 4 + 8) + W::MR * 8 + W::Q_BYTES;
    return ops_launch(blink_attn_near_kernel<T, HD, W>, ctas, FEW_THREADS, need, stream, a.near_ctas, a, a.near_groups);
  }
  const size_t unit = (size_t)FEW_WARPS * W::MR * (W::PITCH * 4 + 8) + W::Q_BYTES;
  const OpsShared smem(unit + (size_t)(a.n + 1) * 16, unit + (size_t)(OPS_MAX_REQUESTS + 1) * 16);
  const int grid = sms * CTAS < FEW_MAX_CTAS ? sms * CTAS : FEW_MAX_CTAS;
  const int rc = ops_launch(blink_attn_few_kernel<T, HD, W, CTAS>, grid, FEW_THREADS, smem, stream, 0, a);
  if (rc != BLINK_OK) return rc;
  return ops_launch(blink_attn_join_kernel<T, HD, W::MR>, grid, JOIN_THREADS, 0, stream, 0, a);
}

template <int HD>
static int few_bf16(const AttnArgs& a, int nt, int sms, void* stream) {
  if (nt == 1) return few_run<__nv_bfloat16, HD, FewBf16<HD, 1>, 4>(a, sms, stream);
  if (nt == 2) return few_run<__nv_bfloat16, HD, FewBf16<HD, 2>, 3>(a, sms, stream);
  if (nt == 3) return few_run<__nv_bfloat16, HD, FewBf16<HD, 3>, 2>(a, sms, stream);
  return few_run<__nv_bfloat16, HD, FewBf16<HD, 4>, 2>(a, sms, stream);
}

// Instructions' worth of rows (eight each) that a unit of the few-rows kernel holds.
static int few_nt(int64_t m_rows) { return m_rows <= 8 ? 1 : m_rows <= 16 || m_rows > 32 ? 2 : m_rows <= 24 ? 3 : 4; }

static int few_rows_of(const blink_model_cfg* m, int max_new) {
  if (m->dtype == BLINK_DTYPE_FP32) return m->head_dim == 128 ? 4 : 8;
  return 8 * few_nt((int64_t)max_new * (m->n_q_heads / m->n_kv_heads));
}

}  // namespace blink

extern "C" {

uint64_t blink_window_attention_workspace(const blink_model_cfg* model, int max_new) {
  if (blink_weights_bytes(model) == 0 || max_new < 1) return 0;   // (no such model)
  // (a unit of up to 24 rows of a head takes as many instructions as it needs, of more 4, and of more than 32 two: requests of up to max_new rows need the most of these)
  const int64_t m_rows = (int64_t)max_new * (model->n_q_heads / model->n_kv_heads);
  const int rows = model->dtype == BLINK_DTYPE_BF16 && m_rows > 24 ? 32 : blink::few_rows_of(model, max_new);
  return blink::few_bytes(rows, model->head_dim);
}

int blink_window_attention(const blink_model_cfg* model, const blink_kv_pool* kv, int layer, const void* q, int64_t q_stride, int rows,
                           const int32_t* row_start, const int32_t* kv_len, int n_requests, const int32_t* block_table, int table_stride,
                           int window, int sinks, int max_new, void* out, int64_t out_stride, void* workspace, uint64_t workspace_bytes,
                           void* stream) {
  using namespace blink;
  AttnArgs a;
  const int rc = ops_pool(model, kv, layer, &a.pool);
  if (rc != BLINK_OK) return rc;
  const int64_t q_dim = (int64_t)a.pool.Hq * a.pool.hd;
  if (!ops_aligned(q, 16) || !ops_aligned(out, 16) || !ops_aligned(row_start, 4) || !ops_aligned(kv_len, 4) || !ops_aligned(block_table, 4))
    return BLINK_EINVAL;
  if (rows < 1 || n_requests < 1 || table_stride < 1 || window < 0 || sinks < 0 || max_new < 1) return BLINK_EINVAL;
  if (q_stride < q_dim || out_stride < q_dim || q_stride % 8 || out_stride % 8) return BLINK_EINVAL;
  if (n_requests > OPS_MAX_REQUESTS || rows > 0x3ffffff || table_stride > 0x3ffffff || sinks > 0x3fffffff || window > 0x3fffffff) return BLINK_ETOOBIG;
  if (!ops_aligned(workspace, 256) || workspace_bytes < few_bytes(few_rows_of(model, max_new), model->head_dim)) return BLINK_EINVAL;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return BLINK_ECUDA;
  a.q = q;
  a.out = out;
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.row_start = row_start;
  a.kv_len = kv_len;
  a.table = block_table;
  a.n = n_requests;
  a.rows = rows;
  a.stride = table_stride;
  a.window = window;
  a.sinks = sinks;
  a.few = 0x7fffffff;
  a.qscale = (float)(1.4426950408889634 / std::sqrt((double)a.pool.hd));
  a.out_32 = ops_aligned(out, 32) && out_stride % 16 == 0;
  a.ws = static_cast<char*>(workspace);
  const int nt = few_nt((int64_t)max_new * a.pool.rep);
  const bool bf16 = model->dtype == BLINK_DTYPE_BF16;
  const bool tiles = (int64_t)max_new * a.pool.rep > (bf16 ? 32 : 8);   // there may be requests of more than a few rows
  if (tiles) a.few = (bf16 ? 8 * nt : 8) / a.pool.rep;
  // keys that a request of few rows, or the rows of a unit of the tiles, see at most
  const int64_t keys = std::min<int64_t>((int64_t)table_stride * OPS_BLOCK, window > 0 ? (int64_t)window + sinks + std::min(max_new, 256) : INT64_MAX);
  // Everything to the tiles, which share nothing out over CTAs, where there are units enough and none can be very long: a tile's rows cost the same
  // however few they are, but its copies run by themselves.  (8B shape, us, with the kernels for few rows | without: 48 requests of 1 to 6 rows behind
  // 300 to 5000 keys 113 | 88, of 1 to 3 92 | 87; 28 of them (1 to 6 rows) 76 | 60, 19 57 | 55, 10 32 | 46; 40 of 1 to 300 rows with a window of 256 49 | 42.  20 of 5
  // rows behind 10000 keys 150 | 202.  Evenly long ones end later where they do not fill the CTAs: 48 of 4 rows behind 2500 keys 92 | 96, of 8 133 | 96.  Eight rows of a
  // head or less, one instruction of those kernels: 64 rows behind 5000 keys 196 | 225.)  Where no row sees more
  // than some 1500 keys fewer units will do, and none have to be there when the tiles are called anyway: 10 of 1 to 6 rows behind 200 to 900
  // keys 16.7 | 17.1; with a window of 1024 8 rows beside a prompt of 64 21 | 19, beside two of 1000 51 | 43, whole prompts of three requests 175 | 175.
  const int64_t least = keys > ALL_SHORT ? sms + sms / 2 : tiles ? 0 : sms / 2;
  if (bf16 && (int64_t)max_new * a.pool.rep > ALL_ROWS && (int64_t)n_requests * a.pool.Hkv >= least && keys <= ALL_KEYS) {
    a.few = 0;
    return attn_tiles(a, sms, stream);
  }
  const int64_t mr = few_rows_of(model, max_new), rows_few = std::min<int64_t>(max_new, a.few);
  const int64_t groups = (rows_few * a.pool.rep + mr - 1) / mr, units = (int64_t)n_requests * a.pool.Hkv * groups;
  a.near_ctas = 0;
  // A cluster for each unit, of as many CTAs as its keys are worth and there is room for; the sequence of tiles where units are many or long.  (One row of the 8B
  // shape, us, clusters of 1 | 4 | 8 | 16: behind 15 keys 4.8 | 5.4 | 5.9 | 6.9, 250 7.4 | 6.0 | 6.4 | 7.7, 1000 15.0 | 8.0 | 7.1 | 7.7, 2000 25 | 10.5 | 8.5 | 8.8; 32 bits, 500
  // 22 | 10.1 | 8.6 | 10.4, 1000 39 | 14.3 | 10.9 | 10.5.  The sequence | so: 1 x 4000 18.4 | 10.9, 16000 25.9 | 24.3, 30000 33.9 | 39.9; heads of 64, 8000
  // 17.3 | 13.4, 16000 18.9 | 22.5; 4 x 100 9.2 | 5.9, 3 x 1000 of 4 rows 13.1 | 9.6, 8 x 1000 14.7 | 11.7, 16 x 400 14.4 | 10.5, 16 x 800 17.3 | 16.4, 64 x 50 13.7 | 11.2,
  // 64 x 200 18.6 | 19.3.)
  int ctas = keys <= 64 ? 1 : keys <= 256 ? 4 : keys <= (bf16 ? 2048 : 512) ? 8 : 16;
  while (ctas > 1 && units * ctas > (ctas == 16 ? sms : 2 * sms)) ctas /= 2;
  if (ctas == 2 && keys <= 512) ctas = 1;   // (16 x 200: 8.5 | 7.8)
  const int64_t limit = ctas == 16 ? (bf16 ? 128 : 32) * a.pool.hd : units > 2 * sms ? (units > 4 * sms ? 0 : 128) : (bf16 ? 512 : 256) * ctas;
  if (keys <= limit) {
    a.near_groups = (int)groups;
    a.near_ctas = ctas;
  }
  // In 32 bits where a row sees so little that the kernels for few rows only add their launches.  (us, with them | without: the small shape, 8 requests of
  // 40 rows behind 30 keys 17.1 | 13.1, 64 of one row and one of 40 behind 200 keys 46 | 26; the 8B shape, 4 and one 43 | 35, but behind 450 keys 24 | 62
  // where the 40 rows see none of them.)
  if (!bf16 && tiles && keys <= ALL_KEYS_32) {
    a.few = 0;
    return attn_blocks(a, sms, stream);
  }
  if (!bf16) {   // the many rows first: the few find room beside them
    const int done = tiles ? attn_blocks(a, sms, stream) : BLINK_OK;
    if (done != BLINK_OK) return done;
    return a.pool.hd == 128 ? few_run<float, 128, FewFp32<128>, 2>(a, sms, stream) : few_run<float, 64, FewFp32<64>, 2>(a, sms, stream);
  }
  const int done = a.pool.hd == 128 ? few_bf16<128>(a, nt, sms, stream) : few_bf16<64>(a, nt, sms, stream);
  return done != BLINK_OK || !tiles ? done : attn_tiles(a, sms, stream);   // (whose counter the first kernel zeroes)
}

}  // extern "C"
