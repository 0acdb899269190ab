// Drafted tokens held against the target's probabilities: blink_verify_drafts.
//
//   p_i = softmax(logits_i / T);  draft x_i is accepted while u_i * q_i(x_i) < p_i(x_i)
//   first refused i: a token from max(0, p_i - q_i), none refused: from p of the last row; by the inverse of its running sum in the order of
//   the indexes: the first j with sum_{<= j} > v * sum
//
// Three kernels (or two).
//   rows    largest value and sum of exponentials of pieces of 1024 entries of every row, a warp each: one pass over the logits
//           (HBM, 4 bytes an entry: 215 rows of 128256 23 us, cold, 4.8 TB/s).  A lane has its 32 entries on their way at once and sums against its own largest
//           value, so that nothing waits for another warp.  Exponentials in 32 bits, sums of a lane's entries in 32, everything above in
//           64: the acceptance test is off by some 1e-8 where the entries differ, and by 1e-6 at worst (most of the weight on entries that are
//           all alike, 12 below the largest: an argument's rounding of 2^-24 of itself, and the exponential's own 2^-22).
//   choose  a CTA per request: the first refused draft, from the pieces (with few requests every CTA of the draw does so for itself)
//   draw    a cluster of 16 CTAs per request: the exponentials of that row, which stay in registers (up to 16 a thread; beyond 131072 entries they are
//           made again from tile to tile), their sum, then the weights
//           max(0, p - q), their sum, and the entry at which the running sum passes its target.  Sums go from CTA to CTA through
//           distributed shared memory.  What bounds it: latency, the chain load, sum, exchange, sum, exchange, search of each of the waves that many
//           requests take, with some 70 instructions an entry (issue slots 45 % busy, the 64-bit pipe 21 %, 40 % of the warps resident): 57 rows of 128256
//           42 us in four waves, one of 32000 5.
// The chosen row's sums decide between neighbours that are as close as 1e-6, so its exponentials, sums and running sum are in 64 bits.  Sums are
// taken in an order that sizes alone fix: the same call gives the same token.
#include <cooperative_groups.h>

#include <cmath>
#include <utility>

#include "ops.h"

namespace blink {

constexpr int VER_WARPS = 8, VER_THREADS = VER_WARPS * 32;
constexpr int VER_EACH = 32, VER_CHUNK = 32 * VER_EACH;   // rows: entries of a lane, a warp
constexpr int PICK_THREADS = 512, PICK_WARPS = 16, PICK_CTAS = 16;   // draw
constexpr int PICK_CHOOSE = 12;   // requests up to which each draw chooses for itself

struct VerChunk {
  double sum;   // of exp((z - max) / T)
  float max;
  int index;    // first of the largest, where that may matter (see ver_one)
};
struct VerChoice {
  int row;      // that is drawn from; -1: none, or one that stands for its largest entry alone
  int refused;  // a draft of it was
  float max;
  int unused;
};
struct VerifyArgs {
  const float* logits;
  const float* probs;
  long long logits_stride, probs_stride;
  const int32_t *row_start, *draft;
  const float *temperature, *u_accept, *u_pick;
  int32_t *tokens, *accepted;
  VerChunk* chunks_of;   // [rows][chunks]
  VerChoice* choice;     // [n]
  int n, rows, vocab, chunks, groups;
  bool vec, probs_vec;   // rows on 16-byte boundaries
  bool clear;            // rows that belong to nobody get the token -1
  double sixteenths[16]; // 2^(i / 16)
  double series[5];      // (ln 2 / 16)^i / i!, i = 1 .. 5 (as operands from the constant bank: written out they take two moves each at every use)
};

// No number: as if the entry were not there.
__device__ __forceinline__ float ver_entry(float z) { return z == z ? z : -INFINITY; }

__device__ __forceinline__ float ver_ex2(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 ver_add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 ver_mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// The larger of two, of equal ones that of the lower index.
__device__ __forceinline__ void ver_larger(float& m, int& i, float m2, int i2) {
  if (m2 > m || (m2 == m && i2 < i)) { m = m2; i = i2; }
}

// Entries of 4 * lane + 128 * k + 0 .. 3 of a tile that has n of them; 16 bytes at a time where rows are aligned.
template <int EACH>
__device__ __forceinline__ void ver_load(float (&v)[EACH], const float* z, int n, bool vec, float behind) {
  const int lane = threadIdx.x & 31;
  if (vec && n >= 32 * EACH) {   // (no question at every piece)
#pragma unroll
    for (int k = 0; k < EACH / 4; ++k) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(z + k * 128 + lane * 4));   // (the chosen row is read again, from L2)
      v[4 * k] = x.x; v[4 * k + 1] = x.y; v[4 * k + 2] = x.z; v[4 * k + 3] = x.w;
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < EACH / 4; ++k) {
    const int at = k * 128 + lane * 4;
    if (vec && at + 4 <= n) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(z + at));
      v[4 * k] = x.x; v[4 * k + 1] = x.y; v[4 * k + 2] = x.z; v[4 * k + 3] = x.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * k + j] = at + j < n ? __ldcg(z + at + j) : behind;
    }
  }
}

// At a temperature that is not above 0 and finite a row stands for its largest entry alone; so does one whose largest entry is infinite, or that
// holds no number.
__device__ __forceinline__ bool ver_one(float T, float m) { return !(T > 0.f && T < INFINITY) || !(m > -INFINITY) || !(m < INFINITY); }

__global__ void __launch_bounds__(VER_THREADS) blink_verify_rows_kernel(const __grid_constant__ VerifyArgs a) {
  __shared__ int s_req;
  __shared__ float s_T;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = (int)(blockIdx.x / (unsigned)a.groups), chunk = (int)(blockIdx.x - (unsigned)row * a.groups) * VER_WARPS + warp;
  ops_begin();
  float v[VER_EACH];
  if (chunk < a.chunks)
    ver_load(v, a.logits + row * a.logits_stride + (long long)chunk * VER_CHUNK, min(VER_CHUNK, a.vocab - chunk * VER_CHUNK), a.vec, -INFINITY);
  if (threadIdx.x == 0) s_req = -1;
  __syncthreads();
  for (int r = threadIdx.x; r < a.n; r += VER_THREADS) {
    if (a.row_start[r] <= row && row < a.row_start[r + 1]) {
      s_req = r;
      s_T = a.temperature[r];
    }
  }
  __syncthreads();
  const int req = s_req;
  if (req < 0 && a.clear && chunk == 0 && lane == 0) a.tokens[row] = -1;
  if (req < 0 || chunk >= a.chunks) return;   // (whole warps) a row behind the last request
  const float T = s_T;
  float m0 = -INFINITY, m1 = -INFINITY;   // (the larger of a number and none is the number)
#pragma unroll
  for (int k = 0; k < VER_EACH; k += 4) {
    m0 = fmaxf(fmaxf(m0, v[k]), v[k + 1]);
    m1 = fmaxf(fmaxf(m1, v[k + 2]), v[k + 3]);
  }
  const float mine = fmaxf(m0, m1);
  float m = mine;
#pragma unroll
  for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  double sum = 0.0;
  int idx = 0;
  if (ver_one(T, m)) {
    idx = 0x7fffffff;
#pragma unroll
    for (int k = VER_EACH - 1; k >= 0; --k)
      if (ver_entry(v[k]) == m) idx = (k >> 2) * 128 + lane * 4 + (k & 3);
#pragma unroll
    for (int d = 16; d; d >>= 1) idx = min(idx, __shfl_xor_sync(0xffffffffu, idx, d));
  } else {
    // At the ends of T's range entries are taken times a power of two, and the scale by that less: their differences, or the scale itself, would leave
    // 32 bits.  (With entries above 1 there is no need at the lower end: what is not the largest has no weight there.)
    const float unit = T > 0x1p100f ? 0x1p-8f : T < 0x1p-100f && fabsf(mine) < 1.f ? 0x1p64f : 1.f;
    if (unit != 1.f) {
#pragma unroll
      for (int k = 0; k < VER_EACH; ++k) v[k] *= unit;
    }
    const float scale = fminf(1.4426950408889634f / (T * unit), 3e38f);
    const float base = mine == -INFINITY ? 0.f : mine * unit;
    const float2 scale2 = make_float2(scale, scale), base2 = make_float2(-base, -base);
    auto lane_sum = [&]() {
      float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
      for (int k = 0; k < VER_EACH; k += 4) {   // (no entry: 2^-inf)
        const float2 x = ver_mul2(ver_add2(make_float2(v[k], v[k + 1]), base2), scale2), y = ver_mul2(ver_add2(make_float2(v[k + 2], v[k + 3]), base2), scale2);
        s0 = ver_add2(s0, make_float2(ver_ex2(x.x), ver_ex2(x.y)));
        s1 = ver_add2(s1, make_float2(ver_ex2(y.x), ver_ex2(y.y)));
      }
      return (s0.x + s0.y) + (s1.x + s1.y);
    };
    float s = lane_sum();
    if (s != s) {   // an entry that is no number
#pragma unroll
      for (int k = 0; k < VER_EACH; ++k) v[k] = ver_entry(v[k]);
      s = lane_sum();
    }
    sum = (double)s * (double)ver_ex2((mine * unit - m * unit) * scale);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  }
  if (lane == 0) a.chunks_of[(size_t)row * a.chunks + chunk] = VerChunk{sum, m, chunk * VER_CHUNK + idx};
}

// exp((z - top) / T) in 64 bits, as 2^(n / 16) 2^(f / 16): n whole, its sixteenths from a table in shared memory (16 entries: two banks
// each, no conflicts) and the rest into the exponent; |f| <= 1/2, by the series of exp(f ln 2 / 16) up to its fifth power (off by
// (ln 2 / 32)^6 / 6! = 1.4e-13).  The largest entry is taken away first: it is exactly 1 at every temperature, where the rounding of top * scale
// alone would be many powers of two at 1e-18.  64-bit operations are what the kernels below are bound by: twelve here, one of them the conversion.
struct VerExp {
  const double* table;   // 2^(i / 16)
  const double* series;
  double scale, top;     // 16 log2(e) / T
  float below;         // entries below this are 0: (z - top) / T < -700
};
__device__ __forceinline__ VerExp ver_exp_of(const VerifyArgs& a, const double* table, float top, float T) {
  VerExp x;
  x.table = table;
  x.series = a.series;
  x.scale = 16.0 * 1.44269504088896340736 / (double)T;
  x.top = (double)top;
  x.below = fmaxf(__double2float_ru((double)top - 700.0 * (double)T), -3.402823466e38f);   // (rounded up: no less than -700; above -inf)
  return x;
}
__device__ __forceinline__ double ver_exp(const VerExp& x, float z) {
  constexpr double SHIFT = 6755399441055744.0;   // 1.5 * 2^52: adding it leaves the nearest whole number in the low bits
  const double d = (double)z - x.top, s = fma(d, x.scale, SHIFT), f = fma(d, x.scale, -(s - SHIFT));
  const int n = __double2loint(s);
  const double p = fma(f, fma(f, fma(f, fma(f, fma(f, x.series[4], x.series[3]), x.series[2]), x.series[1]), x.series[0]), 1.0) * x.table[n & 15];
  return z >= x.below ? __hiloint2double(__double2hiint(p) + ((n >> 4) << 20), __double2loint(p)) : 0.0;   // (no number: 0 too)
}
__device__ __forceinline__ void ver_table(double* table, const VerifyArgs& a) {   // before a barrier
  if (threadIdx.x < 16) table[threadIdx.x] = a.sixteenths[threadIdx.x];
}

// The request's rows, first and behind the last.
__device__ __forceinline__ int2 ver_rows(const VerifyArgs& a, int req) {
  const int start = min(max(a.row_start[req], 0), a.rows);
  return make_int2(start, min(max(a.row_start[req + 1], start), a.rows));
}

// What is chosen for a request: its rows, the accepted drafts, what the draw needs, and the token of a row that stands for its largest entry alone.
struct VerPicked {
  int start, k, accepted, index;   // k: drafts, -1 for a request without rows; index: -1 where a token is drawn
  VerChoice choice;
};
// By a CTA of WARPS warps, which all get it; s_table is there.  Waits for the first kernel.
template <int WARPS>
__device__ __forceinline__ VerPicked ver_choose(const VerifyArgs& a, int req, const double* s_table, VerPicked* s_out) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  ops_wait();
  const int2 rows = ver_rows(a, req);
  const int start = rows.x, k = rows.y - rows.x - 1;
  const float T = a.temperature[req];
  if (tid == 0) s_out->accepted = max(k, 0);
  __syncthreads();
  // A row from its pieces: largest value and its index (and whether the row stands for that entry alone); then its sum.
  auto top_of = [&](int row, float& m, int& idx) {
    const VerChunk* c = a.chunks_of + (size_t)row * a.chunks;
    m = -INFINITY;
    idx = 0x7fffffff;
#pragma unroll 4
    for (int j = lane; j < a.chunks; j += 32) ver_larger(m, idx, c[j].max, c[j].index);
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      const float m2 = __shfl_xor_sync(0xffffffffu, m, d);
      const int i2 = __shfl_xor_sync(0xffffffffu, idx, d);
      ver_larger(m, idx, m2, i2);
    }
    return ver_one(T, m);
  };
  auto sum_of = [&](int row, float m) {
    const VerChunk* c = a.chunks_of + (size_t)row * a.chunks;
    const VerExp x = ver_exp_of(a, s_table, m, T);
    double sum = 0.0;
#pragma unroll 4
    for (int j = lane; j < a.chunks; j += 32) sum += c[j].sum * ver_exp(x, c[j].max);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    return sum;
  };
  for (int i = warp; i < k; i += WARPS) {   // (loads that wait for one another: those of the draft are on their way beside those of the pieces)
    float m;
    int idx;
    const int row = start + i, x = a.draft[row];
    const float u = a.u_accept[row];
    const bool one = top_of(row, m, idx);
    const bool in = x >= 0 && x < a.vocab;
    const float z = in ? ver_entry(__ldcg(a.logits + row * a.logits_stride + x)) : -INFINITY, q = in && a.probs ? a.probs[row * a.probs_stride + x] : 1.f;
    const double sum = one ? 0.0 : sum_of(row, m);
    const bool ok = one ? x == idx : in && (double)u * (double)q * sum < ver_exp(ver_exp_of(a, s_table, m, T), z);
    if (lane == 0 && !ok) atomicMin(&s_out->accepted, i);
  }
  __syncthreads();
  if (warp == 0) {
    const int acc = s_out->accepted, row = start + acc;
    float top = 0.f;
    int index = -1;
    const bool one = k < 0 || top_of(row, top, index);
    if (lane == 0) {
      s_out->start = start;
      s_out->k = k;
      s_out->index = one ? index : -1;
      s_out->choice = VerChoice{one ? -1 : row, acc < k, top, 0};
    }
  }
  __syncthreads();
  return *s_out;
}
// The outputs that stand fixed then, by a CTA.
__device__ __forceinline__ void ver_write(const VerifyArgs& a, int req, const VerPicked& p) {
  if (threadIdx.x == 0) a.accepted[req] = p.accepted;
  for (int i = threadIdx.x; i <= p.k; i += blockDim.x)
    if (i != p.accepted || p.index >= 0) a.tokens[p.start + i] = i < p.accepted ? a.draft[p.start + i] : i == p.accepted ? p.index : -1;
}

__global__ void __launch_bounds__(VER_THREADS) blink_verify_choose_kernel(const __grid_constant__ VerifyArgs a) {
  __shared__ VerPicked s_out;
  __shared__ double s_table[16];
  const int req = (int)blockIdx.x;
  ops_next();
  ver_table(s_table, a);
  const VerPicked p = ver_choose<VER_WARPS>(a, req, s_table, &s_out);
  if (threadIdx.x == 0) a.choice[req] = p.choice;
  ver_write(a, req, p);
}

// The first of 16 parts (a lane each, lanes 16 .. 31 have 0) whose running sum exceeds target, else the last with anything in it; `base` grows by
// what stands before it.
__device__ __forceinline__ int ver_part(double part, double target, double& base) {
  const int lane = threadIdx.x & 31;
  double c = part;
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) {
    const double u = __shfl_up_sync(0xffffffffu, c, d);
    if (lane >= d) c += u;
  }
  const unsigned hit = __ballot_sync(0xffffffffu, part > 0.0 && base + c > target), any = __ballot_sync(0xffffffffu, part > 0.0);
  const int at = hit ? __ffs(hit) - 1 : any ? 31 - __clz(any) : 0;
  const double before = __shfl_sync(0xffffffffu, c, max(at - 1, 0));
  if (at > 0) base += before;
  return at;
}

// EACH: entries of a lane at a time.  CHOOSE: every CTA chooses for itself, and the kernel before this one is left out.  With as many requests
// as there is room for clusters at a time that is a launch less, with more each wave of them would choose first.  (Five rows of 32000 a request, us, with
// the kernel before it | without: 1 request 9.5 | 9.0, 8 11.6 | 10.4, 12 13.1 | 12.0, 16 15.7 | 17.6, 64 34 | 43.)
template <int EACH, bool CHOOSE>
__global__ void __launch_bounds__(PICK_THREADS, 2) blink_verify_draw_kernel(const __grid_constant__ VerifyArgs a) {
  namespace cg = cooperative_groups;
  constexpr int TILE = 32 * EACH;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ __align__(16) float s_q[PICK_WARPS][TILE];   // a tile of q per warp, each lane's own entries
  __shared__ double s_part[PICK_WARPS];                   // a sum per warp
  __shared__ double s_all[2][PICK_CTAS];                  // a sum per CTA, the same in all of them
  __shared__ double s_table[16];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster.block_rank(), req = (int)(blockIdx.x / PICK_CTAS);
  const int V = a.vocab;
  ver_table(s_table, a);
  __shared__ VerPicked s_out;
  VerPicked picked;
  VerChoice choice;
  if constexpr (CHOOSE) {
    ops_next();
    picked = ver_choose<PICK_WARPS>(a, req, s_table, &s_out);
    choice = picked.choice;
  } else {
    __syncthreads();
    ops_wait();
    ops_next();
    choice = a.choice[req];
  }
  const float T = a.temperature[req], u = a.u_pick[req];
  const int row = choice.row;
  if (!CHOOSE && row < 0) return;   // (the whole cluster)
  cg::cluster_group::arrival_token there = cluster.barrier_arrive();   // all CTAs have to be there before they are written to
  if constexpr (CHOOSE) {
    if (row < 0) {
      cluster.barrier_wait(std::move(there));
      if (rank == 0) ver_write(a, req, picked);
      return;
    }
  }
  // the row's entries: a run of tiles per warp, in the order of CTAs, warps and tiles
  const int tiles = (V + PICK_CTAS * PICK_WARPS * TILE - 1) / (PICK_CTAS * PICK_WARPS * TILE);
  const int w0 = (rank * PICK_WARPS + warp) * tiles * TILE;
  const float* z = a.logits + row * a.logits_stride;
  const float* q = choice.refused && a.probs ? a.probs + row * a.probs_stride : nullptr;
  const float* const q_rests = q;
  if (tiles > 1) q = nullptr;   // (of several tiles each is copied when its rests are taken: the sum of exponentials does without q)
  float zv[EACH];   // of the warp's first tile
  ver_load(zv, z + w0, V - w0, a.vec, -INFINITY);
  auto fetch_q = [&](int at) {   // behind the end: zeros
    asm volatile("cp.async.wait_group 0;" ::: "memory");   // (copies that are on their way into the same place have no order among themselves)
    const bool whole = a.probs_vec && at + TILE <= V;
#pragma unroll
    for (int g = 0; g < EACH / 4; ++g) {
      const int o = g * 128 + lane * 4;
      const uint32_t dst = (uint32_t)__cvta_generic_to_shared(&s_q[warp][o]);
      if (whole) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(q + at + o) : "memory");
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + 4 * j), "l"(q + (at + o + j < V ? at + o + j : 0)), "r"(at + o + j < V ? 4u : 0u) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (q) fetch_q(w0);
  const VerExp exp = ver_exp_of(a, s_table, choice.max, T);
  double e[EACH];
  auto exps = [&]() {
#pragma unroll
    for (int i = 0; i < EACH; ++i) e[i] = ver_exp(exp, zv[i]);
  };
  auto lane_sum = [&]() {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < EACH; i += 4) s += (e[i] + e[i + 1]) + (e[i + 2] + e[i + 3]);
    return s;
  };
  // sum over the lanes -> over the CTA -> over the cluster; s_part keeps the warps', s_all the CTAs'
  auto sum_all = [&](double s, int which) {
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if (lane == 0) s_part[warp] = s;
    __syncthreads();
    if (warp == 0) {
      double t = s_part[lane & 15];
#pragma unroll
      for (int d = 8; d; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
      if (lane < PICK_CTAS) *cluster.map_shared_rank(&s_all[which][rank], lane) = t;
    }
    cluster.sync();
    double t = s_all[which][lane & 15];
#pragma unroll
    for (int d = 8; d; d >>= 1) t += __shfl_xor_sync(0xffffffffu, t, d);
    return t;
  };
  auto load_more = [&](int t) {   // tiles behind the first are read again in every pass
    const int at = w0 + t * TILE;
    ver_load(zv, z + at, V - at, a.vec, -INFINITY);
    if (q) fetch_q(at);
  };
  double s = 0.0;
#pragma unroll 1
  for (int t = tiles - 1; t >= 0; --t) {   // (the first last: it stays)
    if (tiles > 1) load_more(t);
    exps();
    s += lane_sum();
  }
  cluster.barrier_wait(std::move(there));
  if constexpr (CHOOSE)
    if (rank == 0) ver_write(a, req, picked);   // (all CTAs have read the drafts, which may lie there)
  const double inv_S = 1.0 / sum_all(s, 0);

  // what is drawn from: p - q where a draft was refused (what is no number or negative in q counts as 0), p otherwise
  int x = choice.refused && !a.probs ? a.draft[row] : -1;
  auto rests = [&](int t) {   // of tile t, whose exponentials are in e
    if (q) {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
      for (int i = 0; i < EACH; i += 4) {
        const float4 v = *reinterpret_cast<const float4*>(&s_q[warp][i * 32 + lane * 4]);
        const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const double r = fma(e[i + j], inv_S, -(double)fmaxf(w[j], 0.f));   // (the larger of 0 and no number is 0)
          e[i + j] = __double2hiint(r) < 0 ? 0.0 : r;
        }
      }
    } else {
      const int at = w0 + t * TILE + lane * 4;
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const double p = e[i] * inv_S;
        e[i] = at + (i >> 2) * 128 + (i & 3) == x ? 0.0 : p;
      }
    }
  };
  q = q_rests;
  bool have = tiles == 1;   // the exponentials of the only tile are in e
  auto rest_sum = [&]() {
    double r = 0.0;
#pragma unroll 1
    for (int t = tiles - 1; t >= 0; --t) {
      if (!have) {
        load_more(t);
        exps();
      }
      rests(t);
      r += lane_sum();
    }
    return sum_all(r, 1);
  };
  double total;
#pragma unroll 1
  while (true) {
    total = rest_sum();
    if (total > 0.0 || (!q && x < 0)) break;
    q = nullptr;          // q covers p everywhere: from p itself
    x = -1;
    have = false;
    cluster.sync();       // (everybody has read the sums)
  }
  const double target = (double)u * total;
  // the CTA, and the warp in it, whose run takes the sum past the target; else the last with anything in it
  double base = 0.0;
  if (ver_part(lane < PICK_CTAS ? s_all[1][lane] : 0.0, target, base) != rank) return;
  if (ver_part(lane < PICK_WARPS ? s_part[lane] : 0.0, target, base) != warp) return;
  int token = -1, last = 0;
#pragma unroll 1
  for (int t = 0; t < tiles && token < 0; ++t) {
    if (tiles > 1) {   // (one tile: its are in e)
      load_more(t);
      exps();
      rests(t);
    }
    double c[EACH / 4];   // running sums over the lanes, of each group of 128
#pragma unroll
    for (int g = 0; g < EACH / 4; ++g) c[g] = (e[4 * g] + e[4 * g + 1]) + (e[4 * g + 2] + e[4 * g + 3]);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
#pragma unroll
      for (int g = 0; g < EACH / 4; ++g) {
        const double u = __shfl_up_sync(0xffffffffu, c[g], d);
        if (lane >= d) c[g] += u;
      }
    }
#pragma unroll
    for (int g = 0; g < EACH / 4; ++g) {
      const double up = __shfl_up_sync(0xffffffffu, c[g], 1);
      double run = lane ? base + up : base;
      int hit = 4, some = -1;   // of the lane's four
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        run += e[4 * g + j];
        if (e[4 * g + j] > 0.0) {
          some = j;
          if (hit == 4 && run > target) hit = j;
        }
      }
      const unsigned hits = __ballot_sync(0xffffffffu, hit < 4), any = __ballot_sync(0xffffffffu, some >= 0);
      const int at = w0 + t * TILE + g * 128;
      const int l = hits ? __ffs(hits) - 1 : any ? 31 - __clz(any) : 0;
      const int h = __shfl_sync(0xffffffffu, hit, l), o = __shfl_sync(0xffffffffu, some, l);
      if (token < 0) {
        if (hits) token = at + l * 4 + h;
        else if (any) last = at + l * 4 + o;
      }
      base += __shfl_sync(0xffffffffu, c[g], 31);
    }
  }
  if (lane == 0) a.tokens[row] = token >= 0 ? token : last;
}

template <int EACH, bool CHOOSE>
static int verify_draw(const VerifyArgs& a, void* stream) {
  return ops_launch(blink_verify_draw_kernel<EACH, CHOOSE>, (int64_t)a.n * PICK_CTAS, PICK_THREADS, 0, stream, PICK_CTAS, a);
}

struct VerifySpace {
  uint64_t choice, end;   // behind the pieces
  int64_t n_chunks;
};
static VerifySpace verify_space(int64_t rows, int64_t n, int64_t vocab) {
  VerifySpace s;
  s.n_chunks = (vocab + VER_CHUNK - 1) / VER_CHUNK;
  s.choice = (uint64_t)(rows * s.n_chunks) * sizeof(VerChunk);
  s.end = s.choice + (uint64_t)n * sizeof(VerChoice);
  return s;
}

int verify_drafts(const float* logits, int64_t logits_stride, int rows, int vocab, const int32_t* row_start, int n_requests, const int32_t* draft_tokens,
                  const float* draft_probs, int64_t probs_stride, const float* temperature, const float* u_accept, const float* u_pick, int32_t* out_tokens,
                  int32_t* n_accepted, void* workspace, uint64_t workspace_bytes, bool clear, void* stream) {
  const void* must[] = {logits, row_start, draft_tokens, temperature, u_accept, u_pick, out_tokens, n_accepted};
  for (const void* p : must)
    if (!ops_aligned(p, 4)) return BLINK_EINVAL;
  if (((uintptr_t)draft_probs & 3) || rows < 1 || vocab < 2 || n_requests < 1 || logits_stride < vocab || (draft_probs && probs_stride < vocab))
    return BLINK_EINVAL;
  if (vocab > 0x3fffffff || n_requests > OPS_MAX_REQUESTS) return BLINK_ETOOBIG;
  const VerifySpace space = verify_space(rows, n_requests, vocab);
  if (!ops_aligned(workspace, 16) || workspace_bytes < space.end) return BLINK_EINVAL;
  char* ws = static_cast<char*>(workspace);
  VerifyArgs a;
  a.clear = clear;
  a.logits = logits;
  a.probs = draft_probs;
  a.logits_stride = logits_stride;
  a.probs_stride = probs_stride;
  a.row_start = row_start;
  a.draft = draft_tokens;
  a.temperature = temperature;
  a.u_accept = u_accept;
  a.u_pick = u_pick;
  a.tokens = out_tokens;
  a.accepted = n_accepted;
  a.chunks_of = reinterpret_cast<VerChunk*>(ws);
  a.choice = reinterpret_cast<VerChoice*>(ws + space.choice);
  a.n = n_requests;
  a.rows = rows;
  a.vocab = vocab;
  a.chunks = (int)space.n_chunks;
  a.groups = (int)((space.n_chunks + VER_WARPS - 1) / VER_WARPS);
  for (int i = 0; i < 16; ++i) a.sixteenths[i] = std::exp2(i / 16.0);
  const double l = std::log(2.0) / 16;
  double term = 1.0;
  for (int i = 0; i < 5; ++i) a.series[i] = term = term * l / (i + 1);
  a.vec = logits_stride % 4 == 0 && ops_aligned(logits, 16);
  a.probs_vec = draft_probs && probs_stride % 4 == 0 && ops_aligned(draft_probs, 16);
  int rc = ops_launch(blink_verify_rows_kernel, (int64_t)rows * a.groups, VER_THREADS, 0, stream, 0, a);
  const bool choose = n_requests > PICK_CHOOSE;
  if (rc == BLINK_OK && choose) rc = ops_launch(blink_verify_choose_kernel, n_requests, VER_THREADS, 0, stream, 0, a);
  if (rc != BLINK_OK) return rc;
  // as few entries of a lane as hold the row in one go: 32768 entries in 16 CTAs of 16 warps with four, 131072 with 16 (beyond that, runs of tiles)
  if (vocab <= 32768) return choose ? verify_draw<4, false>(a, stream) : verify_draw<4, true>(a, stream);
  if (vocab <= 65536) return choose ? verify_draw<8, false>(a, stream) : verify_draw<8, true>(a, stream);
  return choose ? verify_draw<16, false>(a, stream) : verify_draw<16, true>(a, stream);
}

}  // namespace blink

extern "C" {

uint64_t blink_verify_workspace(int rows, int n_requests, int vocab) {
  if (rows < 1 || n_requests < 1 || vocab < 2) return 0;
  return blink::verify_space(rows, n_requests, vocab).end;
}

int blink_verify_drafts(const float* logits, int64_t logits_stride, int rows, int vocab, const int32_t* row_start, int n_requests,
                        const int32_t* draft_tokens, const float* draft_probs, int64_t probs_stride, const float* temperature,
                        const float* u_accept, const float* u_pick, int32_t* out_tokens, int32_t* n_accepted, void* workspace,
                        uint64_t workspace_bytes, void* stream) {
  return blink::verify_drafts(logits, logits_stride, rows, vocab, row_start, n_requests, draft_tokens, draft_probs, probs_stride, temperature, u_accept, u_pick,
                              out_tokens, n_accepted, workspace, workspace_bytes, false, stream);
}

}  // extern "C"
