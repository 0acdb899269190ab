// Drafted tokens held against the target's probabilities: blink_verify_drafts.
//
//   p_i = softmax(logits_i / T);  draft x_i is accepted while u_i * q_i(x_i) < p_i(x_i)
//   first refused i: a token from max(0, p_i - q_i), none refused: from p of the last row; by the inverse of its running sum in the order of
//   the indexes: the first j with sum_{<= j} > v * sum
//
// Five kernels, each waiting for the one before it only where it needs its results.
//   rows    largest value and sum of exponentials of pieces of 1024 entries of every row, a warp each: one pass over the logits, which is what
//           bounds the whole (HBM: 4 bytes an entry).  A lane has its 32 entries on their way at once and sums against its own largest
//           value, so that nothing waits for another warp.  Exponentials in 32 bits, sums of a lane's entries in 32, everything above in
//           64: the acceptance test is off by some 1e-8.
//   choose  a CTA per request: the first refused draft, from the pieces
//   sums    the exponentials of that row, 512 entries a warp
//   weights the same entries once more: max(0, p - q), and their sum per warp
//   draw    a warp per request: the run of 512 in which the running sum passes its target, and the entry of that run
// (the last two as one kernel, the last CTA of a request to come drawing, were slower: a fence and a counter in every CTA's way)
// The chosen row's sums decide between neighbours that are as close as 1e-6, so its exponentials, sums and running sum are in 64 bits.  Sums are
// taken in an order that sizes alone fix, whoever comes last: the same call gives the same token.
#include <cmath>

#include "ops.h"

namespace blink {

constexpr int VER_WARPS = 8, VER_THREADS = VER_WARPS * 32;
constexpr int VER_EACH = 32, VER_CHUNK = 32 * VER_EACH;   // rows: entries of a lane, a warp
constexpr int VER_FEW = 16, VER_RUN = 32 * VER_FEW, VER_PART = VER_WARPS * VER_RUN;            // sums, weights

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
struct VerRun {
  double rest, all;   // sums over a warp's run: of the weights, and of p
};

struct VerifyArgs {
  const float* logits;
  const float* probs;
  long long logits_stride, probs_stride;
  const int32_t *row_start, *draft;
  const float *temperature, *u_accept, *u_pick;
  int32_t *tokens, *accepted;
  VerChunk* chunks_of;   // [rows][chunks]
  double* sums;          // [n][parts]
  VerRun* runs;          // [n][parts * VER_WARPS], and behind them the same for whole parts, [n][parts]
  VerRun* part_runs;
  VerChoice* choice;     // [n]
  int n, rows, vocab, chunks, groups, parts;
  bool vec, probs_vec;   // rows on 16-byte boundaries
  double sixteenths[16]; // 2^(i / 16)
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
#pragma unroll
  for (int k = 0; k < EACH / 4; ++k) {
    const int at = k * 128 + lane * 4;
    if (vec && at + 4 <= n) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(z + at));   // (the chosen row is read again, from L2)
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

__global__ void __launch_bounds__(VER_THREADS) blink_verify_rows_kernel(const VerifyArgs a) {
  __shared__ int s_req;
  __shared__ float s_T;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = (int)(blockIdx.x / (unsigned)a.groups), chunk = (int)(blockIdx.x - (unsigned)row * a.groups) * VER_WARPS + warp;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (the second kernel waits for the whole of this one itself)
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
    const float scale = fminf(1.4426950408889634f / T, 3e38f);
    const float base = mine == -INFINITY ? 0.f : mine;
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
    sum = (double)s * (double)ver_ex2((mine - m) * scale);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  }
  if (lane == 0) a.chunks_of[(size_t)row * a.chunks + chunk] = VerChunk{sum, m, chunk * VER_CHUNK + idx};
}

// exp((z - top) / T) in 64 bits, as 2^(n / 16) 2^(f / 16): n whole, its sixteenths from a table in shared memory (16 entries: two banks
// each, no conflicts) and the rest into the exponent; |f| <= 1/2, by the series of exp(f ln 2 / 16) up to its fifth power (off by
// (ln 2 / 32)^6 / 6! = 1.4e-13).  64-bit operations are what the kernels below are bound by: twelve here, one of them the conversion.
struct VerExp {
  const double* table;   // 2^(i / 16)
  double scale, shift;   // 16 log2(e) / T, and -top times that
  float top, below;      // entries below this are 0: (z - top) / T < -700
};
__device__ __forceinline__ VerExp ver_exp_of(const double* table, float top, float T) {
  VerExp x;
  x.table = table;
  x.scale = 16.0 * 1.44269504088896340736 / (double)T;
  x.shift = -(double)top * x.scale;
  x.top = top;
  x.below = fmaxf(top - 700.f * T, -3e38f);   // (above -inf)
  return x;
}
__device__ __forceinline__ double ver_exp(const VerExp& x, float z) {
  constexpr double L = 0.693147180559945309417 / 16, C2 = L * L / 2, C3 = C2 * L / 3, C4 = C3 * L / 4, C5 = C4 * L / 5;
  constexpr double SHIFT = 6755399441055744.0;   // 1.5 * 2^52: adding it leaves the nearest whole number in the low bits
  const double t = fma((double)z, x.scale, x.shift), s = t + SHIFT, f = t - (s - SHIFT);
  const int n = __double2loint(s);
  const double p = fma(f, fma(f, fma(f, fma(f, fma(f, C5, C4), C3), C2), L), 1.0) * x.table[n & 15];
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

__global__ void __launch_bounds__(VER_THREADS) blink_verify_choose_kernel(const VerifyArgs a) {
  __shared__ int s_first;
  __shared__ double s_table[16];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int req = (int)blockIdx.x;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // (all but the pieces is there before the first kernel is done)
  const int2 rows = ver_rows(a, req);
  const int start = rows.x, k = rows.y - rows.x - 1;
  const float T = a.temperature[req];
  if (tid == 0) s_first = max(k, 0);
  ver_table(s_table, a);
  __syncthreads();
  // A row from its pieces: largest value, its index, sum.
  auto row_of = [&](int row, float& m, int& idx, double& sum, bool with_sum) {
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
    const bool one = ver_one(T, m);
    sum = 0.0;
    if (!one && with_sum) {
      const VerExp x = ver_exp_of(s_table, m, T);
#pragma unroll 4
      for (int j = lane; j < a.chunks; j += 32) sum += c[j].sum * ver_exp(x, c[j].max);
#pragma unroll
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    }
    return one;
  };
  bool waited = false;
  for (int i = warp; i < k; i += VER_WARPS) {
    float m;
    int idx;
    double sum;
    const int row = start + i, x = a.draft[row];
    const bool in = x >= 0 && x < a.vocab;
    const float z = in ? ver_entry(__ldcg(a.logits + row * a.logits_stride + x)) : -INFINITY, q = in && a.probs ? a.probs[row * a.probs_stride + x] : 1.f;
    const float u = a.u_accept[row];
    if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
    waited = true;
    const bool one = row_of(row, m, idx, sum, true);
    const bool ok = one ? x == idx : in && (double)u * (double)q * sum < ver_exp(ver_exp_of(s_table, m, T), z);
    if (lane == 0 && !ok) atomicMin(&s_first, i);
  }
  if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncthreads();
  const int acc = s_first, row = start + acc;
  if (k < 0) {   // a request without rows
    if (tid == 0) {
      a.accepted[req] = 0;
      a.choice[req].row = -1;
    }
    return;
  }
  if (warp == 0) {
    float top;
    int index;
    double unused;
    const bool one = row_of(row, top, index, unused, false);
    if (lane == 0) {
      a.accepted[req] = acc;
      a.choice[req] = VerChoice{one ? -1 : row, acc < k, top, 0};
      if (one) a.tokens[row] = index;
    }
  }
  for (int i = tid; i <= k; i += VER_THREADS)
    if (i != acc) a.tokens[start + i] = i < acc ? a.draft[start + i] : -1;
}

__global__ void __launch_bounds__(VER_THREADS) blink_verify_sums_kernel(const VerifyArgs a) {
  __shared__ double s_part[VER_WARPS], s_table[16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int req = (int)(blockIdx.x / (unsigned)a.parts), part = (int)(blockIdx.x - (unsigned)req * a.parts);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const float T = a.temperature[req];
  ver_table(s_table, a);
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const VerChoice c = a.choice[req];
  if (c.row < 0) return;
  const int at = part * VER_PART + warp * VER_RUN;   // this warp's run of the row
  float z[VER_FEW];
  ver_load(z, a.logits + c.row * a.logits_stride + at, a.vocab - at, a.vec, -INFINITY);
  const VerExp x = ver_exp_of(s_table, c.max, T);
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < VER_FEW; i += 2) s += ver_exp(x, z[i]) + ver_exp(x, z[i + 1]);
#pragma unroll
  for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  if (lane == 0) s_part[warp] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
#pragma unroll
    for (int w = 0; w < VER_WARPS; ++w) s += s_part[w];
    a.sums[(size_t)req * a.parts + part] = s;
  }
}

// What a token is drawn from: p - q where a draft was refused (what is no number or negative in q counts as 0), p otherwise.
struct VerWeights {
  const float *z, *q;   // the row, and that of q (null: none)
  int x;                // the entry that a certain draft takes out (-1: none)
  VerExp exp;
  double inv_sum;
};
// The row's sum of exponentials, by a whole warp.
__device__ __forceinline__ double ver_sum(const VerifyArgs& a, int req) {
  double s = 0.0;
#pragma unroll 4
  for (int j = threadIdx.x & 31; j < a.parts; j += 32) s += a.sums[(size_t)req * a.parts + j];
#pragma unroll
  for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  return s;
}
// Entries at + 4 lane + 128 g + j of a run, in 64 bits, and the sum of p over the lane's.
__device__ __forceinline__ void ver_weights(const VerWeights& w, int at, const float (&z)[VER_FEW], const float (&q)[VER_FEW], double (&e)[VER_FEW], double& all) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < VER_FEW; ++i) {
    const double p = ver_exp(w.exp, z[i]) * w.inv_sum;
    all += p;
    if (w.q) e[i] = q[i] > 0.f ? fmax(p - (double)q[i], 0.0) : p;
    else e[i] = at + lane * 4 + (i >> 2) * 128 + (i & 3) == w.x ? 0.0 : p;
  }
}

// The first of `count` values, in order, at which the running sum exceeds target, else the last with anything in it; `base`
// grows by what stands before it.  By one warp.
template <typename F>
__device__ __forceinline__ int ver_find(F value, int count, double target, double& base) {
  const int lane = threadIdx.x & 31;
  int last = 0;
  double last_base = base;
  for (int j0 = 0; j0 < count; j0 += 32) {
    const double v = j0 + lane < count ? value(j0 + lane) : 0.0;
    double c = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const double u = __shfl_up_sync(0xffffffffu, c, d);
      if (lane >= d) c += u;
    }
    const double up = __shfl_up_sync(0xffffffffu, c, 1), before = base + (lane ? up : 0.0);
    const unsigned hit = __ballot_sync(0xffffffffu, v > 0.0 && base + c > target), any = __ballot_sync(0xffffffffu, v > 0.0);
    const int l = hit ? __ffs(hit) - 1 : any ? 31 - __clz(any) : 0;
    const double at = __shfl_sync(0xffffffffu, before, l);
    if (hit) {
      base = at;
      return j0 + l;
    }
    if (any) {
      last = j0 + l;
      last_base = at;
    }
    base += __shfl_sync(0xffffffffu, c, 31);
  }
  base = last_base;
  return last;
}

// Of the request's chosen row, all but its sum; false: nothing is drawn.
__device__ __forceinline__ bool ver_choice(const VerifyArgs& a, int req, const double* table, float T, VerWeights& w, int& row) {
  const VerChoice c = a.choice[req];
  row = c.row;
  if (c.row < 0) return false;
  w.z = a.logits + c.row * a.logits_stride;
  w.q = c.refused && a.probs ? a.probs + c.row * a.probs_stride : nullptr;
  w.x = c.refused && !a.probs ? a.draft[c.row] : -1;
  w.exp = ver_exp_of(table, c.max, T);
  return true;
}

__global__ void __launch_bounds__(VER_THREADS) blink_verify_weights_kernel(const VerifyArgs a) {
  __shared__ VerRun s_run[VER_WARPS];
  __shared__ double s_inv, s_table[16];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int req = (int)(blockIdx.x / (unsigned)a.parts), part = (int)(blockIdx.x - (unsigned)req * a.parts);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  VerWeights w;
  const float T = a.temperature[req];
  ver_table(s_table, a);
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int row;
  if (!ver_choice(a, req, s_table, T, w, row)) return;
  const int at = part * VER_PART + warp * VER_RUN;
  float z[VER_FEW], q[VER_FEW];
  ver_load(z, w.z + at, a.vocab - at, a.vec, -INFINITY);
  if (w.q) ver_load(q, w.q + at, a.vocab - at, a.probs_vec, 0.f);
  if (warp == 0) {
    const double s = ver_sum(a, req);
    if (lane == 0) s_inv = 1.0 / s;
  }
  __syncthreads();
  w.inv_sum = s_inv;
  double rest = 0.0, all = 0.0, e[VER_FEW];
  ver_weights(w, at, z, q, e, all);
#pragma unroll
  for (int i = 0; i < VER_FEW; i += 2) rest += e[i] + e[i + 1];
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    rest += __shfl_xor_sync(0xffffffffu, rest, d);
    all += __shfl_xor_sync(0xffffffffu, all, d);
  }
  if (lane == 0) s_run[warp] = a.runs[((size_t)req * a.parts + part) * VER_WARPS + warp] = VerRun{rest, all};
  __syncthreads();
  if (threadIdx.x == 0) {
    VerRun r = {0.0, 0.0};
#pragma unroll
    for (int i = 0; i < VER_WARPS; ++i) {
      r.rest += s_run[i].rest;
      r.all += s_run[i].all;
    }
    a.part_runs[(size_t)req * a.parts + part] = r;
  }
}

__global__ void __launch_bounds__(32) blink_verify_draw_kernel(const VerifyArgs a) {
  __shared__ double s_table[16];
  const int lane = threadIdx.x, req = (int)blockIdx.x;
  const float T = a.temperature[req], u = a.u_pick[req];
  VerWeights w;
  ver_table(s_table, a);
  __syncwarp();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int row;
  if (!ver_choice(a, req, s_table, T, w, row)) return;
  w.inv_sum = 1.0 / ver_sum(a, req);
  const VerRun* r = a.part_runs + (size_t)req * a.parts;
  double total = 0.0, total_all = 0.0;
#pragma unroll 4
  for (int j = lane; j < a.parts; j += 32) {
    total += r[j].rest;
    total_all += r[j].all;
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    total += __shfl_xor_sync(0xffffffffu, total, d);
    total_all += __shfl_xor_sync(0xffffffffu, total_all, d);
  }
  const bool none = !(total > 0.0);   // q covers p everywhere: from p itself
  if (none) {
    w.q = nullptr;
    w.x = -1;
    total = total_all;
  }
  const double target = (double)u * total;
  double base = 0.0;
  const int in = ver_find([&](int j) { return none ? r[j].all : r[j].rest; }, a.parts, target, base);
  r = a.runs + ((size_t)req * a.parts + in) * VER_WARPS;
  const int run = ver_find([&](int j) { return none ? r[j].all : r[j].rest; }, VER_WARPS, target, base);
  int token = -1, last = 0;
  const int from = in * VER_PART + run * VER_RUN;
  float z[VER_FEW], q[VER_FEW];
  double e[VER_FEW], all = 0.0;
  ver_load(z, w.z + from, a.vocab - from, a.vec, -INFINITY);
  if (w.q) ver_load(q, w.q + from, a.vocab - from, a.probs_vec, 0.f);
  ver_weights(w, from, z, q, e, all);
  double sum[VER_FEW / 4];   // running sums over the lanes, of each group of 128
#pragma unroll
  for (int g = 0; g < VER_FEW / 4; ++g) sum[g] = (e[4 * g] + e[4 * g + 1]) + (e[4 * g + 2] + e[4 * g + 3]);
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
#pragma unroll
    for (int g = 0; g < VER_FEW / 4; ++g) {
      const double x = __shfl_up_sync(0xffffffffu, sum[g], d);
      if (lane >= d) sum[g] += x;
    }
  }
#pragma unroll
  for (int g = 0; g < VER_FEW / 4; ++g) {
    const double up = __shfl_up_sync(0xffffffffu, sum[g], 1);
    double running = lane ? base + up : base;
    int hit = 4, some = -1;   // of the lane's four
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      running += e[4 * g + j];
      if (e[4 * g + j] > 0.0) {
        some = j;
        if (hit == 4 && running > target) hit = j;
      }
    }
    const unsigned hits = __ballot_sync(0xffffffffu, hit < 4), any = __ballot_sync(0xffffffffu, some >= 0);
    const int l = hits ? __ffs(hits) - 1 : any ? 31 - __clz(any) : 0;
    const int h = __shfl_sync(0xffffffffu, hit, l), o = __shfl_sync(0xffffffffu, some, l);
    if (token < 0) {
      if (hits) token = from + g * 128 + l * 4 + h;
      else if (any) last = from + g * 128 + l * 4 + o;
    }
    base += __shfl_sync(0xffffffffu, sum[g], 31);
  }
  if (lane == 0) a.tokens[row] = token >= 0 ? token : last;
}

struct VerifySpace {
  uint64_t chunks, sums, runs, part_runs, choice, end;
  int64_t n_chunks, n_parts;
};
static VerifySpace verify_space(int64_t rows, int64_t n, int64_t vocab) {
  VerifySpace s;
  s.n_chunks = (vocab + VER_CHUNK - 1) / VER_CHUNK;
  s.n_parts = (vocab + VER_PART - 1) / VER_PART;
  s.chunks = 0;
  s.sums = s.chunks + (uint64_t)(rows * s.n_chunks) * sizeof(VerChunk);
  s.runs = (s.sums + (uint64_t)(n * s.n_parts) * 8 + 15) / 16 * 16;
  s.part_runs = s.runs + (uint64_t)(n * s.n_parts * VER_WARPS) * sizeof(VerRun);
  s.choice = s.part_runs + (uint64_t)(n * s.n_parts) * sizeof(VerRun);
  s.end = s.choice + (uint64_t)n * sizeof(VerChoice);
  return s;
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
  using namespace blink;
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
  a.chunks_of = reinterpret_cast<VerChunk*>(ws + space.chunks);
  a.sums = reinterpret_cast<double*>(ws + space.sums);
  a.runs = reinterpret_cast<VerRun*>(ws + space.runs);
  a.part_runs = reinterpret_cast<VerRun*>(ws + space.part_runs);
  a.choice = reinterpret_cast<VerChoice*>(ws + space.choice);
  a.n = n_requests;
  a.rows = rows;
  a.vocab = vocab;
  a.chunks = (int)space.n_chunks;
  a.groups = (int)((space.n_chunks + VER_WARPS - 1) / VER_WARPS);
  a.parts = (int)space.n_parts;
  for (int i = 0; i < 16; ++i) a.sixteenths[i] = std::exp2(i / 16.0);
  a.vec = logits_stride % 4 == 0 && ops_aligned(logits, 16);
  a.probs_vec = draft_probs && probs_stride % 4 == 0 && ops_aligned(draft_probs, 16);
  int rc = ops_launch(blink_verify_rows_kernel, (int64_t)rows * a.groups, VER_THREADS, 0, stream, 0, false, a);
  if (rc == BLINK_OK) rc = ops_launch(blink_verify_choose_kernel, n_requests, VER_THREADS, 0, stream, 0, true, a);
  if (rc == BLINK_OK) rc = ops_launch(blink_verify_sums_kernel, (int64_t)n_requests * a.parts, VER_THREADS, 0, stream, 0, true, a);
  if (rc == BLINK_OK) rc = ops_launch(blink_verify_weights_kernel, (int64_t)n_requests * a.parts, VER_THREADS, 0, stream, 0, true, a);
  if (rc == BLINK_OK) rc = ops_launch(blink_verify_draw_kernel, n_requests, 32, 0, stream, 0, true, a);
  return rc;
}

}  // extern "C"
