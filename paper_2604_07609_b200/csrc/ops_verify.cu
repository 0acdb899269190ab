// Drafted tokens held against the target's probabilities: blink_verify_drafts.
//
//   p_i = softmax(logits_i / T);  draft x_i is accepted while u_i * q_i(x_i) < p_i(x_i)
//   first refused i: a token from max(0, p_i - q_i), none refused: from p of the last row; by the inverse of its running sum in the order of
//   the indexes: the first j with sum_{<= j} > v * sum
//
// Two kernels.  (1) Largest value, its index and the sum of exponentials of pieces of 1024 entries of every row, a warp each: one pass over
// the logits, which is what bounds the whole (HBM: 4 bytes an entry).  A lane has its 32 entries on their way at once, and sums against its own
// largest, so that nothing waits for another warp.  Exponentials in 32 bits, sums of a lane's entries in 32, everything above in 64: the
// acceptance test is off by some 1e-8.  (2) A cluster of 16 CTAs a request: pieces become rows, the first refused draft is found, and
// its row alone is drawn from.  That row's sums decide between neighbours that are as close as 1e-6, so its exponentials, sums and the running
// sum are in 64 bits; a thread keeps its 16 of them in registers, and sums go from CTA to CTA through distributed shared memory.  Sums
// are taken in an order that sizes alone fix: the same call gives the same token.
#include <cooperative_groups.h>

#include <utility>

#include "ops.h"

namespace blink {

constexpr int VER_WARPS = 8, VER_EACH = 32, VER_CHUNK = 32 * VER_EACH;                             // (1): entries of a lane, of a warp
constexpr int PICK_THREADS = 512, PICK_WARPS = 16, PICK_CTAS = 16;   // (2)
constexpr int PICK_ROWS = 64;   // rows of a request whose largest values are kept until it is known which one is drawn from

struct VerChunk {
  double sum;   // of exp((z - max) / T)
  float max;
  int index;    // first of the largest
};

struct VerifyArgs {
  const float* logits;
  const float* probs;
  long long logits_stride, probs_stride;
  const int32_t *row_start, *draft;
  const float *temperature, *u_accept, *u_pick;
  int32_t *tokens, *accepted;
  VerChunk* chunks_of;   // [rows][chunks]
  int n, rows, vocab, chunks;
  bool vec, probs_vec;   // rows on 16-byte boundaries
};

// No number: as if the entry were not there.
__device__ __forceinline__ float ver_entry(float z) { return z == z ? z : -INFINITY; }

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

__global__ void __launch_bounds__(VER_WARPS * 32) blink_verify_rows_kernel(const VerifyArgs a) {
  __shared__ int s_req;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int groups = (a.chunks + VER_WARPS - 1) / VER_WARPS;
  const int row = (int)(blockIdx.x / (unsigned)groups), chunk = (int)(blockIdx.x - (unsigned)row * groups) * VER_WARPS + warp;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (the second kernel waits for the whole of this one itself)
  float v[VER_EACH];
  if (chunk < a.chunks)
    ver_load(v, a.logits + row * a.logits_stride + (long long)chunk * VER_CHUNK, min(VER_CHUNK, a.vocab - chunk * VER_CHUNK), a.vec, -INFINITY);
  if (threadIdx.x == 0) s_req = -1;
  __syncthreads();
  for (int r = threadIdx.x; r < a.n; r += VER_WARPS * 32)
    if (a.row_start[r] <= row && row < a.row_start[r + 1]) s_req = r;
  __syncthreads();
  const int req = s_req;
  if (req < 0 || chunk >= a.chunks) return;   // (whole warps) a row behind the last request
  const float T = a.temperature[req];
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < VER_EACH; ++k) {
    v[k] = ver_entry(v[k]);
    m = fmaxf(m, v[k]);
  }
  int idx = 0;
#pragma unroll
  for (int k = VER_EACH - 1; k >= 0; --k)
    if (v[k] == m) idx = (k >> 2) * 128 + lane * 4 + (k & 3);
  const float mine = m;
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, d);
    const int i2 = __shfl_xor_sync(0xffffffffu, idx, d);
    ver_larger(m, idx, m2, i2);
  }
  double sum = 0.0;
  if (T > 0.f && T < INFINITY && m > -INFINITY && m < INFINITY) {
    const float scale = fminf(1.4426950408889634f / T, 3e38f);
    const float base = mine == -INFINITY ? 0.f : mine;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int k = 0; k < VER_EACH; k += 2) {   // (no entry: exp2(-inf))
      s0 += exp2f((v[k] - base) * scale);
      s1 += exp2f((v[k + 1] - base) * scale);
    }
    sum = (double)(s0 + s1) * (double)exp2f((mine - m) * scale);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  }
  if (lane == 0) a.chunks_of[(size_t)row * a.chunks + chunk] = VerChunk{sum, m, chunk * VER_CHUNK + idx};
}

// 2^t for t <= 0 in 64 bits: the whole part into the exponent, the rest, at most half, by the series of exp(f ln 2) up to its tenth power
// (off by (ln 2 / 2)^11 / 11! = 2e-13).  Below 2^-1020: 0.
__device__ __forceinline__ double ver_exp2(double t) {
  constexpr double L = 0.693147180559945309417;
  constexpr double C2 = L * L / 2, C3 = C2 * L / 3, C4 = C3 * L / 4, C5 = C4 * L / 5, C6 = C5 * L / 6, C7 = C6 * L / 7, C8 = C7 * L / 8, C9 = C8 * L / 9,
                   C10 = C9 * L / 10;
  constexpr double SHIFT = 6755399441055744.0;   // 1.5 * 2^52: adding it leaves the nearest whole number in the low bits
  const double s = t + SHIFT, f = t - (s - SHIFT), f2 = f * f;
  const int n = __double2loint(s);
  const double a = fma(f2, fma(f2, fma(f2, fma(f2, C10, C8), C6), C4), C2), b = fma(f2, fma(f2, fma(f2, fma(f2, C9, C7), C5), C3), L);
  const double p = fma(f, b, fma(f2, a, 1.0));   // even and odd powers side by side
  return t > -1020.0 ? __hiloint2double(__double2hiint(p) + (n << 20), __double2loint(p)) : 0.0;
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

// EACH: entries of a lane at a time.
template <int EACH>
__global__ void __launch_bounds__(PICK_THREADS, 2) blink_verify_pick_kernel(const VerifyArgs a) {
  namespace cg = cooperative_groups;
  constexpr int TILE = 32 * EACH;
  cg::cluster_group cluster = cg::this_cluster();
  __shared__ __align__(16) float s_q[PICK_WARPS][TILE];   // a tile of q per warp, each lane's own entries
  __shared__ double s_part[PICK_WARPS];                   // a sum per warp
  __shared__ double s_all[2][PICK_CTAS];                  // a sum per CTA, the same in all of them
  __shared__ int s_first, s_one[PICK_ROWS], s_index[PICK_ROWS];
  __shared__ float s_max[PICK_ROWS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster.block_rank(), req = (int)(blockIdx.x / PICK_CTAS);
  const int V = a.vocab;
  // (all but the pieces is there before the first kernel is done)
  const int start = min(max(a.row_start[req], 0), a.rows), end = min(max(a.row_start[req + 1], start), a.rows);
  const int k = end - start - 1;
  const float T = a.temperature[req];
  const double to_exp2 = 1.44269504088896340736 / (double)T;
  if (tid == 0) s_first = k;
  __syncthreads();
  if (start == end) {   // (the whole cluster; not before the first kernel, or the next one in the stream could be)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (rank == 0 && tid == 0) a.accepted[req] = 0;
    return;
  }

  // A row from its pieces: largest value, its index, sum.  A row with an infinite largest value or without any number, and every
  // row at a T that is not above 0 and finite, stands for its largest entry alone.
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
    const bool one = !(T > 0.f && T < INFINITY) || !(m > -INFINITY) || !(m < INFINITY);
    sum = 0.0;
    if (!one && with_sum) {
#pragma unroll 4
      for (int j = lane; j < a.chunks; j += 32) sum += c[j].max > -INFINITY ? c[j].sum * ver_exp2(((double)c[j].max - (double)m) * to_exp2) : 0.0;
#pragma unroll
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    }
    return one;
  };
  for (int i = warp; i <= k; i += PICK_WARPS) {   // (row k: no draft)
    float m;
    int idx;
    double sum;
    const int row = start + i, x = i < k ? a.draft[row] : -1;
    const bool in = x >= 0 && x < V;
    const float z = in ? ver_entry(__ldcg(a.logits + row * a.logits_stride + x)) : -INFINITY, q = in && a.probs ? a.probs[row * a.probs_stride + x] : 1.f;
    const float u = a.u_accept[row];
    if (i == warp) asm volatile("griddepcontrol.wait;" ::: "memory");
    const bool one = row_of(row, m, idx, sum, i < k);
    const bool ok = i == k || (one ? x == idx : in && (double)u * (double)q * sum < ver_exp2(((double)z - (double)m) * to_exp2));
    if (lane == 0) {
      if (i < PICK_ROWS) {
        s_one[i] = one;
        s_max[i] = m;
        s_index[i] = idx;
      }
      if (!ok) atomicMin(&s_first, i);
    }
  }
  if (warp > k) asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncthreads();
  const int acc = s_first, row = start + acc;
  // the row's entries: a run of tiles per warp, in the order of CTAs, warps and tiles
  const int tiles = (V + PICK_CTAS * PICK_WARPS * TILE - 1) / (PICK_CTAS * PICK_WARPS * TILE);
  const int w0 = (rank * PICK_WARPS + warp) * tiles * TILE;
  const float* z = a.logits + row * a.logits_stride;
  const float* q = acc < k && a.probs ? a.probs + row * a.probs_stride : nullptr;
  float zv[EACH];   // of the warp's first tile
  ver_load(zv, z + w0, V - w0, a.vec, -INFINITY);
  auto fetch_q = [&](int at) {
#pragma unroll
    for (int g = 0; g < EACH / 4; ++g) {
      const int o = g * 128 + lane * 4;
      const uint32_t dst = (uint32_t)__cvta_generic_to_shared(&s_q[warp][o]);
      if (a.probs_vec && at + o + 4 <= V) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(q + at + o) : "memory");
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (at + o + j < V) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + 4 * j), "l"(q + at + o + j) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (q) fetch_q(w0);
  if (rank == 0) {
    if (tid == 0) a.accepted[req] = acc;
    for (int i = tid; i <= k; i += PICK_THREADS)
      if (i != acc) a.tokens[start + i] = i < acc ? a.draft[start + i] : -1;
  }
  float top;
  int index;
  bool one;
  if (acc < PICK_ROWS) {
    top = s_max[acc];
    index = s_index[acc];
    one = s_one[acc] != 0;
  } else {
    double sum;
    one = row_of(row, top, index, sum, false);
  }
  if (one) {
    if (rank == 0 && tid == 0) a.tokens[row] = index;
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    return;
  }
  cg::cluster_group::arrival_token there = cluster.barrier_arrive();   // all CTAs have to be there before they are written to

  const double m = (double)top;
  double e[EACH];
  auto exps = [&]() {
#pragma unroll
    for (int i = 0; i < EACH; ++i) e[i] = ver_exp2(((double)ver_entry(zv[i]) - m) * to_exp2);
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
  const double inv_S = 1.0 / sum_all(s, 0);

  // what is drawn from: p - q where a draft was refused (what is no number or negative in q counts as 0), p otherwise
  int x = acc < k && !a.probs ? a.draft[row] : -1;
  auto rests = [&](int t) {   // of tile t, whose exponentials are in e
    const int at = w0 + t * TILE + lane * 4;
    if (q) {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
      for (int i = 0; i < EACH; i += 4) {
        const float4 v = *reinterpret_cast<const float4*>(&s_q[warp][i * 32 + lane * 4]);
        const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const double p = e[i + j] * inv_S;
          e[i + j] = w[j] > 0.f && at + i * 32 + j < V ? fmax(p - (double)w[j], 0.0) : p;   // (behind the end: nothing was fetched, and p is 0)
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const double p = e[i] * inv_S;
        e[i] = at + (i >> 2) * 128 + (i & 3) == x ? 0.0 : p;
      }
    }
  };
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
  const double target = (double)a.u_pick[req] * total;
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

static int64_t verify_chunks(int vocab) { return ((int64_t)vocab + VER_CHUNK - 1) / VER_CHUNK; }

}  // namespace blink

extern "C" {

uint64_t blink_verify_workspace(int rows, int vocab) {
  if (rows < 0 || vocab < 1) return 0;
  return (uint64_t)rows * blink::verify_chunks(vocab) * sizeof(blink::VerChunk);
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
  if (vocab > 0x3fffffff) return BLINK_ETOOBIG;
  if (!ops_aligned(workspace, 16) || workspace_bytes < blink_verify_workspace(rows, vocab)) return BLINK_EINVAL;
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
  a.chunks_of = static_cast<VerChunk*>(workspace);
  a.n = n_requests;
  a.rows = rows;
  a.vocab = vocab;
  a.chunks = (int)verify_chunks(vocab);
  a.vec = logits_stride % 4 == 0 && ops_aligned(logits, 16);
  a.probs_vec = draft_probs && probs_stride % 4 == 0 && ops_aligned(draft_probs, 16);
  const int64_t grid = (int64_t)rows * ((a.chunks + VER_WARPS - 1) / VER_WARPS);
  int rc = ops_launch(blink_verify_rows_kernel, grid, VER_WARPS * 32, 0, stream, 0, false, a);
  if (rc != BLINK_OK) return rc;
  // as few entries of a lane as hold the row in one go: 32768 entries in 16 CTAs of 16 warps with four, 131072 with 16 (beyond that, runs of tiles)
  const int64_t ctas = (int64_t)n_requests * PICK_CTAS;
  if (vocab <= 32768) return ops_launch(blink_verify_pick_kernel<4>, ctas, PICK_THREADS, 0, stream, PICK_CTAS, true, a);
  if (vocab <= 65536) return ops_launch(blink_verify_pick_kernel<8>, ctas, PICK_THREADS, 0, stream, PICK_CTAS, true, a);
  return ops_launch(blink_verify_pick_kernel<16>, ctas, PICK_THREADS, 0, stream, PICK_CTAS, true, a);
}

}  // extern "C"
