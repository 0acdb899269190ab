// Drafted tokens held against the target's probabilities: blink_verify_drafts.
//
//   p_i = softmax(logits_i / T);  draft x_i is accepted while u_i * q_i(x_i) < p_i(x_i)
//   first refused i: a token from max(0, p_i - q_i), none refused: from p of the last row; by the inverse of its running sum in the order of
//   the indexes: the first j with sum_{<= j} > v * sum
//
// Two kernels.  (1) Largest value, its index and the sum of exponentials of every chunk of every row: one pass over the logits, which is what
// bounds the whole (HBM: 4 bytes an entry).  Exponentials in 32 bits, sums of a thread's entries in 32, everything above in 64: the
// acceptance test is off by some 1e-8.  (2) A cluster of eight CTAs a request: the chunks become rows, the first refused draft is found, and
// its row alone is drawn from.  That row's sums decide between neighbours that are as close as 1e-6, so its exponentials, sums and the running sum
// are in 64 bits; a CTA keeps its eighth of them in shared memory, and sums go from CTA to CTA through distributed shared memory.  Sums
// are taken in an order that sizes alone fix: the same call gives the same token.
#include <cooperative_groups.h>

#include <cmath>

#include "ops.h"

namespace blink {

constexpr int VER_THREADS = 256, VER_EACH = 16, VER_CHUNK = VER_THREADS * VER_EACH;   // (1)
constexpr int PICK_THREADS = 512, PICK_WARPS = PICK_THREADS / 32, PICK_CTAS = 8;      // (2)
constexpr int PICK_SMEM = 200 * 1024;   // exponentials of up to 8 * 25600 entries are kept

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
  int n, rows, vocab, chunks, kept;
};

// No number: as if the entry were not there.
__device__ __forceinline__ float ver_entry(float z) { return z == z ? z : -INFINITY; }

// The larger of two, of equal ones that of the lower index.
__device__ __forceinline__ void ver_larger(float& m, int& i, float m2, int i2) {
  if (m2 > m || (m2 == m && i2 < i)) { m = m2; i = i2; }
}

template <bool VEC>
__global__ void __launch_bounds__(VER_THREADS) blink_verify_rows_kernel(const VerifyArgs a) {
  __shared__ float s_m[VER_THREADS / 32];
  __shared__ int s_i[VER_THREADS / 32], s_req;
  __shared__ double s_sum[VER_THREADS / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = (int)(blockIdx.x / (unsigned)a.chunks), chunk = (int)(blockIdx.x - (unsigned)row * a.chunks);
  const float* z = a.logits + row * a.logits_stride + (long long)chunk * VER_CHUNK;
  const int n = min(VER_CHUNK, a.vocab - chunk * VER_CHUNK);
  float v[VER_EACH];
#pragma unroll
  for (int k = 0; k < VER_EACH / 4; ++k) {
    const int at = (k * VER_THREADS + tid) * 4;
    if (VEC && at + 4 <= n) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(z + at));   // (the chosen row is read again, from L2)
      v[4 * k] = x.x; v[4 * k + 1] = x.y; v[4 * k + 2] = x.z; v[4 * k + 3] = x.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * k + j] = at + j < n ? __ldcg(z + at + j) : -INFINITY;
    }
  }
  if (tid == 0) s_req = -1;
  __syncthreads();
  for (int r = tid; r < a.n; r += VER_THREADS)
    if (a.row_start[r] <= row && row < a.row_start[r + 1]) s_req = r;
  float m = -INFINITY;
  int idx = 0x7fffffff;
#pragma unroll
  for (int k = 0; k < VER_EACH; ++k) {
    v[k] = ver_entry(v[k]);
    const int at = ((k >> 2) * VER_THREADS + tid) * 4 + (k & 3);
    if (v[k] > m || idx == 0x7fffffff) { m = v[k]; idx = at; }   // ascending
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, d);
    const int i2 = __shfl_xor_sync(0xffffffffu, idx, d);
    ver_larger(m, idx, m2, i2);
  }
  if (lane == 0) { s_m[warp] = m; s_i[warp] = idx; }
  __syncthreads();
  const int req = s_req;
  if (req < 0) return;   // a row behind the last request
#pragma unroll
  for (int w = 0; w < VER_THREADS / 32; ++w) ver_larger(m, idx, s_m[w], s_i[w]);
  const float T = a.temperature[req];
  double sum = 0.0;
  if (T > 0.f && T < INFINITY && m > -INFINITY && m < INFINITY) {
    const float scale = fminf(1.4426950408889634f / T, 3e38f);
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < VER_EACH; ++k) s += exp2f((v[k] - m) * scale);   // (behind the end: exp2(-inf))
    sum = (double)s;
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < VER_THREADS / 32; ++w) sum += s_sum[w];
  }
  if (tid == 0) a.chunks_of[(size_t)row * a.chunks + chunk] = VerChunk{sum, m, chunk * VER_CHUNK + idx};
}

__global__ void __launch_bounds__(PICK_THREADS) blink_verify_pick_kernel(const VerifyArgs a) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  extern __shared__ double s_e[];            // exp((z - max) / T) of this CTA's entries, when they fit
  __shared__ double s_part[PICK_WARPS];      // a sum per warp
  __shared__ double s_all[2][PICK_CTAS];     // a sum per CTA, the same in all of them
  __shared__ int s_first, s_index, s_one;
  __shared__ float s_max;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cluster.block_rank(), req = (int)(blockIdx.x / PICK_CTAS);
  const int V = a.vocab;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int start = min(max(a.row_start[req], 0), a.rows), end = min(max(a.row_start[req + 1], start), a.rows);
  if (start == end) {   // (the whole cluster)
    if (rank == 0 && tid == 0) a.accepted[req] = 0;
    return;
  }
  const int k = end - start - 1;
  const float T = a.temperature[req];
  const double inv_T = 1.0 / (double)T;

  // A row from its chunks: largest value, its index, sum.  A row with an infinite largest value or without any number, and every
  // row at a T that is not above 0 and finite, stands for its largest entry alone.
  auto row_of = [&](int row, float& m, int& idx, double& sum) {
    const VerChunk* c = a.chunks_of + (size_t)row * a.chunks;
    m = -INFINITY;
    idx = 0x7fffffff;
    for (int j = lane; j < a.chunks; j += 32) ver_larger(m, idx, c[j].max, c[j].index);
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      const float m2 = __shfl_xor_sync(0xffffffffu, m, d);
      const int i2 = __shfl_xor_sync(0xffffffffu, idx, d);
      ver_larger(m, idx, m2, i2);
    }
    const bool one = !(T > 0.f && T < INFINITY) || !(m > -INFINITY) || !(m < INFINITY);
    sum = 0.0;
    if (!one) {
      for (int j = lane; j < a.chunks; j += 32) sum += c[j].max > -INFINITY ? c[j].sum * exp(((double)c[j].max - (double)m) * inv_T) : 0.0;
#pragma unroll
      for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    }
    return one;
  };
  if (tid == 0) s_first = k;
  __syncthreads();
  for (int i = warp; i < k; i += PICK_WARPS) {
    float m;
    int idx;
    double sum;
    const int row = start + i, x = a.draft[row];
    const bool one = row_of(row, m, idx, sum);
    bool ok = false;
    if (one) ok = x == idx;
    else if (x >= 0 && x < V) {
      const float z = ver_entry(__ldcg(a.logits + row * a.logits_stride + x));
      const double p = exp(((double)z - (double)m) * inv_T);   // times sum
      const double q = a.probs ? (double)a.probs[row * a.probs_stride + x] : 1.0;
      ok = (double)a.u_accept[row] * q * sum < p;
    }
    if (lane == 0 && !ok) atomicMin(&s_first, i);
  }
  __syncthreads();
  const int acc = s_first, row = start + acc;
  if (warp == 0) {
    float m;
    int idx;
    double sum;
    const bool one = row_of(row, m, idx, sum);
    if (lane == 0) { s_one = one; s_max = m; s_index = idx; }
  }
  __syncthreads();
  if (rank == 0) {
    if (tid == 0) a.accepted[req] = acc;
    for (int i = tid; i <= k; i += PICK_THREADS)
      if (i != acc) a.tokens[start + i] = i < acc ? a.draft[start + i] : -1;
  }
  if (s_one) {
    if (rank == 0 && tid == 0) a.tokens[row] = s_index;
    return;
  }

  cluster.sync();   // all CTAs are there to be written to
  // the row's sum: this CTA's entries [lo, hi), a run of them per warp
  const double m = (double)s_max;
  const float* z = a.logits + row * a.logits_stride;
  const int per = ((V + PICK_CTAS - 1) / PICK_CTAS + 31) & ~31, run = ((per + PICK_WARPS - 1) / PICK_WARPS + 31) & ~31;
  const int lo = min(V, rank * per), hi = min(V, lo + per);
  const int w0 = min(hi, lo + warp * run), w1 = min(hi, w0 + run);
  const bool kept = a.kept != 0;
  auto e_of = [&](int j) { return exp(((double)ver_entry(__ldcg(z + j)) - m) * inv_T); };
  // sum over the warp's run -> over the CTA -> over the cluster; s_part keeps the warps', s_all the CTAs'
  auto sum_all = [&](double s, int which) {
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    __syncthreads();
    if (lane == 0) s_part[warp] = s;
    __syncthreads();
    if (tid < PICK_CTAS) {
      double t = 0.0;
      for (int w = 0; w < PICK_WARPS; ++w) t += s_part[w];
      *cluster.map_shared_rank(&s_all[which][rank], tid) = t;
    }
    cluster.sync();
    double t = 0.0;
    for (int c = 0; c < PICK_CTAS; ++c) t += s_all[which][c];
    return t;
  };
  double s = 0.0;
  for (int j = w0 + lane; j < w1; j += 32) {
    const double e = e_of(j);
    if (kept) s_e[j - lo] = e;
    s += e;
  }
  const double inv_S = 1.0 / sum_all(s, 0);

  // what is drawn from: p - q where a draft was refused (what is no number or negative in q counts as 0), p otherwise
  const float* q = acc < k && a.probs ? a.probs + row * a.probs_stride : nullptr;
  int x = acc < k && !a.probs ? a.draft[row] : -1;
  auto rest_of = [&](int j) {
    const double p = (kept ? s_e[j - lo] : e_of(j)) * inv_S;
    if (q) {
      const float t = __ldg(q + j);
      return t > 0.f ? fmax(p - (double)t, 0.0) : p;
    }
    return j == x ? 0.0 : p;
  };
  auto rest_sum = [&]() {
    double t = 0.0;
    for (int j = w0 + lane; j < w1; j += 32) t += rest_of(j);
    return sum_all(t, 1);
  };
  double total = rest_sum();
  if (!(total > 0.0)) {   // q covers p everywhere: from p itself
    q = nullptr;
    x = -1;
    cluster.sync();       // (everybody has read the sums)
    total = rest_sum();
  }
  const double target = (double)a.u_pick[req] * total;
  // the CTA, and the warp in it, whose run takes the sum past the target; else the last with anything in it
  int cta = -1, last_cta = 0;
  double before = 0.0, base = 0.0, last_base = 0.0;
  for (int c = 0; c < PICK_CTAS; ++c) {
    const double t = s_all[1][c];
    if (t > 0.0) {
      last_cta = c;
      last_base = before;
      if (cta < 0 && before + t > target) { cta = c; base = before; }
    }
    before += t;
  }
  if (cta < 0) { cta = last_cta; base = last_base; }
  if (cta == rank) {
    int w = -1, last_w = 0;
    double at = base, w_base = base, last_w_base = base;
    for (int c = 0; c < PICK_WARPS; ++c) {
      const double t = s_part[c];
      if (t > 0.0) {
        last_w = c;
        last_w_base = at;
        if (w < 0 && at + t > target) { w = c; w_base = at; }
      }
      at += t;
    }
    if (w < 0) { w = last_w; w_base = last_w_base; }
    if (w == warp) {
      int token = -1, last = w0;
      for (int j0 = w0; j0 < w1 && token < 0; j0 += 32) {
        const int j = j0 + lane;
        const double r = j < w1 ? rest_of(j) : 0.0;
        double c = r;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const double u = __shfl_up_sync(0xffffffffu, c, d);
          if (lane >= d) c += u;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, r > 0.0 && w_base + c > target), some = __ballot_sync(0xffffffffu, r > 0.0);
        if (hit) token = j0 + __ffs(hit) - 1;
        else if (some) last = j0 + 31 - __clz(some);
        w_base += __shfl_sync(0xffffffffu, c, 31);
      }
      if (lane == 0) a.tokens[row] = token >= 0 ? token : last;
    }
  }
  cluster.sync();   // nobody leaves while another may still write into its shared memory
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
  const int64_t slice = (((int64_t)vocab + PICK_CTAS - 1) / PICK_CTAS + 31) & ~31ll;
  a.kept = slice * 8 <= PICK_SMEM;
  const bool vec = logits_stride % 4 == 0 && ops_aligned(logits, 16);
  const int64_t grid = (int64_t)rows * a.chunks;
  int rc = ops_launch(vec ? blink_verify_rows_kernel<true> : blink_verify_rows_kernel<false>, grid, VER_THREADS, 0, stream, 0, false, a);
  if (rc != BLINK_OK) return rc;
  return ops_launch(blink_verify_pick_kernel, (int64_t)n_requests * PICK_CTAS, PICK_THREADS, a.kept ? (size_t)slice * 8 : 0, stream, PICK_CTAS, true, a);
}

}  // extern "C"
