// Norms of queries and keys for each head with the position rotation, and the new keys and values into the paged cache, in one pass:
// blink_qk_norm_rope.
//
//   y = x * rsqrt(mean(x^2) + eps) * gain          (per head; without gains y = x)
//   (y_i, y_{i+hd/2}) turned by position * theta^(-2 i / hd)
//   q -> q_out, k -> the pool's key of the row's slot; v -> its value as it is
//
// What bounds it: HBM, every element in once and out once (8B shape: 16000 rows in 16 bits 70 us, 5.6 TB/s; 4099 rows of 32 bits, cold, 31 us, 4.9
// TB/s); 64 rows 6 us, latency.  A lane takes 8 elements of either half of a head, so that the two
// partners of a rotation meet in one thread, loads and stores are 16 bytes, and a head is 8 lanes (head_dim 128; 4 at 64): its sum of
// squares takes three shuffles.  A warp turns U groups of heads of one row; their loads are all on their way before the angles,
// which the warp's lanes share out (two each at most) and pass on through shared memory.  Angles in 64 bits, reduced there to less than
// half a turn: a position times a frequency has more digits than 32 bits hold.  Sums and products in 32 bits, one rounding at the store.
#include <cuda_bf16.h>

#include <cmath>

#include "ops.h"

namespace blink {

constexpr int NR_WARPS = 4;

struct NormRopeArgs {
  OpsPool pool;
  const void* qkv;
  long long qkv_stride, q_stride;   // elements between rows
  const float *q_gain, *k_gain;
  const int32_t *positions, *slot_map;
  void* q_out;
  int rows, slots;                  // slots: of the pool
  float eps;
  double turns[64];                 // theta^(-2 i / hd) / (2 pi)
};

// Eight elements as they come (so that those on their way take no more registers than that), and as numbers.
template <typename T>
struct NrEight {
  uint4 raw[sizeof(T) * 8 / 16];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * 8 / 16); ++i)
      asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(raw[i].x), "=r"(raw[i].y), "=r"(raw[i].z), "=r"(raw[i].w) : "l"(p + i * (16 / (int)sizeof(T))));
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t r[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(r[i] << 16);
        x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[4 * i] = __uint_as_float(raw[i].x);
        x[4 * i + 1] = __uint_as_float(raw[i].y);
        x[4 * i + 2] = __uint_as_float(raw[i].z);
        x[4 * i + 3] = __uint_as_float(raw[i].w);
      }
    }
  }
};
__device__ __forceinline__ void nr_store(__nv_bfloat16* p, const float (&x)[8]) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    r[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(r[0], r[1], r[2], r[3]);
}
__device__ __forceinline__ void nr_store(float* p, const float (&x)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

template <typename TI, typename TO, int HD, int U>
__global__ void __launch_bounds__(NR_WARPS * 32) blink_norm_rope_kernel(const __grid_constant__ NormRopeArgs a) {
  constexpr int HALF = HD / 2, LANES = HALF / 8, GROUP = 32 / LANES;   // lanes of a head, heads of a warp at a time
  __shared__ float2 s_turn[NR_WARPS][HALF];
  ops_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int heads = a.pool.Hq + 2 * a.pool.Hkv, tasks_row = (heads + GROUP * U - 1) / (GROUP * U);
  const long long task = (long long)blockIdx.x * NR_WARPS + warp;
  if (task >= (long long)a.rows * tasks_row) return;   // (whole warps)
  const int row = (int)(task / tasks_row), h0 = (int)(task - (long long)row * tasks_row) * GROUP * U + lane / LANES;
  const int i0 = (lane % LANES) * 8;
  const TI* src = static_cast<const TI*>(a.qkv) + row * a.qkv_stride + i0;
  NrEight<TI> in1[U], in2[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = min(h0 + u * GROUP, heads - 1);   // behind the end: the last head once more, not stored
    in1[u].load(src + h * HD);
    in2[u].load(src + h * HD + HALF);
  }
  const int pos = a.positions[row], slot = a.slot_map[row];
  if (pos < 0) return;
#pragma unroll
  for (int j = 0; j < (HALF + 31) / 32; ++j) {
    const int i = lane + 32 * j;
    const double t = (double)pos * a.turns[i];
    const double r = (t - rint(t)) * 2.0;   // in half turns, -1 .. 1
    const float hi = (float)r, lo = (float)(r - (double)hi) * 3.14159265f;   // (to first order in what 32 bits leave of the angle)
    float s, c;
    sincospif(hi, &s, &c);
    s_turn[warp][i] = make_float2(fmaf(-s, lo, c), fmaf(c, lo, s));
  }
  __syncwarp();
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 t = s_turn[warp][i0 + i];
    c[i] = t.x;
    s[i] = t.y;
  }
  const bool cached = slot >= 0 && slot < a.slots;
  const long long tile = cached ? ((long long)(slot / OPS_BLOCK) * a.pool.Hkv * OPS_BLOCK + slot % OPS_BLOCK) * HD + i0 : 0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = h0 + u * GROUP;
    const bool is_q = h < a.pool.Hq, turn = h < a.pool.Hq + a.pool.Hkv;
    const float* gain = is_q ? a.q_gain : a.k_gain;
    float x1[8], x2[8];
    in1[u].get(x1);
    in2[u].get(x2);
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x1[i], x1[i], fmaf(x2[i], x2[i], ss));
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
    if (h >= heads) continue;
    if (turn) {
      if (gain) {
        const float f = rsqrtf(ss * (1.0f / HD) + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x1[i] *= f * gain[i0 + i];
          x2[i] *= f * gain[HALF + i0 + i];
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = fmaf(x1[i], c[i], -x2[i] * s[i]);
        x2[i] = fmaf(x2[i], c[i], x1[i] * s[i]);
        x1[i] = y;
      }
    }
    TO* dst;
    if (is_q) dst = static_cast<TO*>(a.q_out) + row * a.q_stride + h * HD + i0;
    else if (!cached) continue;
    else dst = reinterpret_cast<TO*>(turn ? a.pool.k : a.pool.v) + tile + (long long)(h - a.pool.Hq - (turn ? 0 : a.pool.Hkv)) * OPS_BLOCK * HD;
    nr_store(dst, x1);
    nr_store(dst + HALF, x2);
  }
}

template <typename TI, typename TO>
int norm_rope_launch(const NormRopeArgs& a, int sms, void* stream) {
  const int heads = a.pool.Hq + 2 * a.pool.Hkv;
  // Few rows: a warp per group of heads, so that a row is spread over as many SMs as it can be.  Many: several groups a warp, which share the
  // row's angles and have more on its way: 1.5 KB a lane's worth in 32 bits or of heads of 64, 3 KB of wide heads in 16 bits.  (16000 rows of the 8B
  // shape, us, with 2 | 3 | 4 | 6 groups: fp32 in 113 | 105 | 105 | 109, bf16 in 92 | 80 | 77 | 72; 4099 rows of the 1B shape in bf16 14.4 | 12.7 | 14.5 | 14.4.)
  const int group = a.pool.hd == 128 ? 4 : 8;
  const bool few = (long long)a.rows * ((heads + group - 1) / group) <= 4ll * sms * 16;
  constexpr int WIDE = sizeof(TI) == 2 ? 6 : 3;
  const int u = few ? 1 : a.pool.hd == 128 ? WIDE : 3;
  const long long tasks = (long long)a.rows * ((heads + group * u - 1) / (group * u));
  const long long grid = (tasks + NR_WARPS - 1) / NR_WARPS;
  if (a.pool.hd == 128)
    return few ? ops_launch(blink_norm_rope_kernel<TI, TO, 128, 1>, grid, NR_WARPS * 32, 0, stream, 0, a)
               : ops_launch(blink_norm_rope_kernel<TI, TO, 128, WIDE>, grid, NR_WARPS * 32, 0, stream, 0, a);
  return few ? ops_launch(blink_norm_rope_kernel<TI, TO, 64, 1>, grid, NR_WARPS * 32, 0, stream, 0, a)
             : ops_launch(blink_norm_rope_kernel<TI, TO, 64, 3>, grid, NR_WARPS * 32, 0, stream, 0, a);
}

}  // namespace blink

extern "C" int blink_qk_norm_rope(const blink_model_cfg* model, const blink_kv_pool* kv, int layer, const void* qkv, int qkv_dtype,
                                  int64_t qkv_stride, const float* q_gain, const float* k_gain, const int32_t* positions,
                                  const int32_t* slot_map, int rows, void* q_out, int64_t q_stride, void* stream) {
  using namespace blink;
  NormRopeArgs a;
  const int rc = ops_pool(model, kv, layer, &a.pool);
  if (rc != BLINK_OK) return rc;
  if (qkv_dtype != BLINK_DTYPE_BF16 && qkv_dtype != BLINK_DTYPE_FP32) return BLINK_EINVAL;
  if (qkv_dtype == BLINK_DTYPE_BF16 && model->dtype != BLINK_DTYPE_BF16) return BLINK_EINVAL;
  const int64_t q_dim = (int64_t)a.pool.Hq * a.pool.hd, dim = q_dim + 2ll * a.pool.Hkv * a.pool.hd;
  if (rows < 0 || !ops_aligned(qkv, 16) || !ops_aligned(q_out, 16) || !ops_aligned(positions, 4) || !ops_aligned(slot_map, 4)) return BLINK_EINVAL;
  if ((q_gain && ((uintptr_t)q_gain & 3)) || (k_gain && ((uintptr_t)k_gain & 3))) return BLINK_EINVAL;
  if (qkv_stride < dim || q_stride < q_dim || qkv_stride % 8 || q_stride % 8) return BLINK_EINVAL;
  if (!(model->rope_theta > 0.f) || !(model->rms_eps >= 0.f)) return BLINK_EINVAL;
  a.qkv = qkv;
  a.qkv_stride = qkv_stride;
  a.q_stride = q_stride;
  a.q_gain = q_gain;
  a.k_gain = k_gain;
  a.positions = positions;
  a.slot_map = slot_map;
  a.q_out = q_out;
  a.rows = rows;
  a.slots = (int)(a.pool.n_blocks * OPS_BLOCK);
  a.eps = model->rms_eps;
  for (int i = 0; i < a.pool.hd / 2; ++i) a.turns[i] = std::pow((double)model->rope_theta, -2.0 * i / a.pool.hd) / 6.283185307179586476925;
  for (int i = a.pool.hd / 2; i < 64; ++i) a.turns[i] = 0.0;
  if (rows == 0) return BLINK_OK;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return BLINK_ECUDA;
  if (qkv_dtype == BLINK_DTYPE_FP32)
    return model->dtype == BLINK_DTYPE_FP32 ? norm_rope_launch<float, float>(a, sms, stream) : norm_rope_launch<float, __nv_bfloat16>(a, sms, stream);
  return norm_rope_launch<__nv_bfloat16, __nv_bfloat16>(a, sms, stream);
}
