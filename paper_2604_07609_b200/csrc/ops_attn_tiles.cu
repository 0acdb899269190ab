// blink_window_attention for requests of many rows (prompts and their chunks), and for batches that are sent here whole (drafts; the rule is beside the
// entry point), on tcgen05.
//
//   s = q k / sqrt(hd) * log2(e) of 128 rows and 128 keys;  p = 2^(s - m), l += sum p,  o += p v;  m follows the largest s;  output o / l
//
// A unit is a request, a kv head and 2 * 128 (query row, head) rows: two streams of 128, the rep heads of the kv head beside one another, so that a
// narrow window wastes little (4 heads: 64 query rows read the keys of their window once).  Keys come in tiles of 128: the visible
// blocks of the unit, sinks first, eight to a tile, whatever lies between them.
//
//   warps 0-7 | 8-15  softmax of stream 0 | 1, two threads per row (64 keys of a tile each): scores from TMEM, probabilities back to TMEM
//                     over the same scores
//   warp 16           issues the MMAs of both streams: scores = Q K^T (operands in shared memory), output += P V (P in TMEM, V as it lies in the
//                     cache)
//   warps 17 | 18     copies of the keys | of the values, eight a tile (with twice as many smaller ones for the keys that warp was the slowest of
//                     all: 4096 rows 170 us, 145 so).  Warp 17 also hands out the units, heaviest of a request first, from a counter
//
// While one stream is in its softmax the tensor core works for the other; the next scores of a stream are issued behind its output MMAs, so a
// stream's scores being complete also says that its accumulator is.  The maximum in use, the same for both threads of a row, follows the
// largest score only when that has grown by more than 2^8 (the sum takes up smaller growth); then the scores, still in TMEM, are gone over once
// more and the accumulator is rescaled.  CTAs are persistent; keys of the next unit are on their way while the last tile of one is worked on.
//
// A unit with rows for one stream only is worked on by both, stream 0 the even tiles and stream 1 the odd ones, and joined in the epilogue:
// stream 0 reads both accumulators, once stream 1 has said that its own is there, with its rows' maxima and sums (48 requests of 12
// rows behind 2500 keys, 8B shape: 128 us with one stream, 97 so; 512 rows behind 3500 keys 70 and 45).
//
// What bounds it.  Prompts: the chain of a stream, softmax -> output -> next scores, of which two overlap: 8192 rows of the 8B shape 504 us, 1090
// TFLOP/s of the pairs that are seen, the tensor pipe busy half of the time.  With one thread per row (eight warps) the softmax alone took 1900 cycles a
// tile, at four cycles an instruction with one warp of a stream on a scheduler.  Exponentials on the multiply-adds (a quarter to a half of
// them, degree 3) made it longer, not shorter: they are not what it waits for.  Few rows: HBM (48 requests of 1 to 6 rows behind 300 to
// 5000 keys 88 us, 5.5 TB/s; those of 8 rows behind 2500 96 us, 5.1), and that units are whole.  Narrow windows: what a unit costs beside its tiles, some 4000
// cycles (4096 rows with a window of 128 38 to 43 us from box to box).
#include <cuda.h>

#include <cmath>

#include "ops_attention.cuh"

namespace blink {

constexpr int TIL_KEYS = 128, TIL_BLOCKS = TIL_KEYS / OPS_BLOCK;
constexpr int TIL_SOFT = 16, TIL_COPY = TIL_SOFT + 1, TIL_K = 1, TIL_WARPS = TIL_COPY + TIL_K + 1, TIL_THREADS = TIL_WARPS * 32;   // softmax; first of the copies, of them for keys; all
constexpr int TIL_SORTED = 256;   // requests of a call that are put in order
constexpr long long TIL_WAIT_CYCLES = 1ll << 32;   // some two seconds

template <int HD>
struct TilShape {
  static constexpr int SLABS = HD / 64, GROUP = SLABS * 1024;   // slabs of 64 dims (128-byte rows); bytes of eight keys
  static constexpr int TILE = TIL_KEYS * HD * 2;        // bytes of 128 rows
  static constexpr int RING = 131072 / (2 * TILE);      // tiles of keys, and of values, in shared memory
  static constexpr int Q = 0, K = 2 * TILE, V = K + RING * TILE, END = V + RING * TILE;
};

struct TilShared {
  uint64_t q_full[2], s_full[2], p_full[2], o_full[2];
  uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4], v_land, unit_full[8], unit_empty[8];
  float row[2][2][128];   // of a stream's rows, from either of their threads: maxima, or sums
  uint64_t x_full, x_done;   // a unit that the streams share: stream 1's results are there; have been read
  float2 other[128];         // maxima and sums of stream 1's rows then
  uint32_t tmem;
  int dead, first;
  unsigned long long warp_sum[TIL_WARPS];
  int weight[TIL_SORTED], rows[TIL_SORTED];    // of requests: blocks that their last unit sees; rows (by place)
  uint16_t order[TIL_SORTED];                  // request of a place
};

__device__ __forceinline__ uint32_t til_smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void til_init(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(til_smem(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void til_expect(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(til_smem(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void til_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(til_smem(bar)) : "memory");
}
__device__ __forceinline__ bool til_try(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok)
               : "r"(til_smem(bar)), "r"(parity)
               : "memory");
  return ok != 0;
}
// A whole warp waits, with one answer for all lanes; bounded.  Whoever runs out of time says so, and everybody gives up (see til_give_up).
static __device__ __noinline__ bool til_wait_slow(uint64_t* bar, uint32_t parity, int* dead) {
  const long long t0 = clock64();
  unsigned spins = 0;
  while (!__all_sync(0xffffffffu, til_try(bar, parity))) {
    if ((++spins & 63u) == 0) {
      bool stop = *(volatile int*)dead != 0;
      if (!stop && clock64() - t0 > TIL_WAIT_CYCLES) {
        *(volatile int*)dead = 1;
        stop = true;
      }
      if (__any_sync(0xffffffffu, stop)) return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool til_elect() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ uint32_t til_uniform(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }
__device__ __forceinline__ void til_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void til_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void til_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A block of the cache (16 keys, all dims): two groups of eight keys, each as slabs of 64 dims, 1024 bytes a slab.  So one copy, and
// groups are the same distance apart in a block and between blocks, which is what an operand of 128 keys needs.
__device__ __forceinline__ void til_copy(uint32_t dst, const CUtensorMap* map, int group, int plane, uint64_t* bar, uint64_t policy) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %2, %2, %3, %4}], [%5], %6;" ::"r"(dst),
               "l"(map), "r"(0), "r"(group), "r"(plane), "r"(til_smem(bar)), "l"(policy)
               : "memory");
}
// D (+)= A B^T, both in shared memory
__device__ __forceinline__ void til_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
               "r"(accumulate)
               : "memory");
}
// the same with A in TMEM
__device__ __forceinline__ void til_mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc),
               "r"(accumulate)
               : "memory");
}
__device__ __forceinline__ void til_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(til_smem(bar)) : "memory");
}
// Shared-memory operands with 128-byte swizzle.  K-major (128-byte rows of 64 bf16 along K): groups of eight rows `group` bytes apart.
// MN-major (128-byte rows of 64 along N): groups of eight K-rows `group` bytes apart, the next 64 along N `slab` bytes on.
__device__ __forceinline__ uint64_t til_desc(uint32_t saddr, uint32_t slab, uint32_t group) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(slab >> 4) << 16 | (uint64_t)(group >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ uint32_t til_idesc(int n) {   // bf16 operands, fp32 accumulator, M = 128
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

// 32 lanes x 16 columns, without the wait: nothing may touch the registers before tmem_wait_ld_til() has named them.
__device__ __forceinline__ void til_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
#define BLINK_RW8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
__device__ __forceinline__ void tmem_wait_ld_til(uint32_t (&a)[16], uint32_t (&b)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : BLINK_RW8(a, 0), BLINK_RW8(a, 8), BLINK_RW8(b, 0), BLINK_RW8(b, 8) : : "memory");
}
#undef BLINK_RW8
__device__ __forceinline__ void til_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// The two warps of 32 rows: a barrier, and whether any of their threads says so.
__device__ __forceinline__ void til_pair_sync(int id) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ bool til_pair_any(int id, bool mine) {
  uint32_t any;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbarrier.cta.red.or.pred q, %1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(any)
               : "r"(id), "r"((uint32_t)mine)
               : "memory");
  return any != 0;
}
__device__ __forceinline__ void til_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
      "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void til_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float2 til_fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 til_add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// What a row sees of a tile: key x of block g of it (position at[g] + x) when x <= hi, and x > lo or x < sink.
struct TilMask {
  int pos, window, sinks, first_block, n_sinks, from;   // of the row; of the tile's first block in the unit's list; of the list
};
__device__ __forceinline__ void til_mask(uint32_t (&r)[16], const TilMask& k, int block) {   // block: of the tile
  const int i = k.first_block + block;
  const int at = (i < k.n_sinks ? i : k.from + i - k.n_sinks) * OPS_BLOCK;
  const int hi = min(max(k.pos - at + 1, 0), OPS_BLOCK);                                  // keys up to its own
  const int lo = k.window > 0 ? min(max(k.pos - k.window - at + 1, 0), OPS_BLOCK) : 0;    // keys before its window
  const int sink = min(max(k.sinks - at, 0), OPS_BLOCK);
  const uint32_t bits = ((1u << hi) - 1u) & (~((1u << lo) - 1u) | ((1u << sink) - 1u));
#pragma unroll
  for (int x = 0; x < 16; ++x)
    if (!(bits & (1u << x))) r[x] = 0xff800000u;
}

// Every tile is masked: two instructions a score, which nothing waits for; a second copy of the code for tiles that all rows see whole cost more
// in calls of a few tiles, where its first instructions come from L2 (4096 rows with a window of 128: 4 % longer).
// Half a row of a score tile (blocks block0 .. block0 + 3) -> 32 words of probabilities (bf16 pairs), their sum, and the largest score.
__device__ __forceinline__ void til_probs(uint32_t t_s, float qscale, float neg, const TilMask& mask, int block0, uint32_t (&p)[32], float& mx, float& sum) {
  const float2 scale2 = make_float2(qscale, qscale), neg2 = make_float2(neg, neg);
  float mx0 = -INFINITY, mx1 = -INFINITY;
  float2 s0 = make_float2(0.f, 0.f), s1 = s0;
  auto part = [&](uint32_t (&r)[16], int k) {
    til_mask(r, mask, block0 + k);
#pragma unroll
    for (int x = 0; x < 16; x += 4) {
      mx0 = fmaxf(fmaxf(mx0, __uint_as_float(r[x])), __uint_as_float(r[x + 1]));
      mx1 = fmaxf(fmaxf(mx1, __uint_as_float(r[x + 2])), __uint_as_float(r[x + 3]));
    }
#pragma unroll
    for (int x = 0; x < 16; x += 2) {
      float2 e = til_fma2(make_float2(__uint_as_float(r[x]), __uint_as_float(r[x + 1])), scale2, neg2);
      e.x = attn_ex2(e.x);
      e.y = attn_ex2(e.y);
      if (x & 2) s1 = til_add2(s1, e); else s0 = til_add2(s0, e);
      const __nv_bfloat162 b2 = __floats2bfloat162_rn(e.x, e.y);
      p[k * 8 + x / 2] = *reinterpret_cast<const uint32_t*>(&b2);
    }
  };
  // (a wait for TMEM takes some 400 cycles: what comes second is on its way while the first is worked on)
  uint32_t va[16], vb[16], vc[16], vd[16];
  til_ld16(t_s, va);
  til_ld16(t_s + 16u, vb);
  tmem_wait_ld_til(va, vb);
  til_ld16(t_s + 32u, vc);
  part(va, 0);
  til_ld16(t_s + 48u, vd);
  part(vb, 1);
  tmem_wait_ld_til(vc, vd);
  part(vc, 2);
  part(vd, 3);
  mx = fmaxf(mx0, mx1);
  const float2 s = til_add2(s0, s1);
  sum = s.x + s.y;
}
// A first maximum: the largest score of one block of the row's first tile.
__device__ __forceinline__ float til_max(uint32_t t_s, int block, const TilMask& mask) {
  uint32_t va[16], vb[16];
  til_ld16(t_s + 16u * (uint32_t)block, va);
  til_ld16(t_s + 16u * (uint32_t)block, vb);   // (the wait names two)
  tmem_wait_ld_til(va, vb);
  til_mask(va, mask, block);
  float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
  for (int x = 0; x < 16; x += 4) {
    m0 = fmaxf(fmaxf(m0, __uint_as_float(va[x])), __uint_as_float(va[x + 1]));
    m1 = fmaxf(fmaxf(m1, __uint_as_float(va[x + 2])), __uint_as_float(va[x + 3]));
  }
  return fmaxf(m0, m1);
}

// A unit, and which of its tiles each stream takes.
struct alignas(16) TilUnit {
  int req, h;
  int row, live[2];        // first of its rows; rows of each stream's
  int pos;                 // position of the first row
  AttnSpan span;
  int last;                // position of the last row
  int split;               // 1: rows for one stream only; both have them, stream 0 the even tiles and stream 1 the odd ones
  int begin[2], end[2];    // tiles of each stream: every one, or every second
  // (an array indexed with a register would lie in local memory, all of the record with it)
  __device__ __forceinline__ int live_of(int s) const { return s ? live[1] : live[0]; }
  __device__ __forceinline__ int begin_of(int s) const { return s ? begin[1] : begin[0]; }
  __device__ __forceinline__ int end_of(int s) const { return s ? end[1] : end[0]; }
};
constexpr int TIL_UNITS = 8;   // records of a CTA's units, used in turn: one is written again when all warps have read it

// By all threads of a CTA in which a wait has run out, the first of the call: the status, and no number in every row that the call has here.  Units that are
// not done stay so, and cannot be taken for results where nobody reads the status; what other CTAs store from here on is right.
static __device__ __noinline__ void til_give_up(const AttnArgs& a, int* first) {
  if (threadIdx.x == 0) *first = atomicExch(reinterpret_cast<int*>(a.ws), BLINK_ETIMEDOUT) == BLINK_OK;
  __syncthreads();
  if (!*first) return;
  const int pieces = a.pool.Hq * a.pool.hd / 8;   // 16 bytes each, of a row
  for (int r = 0; r < a.n; ++r) {
    const AttnReq q = attn_req(a, a.row_start[r], a.row_start[r + 1], a.kv_len[r]);
    if (q.rows <= a.few) continue;
    for (long long i = threadIdx.x; i < (long long)q.rows * pieces; i += TIL_THREADS)
      reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + (q.start + i / pieces) * a.out_stride)[i % pieces] = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
  }
}

template <int HD>
__global__ void __launch_bounds__(TIL_THREADS, 1) blink_attn_tiles_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ CUtensorMap map) {
  using S = TilShape<HD>;
  extern __shared__ char s_raw[];
  char* base = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(s_raw) + 1023) & ~(uintptr_t)1023);
  TilUnit* s_unit = reinterpret_cast<TilUnit*>(base + S::END);         // [TIL_UNITS]
  int* s_pre = reinterpret_cast<int*>(base + S::END) + TIL_UNITS * (sizeof(TilUnit) / 4);   // [n + 1] units before a request
  __shared__ __align__(16) TilShared sh;
  ops_next();
  const int w = (int)til_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  int* status = reinterpret_cast<int*>(a.ws);
  const int lr = 31 - __clz(a.pool.rep), P = 128 >> lr;   // query rows of a stream (1, 2, 4 or 8 heads each)

  if (threadIdx.x == 0) {
    for (int s = 0; s < 2; ++s) {
      til_init(&sh.q_full[s], TIL_SOFT / 2);
      til_init(&sh.s_full[s], 1);
      til_init(&sh.p_full[s], TIL_SOFT / 2);
      til_init(&sh.o_full[s], 1);
    }
    for (int i = 0; i < 4; ++i) {
      til_init(&sh.k_full[i], TIL_K);
      til_init(&sh.k_empty[i], 1);
      til_init(&sh.v_full[i], 1);
      til_init(&sh.v_empty[i], 1);
    }
    til_init(&sh.v_land, 1);
    til_init(&sh.x_full, TIL_SOFT / 2);
    til_init(&sh.x_done, TIL_SOFT / 2);
    for (int i = 0; i < TIL_UNITS; ++i) {
      til_init(&sh.unit_full[i], 1);
      til_init(&sh.unit_empty[i], TIL_WARPS);
    }
    sh.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (w == TIL_SOFT) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(til_smem(&sh.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  ops_wait();
  // The sequence of units: requests of more keys first, so that no CTA is left with a long unit at the end (48 requests of 300 to 5000 keys: in their
// own order 99 us, so 88); beyond TIL_SORTED requests units are many and their order matters less.  A run of requests (or places) per thread.
  const bool sorted = a.n <= TIL_SORTED;
  // Rows of a unit: two streams' worth, or one's, which both share, where there are few: twice the CTAs at half the time.  (8B shape, us, two | one: 512
  // rows behind 3500 keys 77 | 45, 40 behind 1000 28 | 19.  Between one and two units a CTA: 1024 rows 27.6 | 23.5, two of 512 behind 3500 79 | 79.  Between
  // two and three: 1500 rows 36.3 | 38.2.)
  int unit_shift = 8 - lr;   // (powers of two)
  {
    const int each = (a.n + TIL_THREADS - 1) / TIL_THREADS;
    const int r0 = min(a.n, (int)threadIdx.x * each), r1 = min(a.n, r0 + each);
    if (sorted) {
      const int r = threadIdx.x;
      int weight = 0, rows = 0;
      if (r < a.n) {
        const AttnReq q = attn_req(a, a.row_start[r], a.row_start[r + 1], a.kv_len[r]);
        rows = q.rows > a.few ? q.rows : 0;
        if (rows > 0) weight = attn_span(a, q.ctx + ((rows - 1) & -(2 * P)), q.ctx + rows - 1).n;
        sh.weight[r] = weight;
      }
      __syncthreads();
      if (r < a.n) {
        int place = 0;
        for (int k = 0; k < a.n; ++k) {
          const int other = sh.weight[k];
          place += other > weight || (other == weight && k < r);
        }
        sh.order[place] = (uint16_t)r;
        sh.rows[place] = rows;
      }
      __syncthreads();
    }
    auto rows_of = [&](int r) {
      if (sorted) return sh.rows[r];
      const AttnReq q = attn_req(a, a.row_start[r], a.row_start[r + 1], a.kv_len[r]);
      return q.rows > a.few ? q.rows : 0;
    };
    unsigned long long mine = 0;   // units: of two streams, and (above) of one
    for (int r = r0; r < r1; ++r) {
      const int rows = rows_of(r);
      mine += (unsigned long long)(((rows + 2 * P - 1) >> (8 - lr)) * a.pool.Hkv) | (unsigned long long)(((rows + P - 1) >> (7 - lr)) * a.pool.Hkv) << 32;
    }
    unsigned long long x = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned long long y = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += y;
    }
    if (lane == 31) sh.warp_sum[w] = x;
    __syncthreads();
    unsigned long long total = 0;
    const int warps = sorted ? (a.n + 31) / 32 : TIL_WARPS;   // that have any
    for (int i = 0; i < warps; ++i) {
      if (i < w) x += sh.warp_sum[i];
      total += sh.warp_sum[i];
    }
    const bool one = (total >> 32) <= 2u * gridDim.x;
    if (one) unit_shift = 7 - lr;
    int at = (int)((x - mine) >> (one ? 32 : 0));
    for (int r = r0; r < r1; ++r) {
      s_pre[r] = at;
      at += ((rows_of(r) + (1 << unit_shift) - 1) >> unit_shift) * a.pool.Hkv;
    }
    if (threadIdx.x == 0) s_pre[a.n] = (int)(total >> (one ? 32 : 0));
  }
  til_fence_before();
  __syncthreads();
  til_fence_after();
  const uint32_t tmem = til_uniform(*(volatile uint32_t*)&sh.tmem);
  const int n_units = (int)til_uniform((uint32_t)s_pre[a.n]);

  bool ok = true;   // false once a wait has run out
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (ok && !__all_sync(0xffffffffu, til_try(bar, parity))) ok = til_wait_slow(bar, parity, &sh.dead);
    return ok;
  };
  auto make_unit = [&](int u) {
    TilUnit t;
    int lo = 0, hi = a.n;   // the last place that begins at or before it
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_pre[mid] <= u) lo = mid; else hi = mid;
    }
    const int r = sorted ? sh.order[lo] : lo;
    const AttnReq q = attn_req(a, a.row_start[r], a.row_start[r + 1], a.kv_len[r]);
    const int unit_rows = 1 << unit_shift, blocks = (q.rows + unit_rows - 1) >> unit_shift;
    const int i = u - s_pre[lo], b = max(0, blocks - 1 - i / a.pool.Hkv);   // later rows, which see more, first
    t.req = r;
    t.h = i % a.pool.Hkv;
    t.row = q.start + b * unit_rows;
    const int rows = min(unit_rows, q.rows - b * unit_rows);
    t.live[0] = min(P, rows);
    t.live[1] = rows - t.live[0];
    t.pos = q.ctx + b * unit_rows;
    t.last = t.pos + rows - 1;
    t.span = attn_span(a, t.pos, t.last);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int first = t.pos + s * P, last = max(0, first + t.live_of(s) - 1);
      const int from = a.window > 0 ? max(0, first - a.window + 1) / OPS_BLOCK : 0;
      t.begin[s] = a.sinks > 0 ? 0 :   // (the sinks may lie in the unit's window, and not in the stream's)
                                   min(max(0, from - t.span.from), t.span.n - 1) / TIL_BLOCKS;
      t.end[s] = min(t.span.n - 1, max(0, t.span.sinks + last / OPS_BLOCK - t.span.from)) / TIL_BLOCKS + 1;
      if (t.live_of(s) == 0) t.begin[s] = t.end[s] = 0;
    }
    t.split = t.live[1] == 0 && t.end[0] > 1;
    if (t.split) {
      t.live[1] = t.live[0];
      t.begin[1] = 1;
      t.end[1] = t.end[0];
    }
    return t;
  };
  // the CTA's i-th unit, live[0] == 0: there is none
  auto unit_of = [&](int i) {
    const int slot = i % TIL_UNITS;
    wait(&sh.unit_full[slot], (uint32_t)(i / TIL_UNITS) & 1u);
    TilUnit t = s_unit[slot];
    __syncwarp();
    if (lane == 0) til_arrive(&sh.unit_empty[slot]);
    if (!ok) t.live[0] = 0;
    return t;
  };
  // by one warp
  auto hand_out = [&](int i, int u) {
    TilUnit t;
    if (u < n_units) t = make_unit(u);
    else t.live[0] = 0;
    if (i >= TIL_UNITS) wait(&sh.unit_empty[i % TIL_UNITS], (uint32_t)(i / TIL_UNITS - 1) & 1u);
    if (ok && lane == 0) {
      s_unit[i % TIL_UNITS] = t;
      til_arrive(&sh.unit_full[i % TIL_UNITS]);
    }
    __syncwarp();
  };
  auto tiles_of = [&](const TilUnit& t) { return max(t.end[0], t.end[1]); };   // (the first tile is one of stream 0, which always has rows)

  if (w < TIL_SOFT) {
    // ---- softmax ----
    const int s = w >> 3, half = (w >> 2) & 1, q = w & 3, m = q * 32 + lane, rep = 1 << lr, pair = 1 + s * 4 + q;
    const uint32_t t_row = (uint32_t)(q * 32) << 16;
    const uint32_t t_s = tmem + (uint32_t)(s * 128) + t_row, t_o = tmem + 256u + (uint32_t)(s * HD + half * (HD / 2)) + t_row;
    const uint32_t b_q = til_smem(base) + S::Q + s * S::TILE;
    uint32_t n_s = 0, n_o = 0, n_x = 0;
    auto load_q = [&](const TilUnit& t) {
      constexpr int CH = HD / 8;   // 16-byte pieces of a row
#pragma unroll 4
      for (int k = 0; k < CH / 2; ++k) {
        const int i = k * 256 + (int)(threadIdx.x & 255), row = i / CH, ck = i % CH;
        const int r = row >> lr;
        const bool live = r < t.live_of(s);
        const char* src = static_cast<const char*>(a.q) + ((long long)(t.row + (live ? (t.split ? 0 : s * P) + r : 0)) * a.q_stride + ((t.h << lr) + (row & (rep - 1))) * HD + ck * 8) * 2;
        const uint32_t dst = b_q + (ck >> 3) * 16384 + row * 128 + (((ck & 7) ^ (row & 7)) << 4);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16u : 0u) : "memory");
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto q_there = [&]() {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      til_proxy_fence();
      __syncwarp();
      if (lane == 0) til_arrive(&sh.q_full[s]);
    };
    // (the two warps of a pair go on together or not at all: a barrier of theirs has no limit)
    auto together = [&](TilUnit& t) {
      if (til_pair_any(pair, !ok)) {
        ok = false;
        t.live[0] = 0;
      }
    };
    TilUnit t = unit_of(0);
    together(t);
    if (t.live[0] && t.live_of(s)) {
      load_q(t);
      q_there();
    }
#pragma unroll 1
    for (int u = 0; t.live[0]; ++u) {
      bool more = false;   // a next unit, in which the stream has rows
      if (t.live_of(s)) {
        const int r = m >> lr, split = t.split, off = split ? 0 : s * P, step = 1 + split;
        TilMask mask;
        mask.pos = r < t.live_of(s) ? t.pos + off + r : -1;
        mask.window = a.window;
        mask.sinks = a.sinks;
        mask.n_sinks = t.span.sinks;
        mask.from = t.span.from;
        const int p_hi = t.pos + off + ((q * 32 + 31) >> lr);
        const int begin = t.begin_of(s), end = t.end_of(s);
        const int t_row0 = t.row + off, t_head = (t.h << lr) + (m & (rep - 1));
        const bool mine = r < t.live_of(s);
        float mx_used = -INFINITY, l = 0.f;
#pragma unroll 1
        for (int j = begin; j < end; j += step) {
          mask.first_block = j * TIL_BLOCKS;
          const int i0 = mask.first_block, i1 = i0 + TIL_BLOCKS - 1;
          const int lowest = i1 < mask.n_sinks ? a.window + p_hi : (mask.from + max(0, i0 - mask.n_sinks)) * OPS_BLOCK;   // of its blocks behind the sinks
          const bool cut = a.window > 0 && lowest <= p_hi - a.window;
          wait(&sh.s_full[s], n_s & 1u);
          ++n_s;
          til_fence_after();
          if (j == begin) {   // a first maximum: from keys next to the window's end where the tile is cut by the window, else from the first ones
            const float x = til_max(t_s, (cut ? 6 : 0) + half, mask) * a.qscale;
            sh.row[s][half][m] = x;
            til_pair_sync(pair);
            mx_used = fmaxf(x, sh.row[s][half ^ 1][m]);
          }
          if (j + step >= end) {   // the last scores are complete: the queries have been read
            t = unit_of(u + 1);
            more = t.live[0] > 0 && t.live_of(s) > 0;
            if (more) load_q(t);
          }
          uint32_t p[32];
          float sum;
#pragma unroll 1
          while (true) {
            float mx;
            const float neg = mx_used == -INFINITY ? 0.f : -mx_used;
            til_probs(t_s + (uint32_t)half * 64u, a.qscale, neg, mask, half * 4, p, mx, sum);
            mx *= a.qscale;
            if (!til_pair_any(pair, mx > mx_used + 8.f)) break;
            sh.row[s][half][m] = mx;
            til_pair_sync(pair);
            const float top = fmaxf(mx_used, fmaxf(mx, sh.row[s][half ^ 1][m]));
            const float f = top == -INFINITY ? 1.f : attn_ex2(mx_used - top);
            mx_used = top;
            l *= f;
            if (j > begin) {   // the stream's accumulator is complete: its MMAs came before these scores'
#pragma unroll 1
              for (int k = 0; k < HD / 2; k += 32) {
                uint32_t x[16], y[16];
                til_ld16(t_o + (uint32_t)k, x);
                til_ld16(t_o + (uint32_t)k + 16u, y);
                tmem_wait_ld_til(x, y);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                  x[i] = __float_as_uint(__uint_as_float(x[i]) * f);
                  y[i] = __float_as_uint(__uint_as_float(y[i]) * f);
                }
                til_st16(t_o + (uint32_t)k, x);
                til_st16(t_o + (uint32_t)k + 16u, y);
              }
              til_wait_st();
            }
            til_pair_sync(pair);   // (both have read the other's)
          }
          l += sum;
          til_st32(t_s + (uint32_t)half * 64u, p);
          til_wait_st();
          til_fence_before();
          __syncwarp();
          if (lane == 0) til_arrive(&sh.p_full[s]);
        }
        if (more) q_there();
        sh.row[s][half][m] = l;
        til_pair_sync(pair);
        l += sh.row[s][half ^ 1][m];
        wait(&sh.o_full[s], n_o & 1u);
        ++n_o;
        til_fence_after();
        float f0 = l > 0.f ? __fdividef(1.0f, l) : 0.f, f1 = 0.f;
        if (split) {
          if (s == 1) {
            if (half == 0) sh.other[m] = make_float2(mx_used, l);
            til_fence_before();
            __syncwarp();
            if (lane == 0) til_arrive(&sh.x_full);
            wait(&sh.x_done, n_x++ & 1u);   // (before the accumulator's next use)
            together(t);
            continue;
          }
          wait(&sh.x_full, n_x++ & 1u);
          til_fence_after();
          const float2 o = sh.other[m];
          const float top = fmaxf(mx_used, o.x), g0 = mx_used == -INFINITY ? 0.f : attn_ex2(mx_used - top), g1 = o.x == -INFINITY ? 0.f : attn_ex2(o.x - top);
          const float sum = l * g0 + o.y * g1;
          const float inv = sum > 0.f ? __fdividef(1.0f, sum) : 0.f;
          f0 = g0 * inv;
          f1 = g1 * inv;
        }
        const bool store = mine && ok && *(volatile int*)&sh.dead == 0;   // (who has given up goes on arriving: what comes of that is nobody's output)
        char* dst = static_cast<char*>(a.out) + ((long long)(t_row0 + (store ? r : 0)) * a.out_stride + t_head * HD + half * (HD / 2)) * 2;
#pragma unroll 1
        for (int k = 0; k < HD / 2; k += 32) {
          uint32_t x[16], y[16];
          til_ld16(t_o + (uint32_t)k, x);
          til_ld16(t_o + (uint32_t)k + 16u, y);
          tmem_wait_ld_til(x, y);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            x[i] = __float_as_uint(__uint_as_float(x[i]) * f0);
            y[i] = __float_as_uint(__uint_as_float(y[i]) * f0);
          }
          if (split) {
            uint32_t x1[16], y1[16];
            til_ld16(t_o + (uint32_t)(HD + k), x1);
            til_ld16(t_o + (uint32_t)(HD + k) + 16u, y1);
            tmem_wait_ld_til(x1, y1);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              x[i] = __float_as_uint(fmaf(__uint_as_float(x1[i]), f1, __uint_as_float(x[i])));
              y[i] = __float_as_uint(fmaf(__uint_as_float(y1[i]), f1, __uint_as_float(y[i])));
            }
          }
          auto put = [&](const uint32_t(&v)[16], int at) {   // a lane's row lies alone: 32 bytes at a time, where they may
            uint32_t o[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const __nv_bfloat162 b2 = __floats2bfloat162_rn(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1]));
              o[c] = *reinterpret_cast<const uint32_t*>(&b2);
            }
            if (store && a.out_32) {
              asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + at * 2), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]),
                           "r"(o[5]), "r"(o[6]), "r"(o[7])
                           : "memory");
            } else if (store) {
              *reinterpret_cast<uint4*>(dst + at * 2) = make_uint4(o[0], o[1], o[2], o[3]);
              *reinterpret_cast<uint4*>(dst + at * 2 + 16) = make_uint4(o[4], o[5], o[6], o[7]);
            }
          };
          put(x, k);
          put(y, k + 16);
        }
        til_fence_before();      // (before the accumulator's next use: the next probabilities' arrival)
        if (split) {
          __syncwarp();
          if (lane == 0) til_arrive(&sh.x_done);
        }
        together(t);             // (and both have read the other's sum)
      } else {
        t = unit_of(u + 1);
        together(t);
        if (t.live[0] && t.live_of(s)) {
          load_q(t);
          q_there();
        }
      }
    }
  } else if (w < TIL_COPY) {
    // ---- MMAs ----
    // (what they are issued with comes from uniform registers, and their loops turn on uniform values: otherwise an MMA's operands are moved first
    // and its warp is taken for a diverged one, some 100 cycles each, more than the tensor core takes for it)
    const uint32_t idesc_s = til_idesc(TIL_KEYS), idesc_o = til_idesc(HD) | (1u << 16);   // (bit 16: B is MN-major)
    const uint32_t b0 = til_uniform(til_smem(base));
    uint32_t n_tile = 0, n_q0 = 0, n_q1 = 0, n_p0 = 0, n_p1 = 0;
#pragma unroll 1
    for (int u = 0; ok; ++u) {
      const TilUnit t = unit_of(u);
      if (til_uniform((uint32_t)t.live[0]) == 0u) break;
      const int begin1 = (int)til_uniform((uint32_t)t.begin[1]), end0 = (int)til_uniform((uint32_t)t.end[0]), end1 = (int)til_uniform((uint32_t)t.end[1]);
      const int tiles = max(end0, end1);   // (stream 0 takes tiles 0 .. end0 - 1, stream 1 begin1 .. end1 - 1, which is none where it has no rows; shared: 0, 2 .., and 1, 3 ..)
      const int split = (int)til_uniform((uint32_t)t.split), step = 1 + split;
      auto scores = [&](int s, int j) {
        const uint32_t n = n_tile + (uint32_t)j, slot = n % S::RING;
        wait(&sh.k_full[slot], (n / S::RING) & 1u);
        if (!ok) return;
        til_fence_after();
        const uint64_t dq = til_desc(b0 + S::Q + s * S::TILE, 16, 1024), dk = til_desc(b0 + S::K + slot * S::TILE, 16, S::GROUP);
        const bool last = split || s == 1 || j < begin1 || j >= end1;
        if (til_elect()) {
#pragma unroll
          for (int i = 0; i < HD / 16; ++i)
            til_mma(tmem + (uint32_t)s * 128u, dq + (uint64_t)((i >> 2) * 1024 + (i & 3) * 2), dk + (uint64_t)((i >> 2) * 64 + (i & 3) * 2), idesc_s, i ? 1u : 0u);
          til_commit(&sh.s_full[s]);
          if (last) til_commit(&sh.k_empty[slot]);
        }
        __syncwarp();
      };
      auto outputs = [&](int s, int j, uint32_t n_p) {
        const uint32_t n = n_tile + (uint32_t)j, slot = n % S::RING;
        wait(&sh.p_full[s], n_p & 1u);
        wait(&sh.v_full[slot], (n / S::RING) & 1u);
        if (!ok) return;
        til_fence_after();
        const uint64_t dv = til_desc(b0 + S::V + slot * S::TILE, 1024, S::GROUP);
        const uint32_t keep = j > (s ? begin1 : 0) ? 1u : 0u;
        const bool end = j + step >= (s ? end1 : end0), last = split || s == 1 || j < begin1 || j >= end1;
        if (til_elect()) {
#pragma unroll
          for (int i = 0; i < TIL_BLOCKS; ++i)   // 16 keys each, a block of the cache
            til_mma_tmem(tmem + 256u + (uint32_t)(s * HD), tmem + (uint32_t)s * 128u + (uint32_t)((i >> 2) * 64 + (i & 3) * 8),
                         dv + (uint64_t)(i * (S::TILE / TIL_BLOCKS / 16)), idesc_o, i ? 1u : keep);
          if (end) til_commit(&sh.o_full[s]);
          if (last) til_commit(&sh.v_empty[slot]);
        }
        __syncwarp();
      };
      wait(&sh.q_full[0], n_q0++ & 1u);
      scores(0, 0);
      if (end1 > 0) {
        wait(&sh.q_full[1], n_q1++ & 1u);
        if (begin1 == split) scores(1, split);
      }
#pragma unroll 1
      for (int j = 0; j < tiles && ok; j += step) {
        const int j1 = j + split;
        if (j < end0) outputs(0, j, n_p0++);
        if (j + step < end0) scores(0, j + step);
        if (j1 >= begin1 && j1 < end1) outputs(1, j1, n_p1++);
        if (j1 + step >= begin1 && j1 + step < end1) scores(1, j1 + step);
      }
      n_tile += (uint32_t)tiles;
    }
  } else {
    // ---- copies ----
    const int part = w - TIL_COPY;   // 0 .. TIL_K - 1: keys
    const bool values = part == TIL_K;
    {
      uint64_t policy;
      asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
      const int none = (int)a.pool.n_blocks * a.pool.Hkv * 2;   // (a group behind the pool: zeros)
      uint32_t n_tile = 0, n_land = 0;
      auto block_id = [&](const TilUnit& t, int j) {   // lane: block of the tile; behind the list the last one again (nobody sees it there)
        const int i = min(j * TIL_BLOCKS + (lane & 7), t.span.n - 1);
        return t.last >= 0 ? a.table[(long long)t.req * a.stride + (i < t.span.sinks ? i : t.span.from + i - t.span.sinks)] : -1;
      };
      if (part == 0) hand_out(0, (int)blockIdx.x);
#pragma unroll 1
      for (int u = 0; ok; ++u) {
        const TilUnit t = unit_of(u);
        if (!t.live[0]) break;
        int id = block_id(t, 0);
        const int tiles = tiles_of(t);
#pragma unroll 1
        for (int j = 0; j < tiles; ++j) {
          const int mine = (unsigned)id < (unsigned)a.pool.n_blocks ? (id * a.pool.Hkv + t.h) * 2 : none;
          if (j + 1 < tiles) id = block_id(t, j + 1);
          const uint32_t n = n_tile + (uint32_t)j, slot = n % S::RING, use = n / S::RING;
          uint64_t* empty = values ? &sh.v_empty[slot] : &sh.k_empty[slot];
          if (use > 0) wait(empty, (use - 1u) & 1u);
          if (!ok) break;
          if (part == 0 && j == max(0, tiles - 2)) {   // the next unit, late, so that the CTAs end together; the counter was zeroed by a kernel before this one
            int next = 0;
            if (lane == 0) next = (int)gridDim.x + atomicAdd(status + 1, 1);
            hand_out(u + 1, __shfl_sync(0xffffffffu, next, 0));
          }
          const uint32_t dst = til_smem(base) + (values ? S::V : S::K) + slot * S::TILE;
          bool clean = true;   // some row sees every key of the tile, so that its values are numbers
          if (values) {
            const int i0 = j * TIL_BLOCKS, i1 = i0 + TIL_BLOCKS - 1;
            clean = t.last >= (t.span.from + i1 - t.span.sinks) * OPS_BLOCK + OPS_BLOCK - 1 && !(i0 < t.span.sinks && (a.sinks & (OPS_BLOCK - 1))) &&
                    !(a.window > 0 && i1 >= t.span.sinks && (t.span.from + max(0, i0 - t.span.sinks)) * OPS_BLOCK <= t.pos - a.window);
          }
          uint64_t* full = !values ? &sh.k_full[slot] : clean ? &sh.v_full[slot] : &sh.v_land;
          if (til_elect()) til_expect(full, (uint32_t)(values ? S::TILE : S::TILE / TIL_K));
          __syncwarp();
#pragma unroll
          for (int k = 0; k < TIL_BLOCKS; ++k) {
            if (!values && k >= TIL_BLOCKS / TIL_K) break;
            const int i = values ? k : part * (TIL_BLOCKS / TIL_K) + k;
            const int group = (int)til_uniform((uint32_t)__shfl_sync(0xffffffffu, mine, i));
            if (til_elect()) til_copy(dst + i * (S::TILE / TIL_BLOCKS), &map, group, values, full, policy);
            __syncwarp();
          }
          if (values && !clean) {   // what no row sees may be anything, and 0 x NaN is not 0
            wait(&sh.v_land, n_land & 1u);
            ++n_land;
            char* v = base + S::V + slot * S::TILE;
#pragma unroll 1
            for (int x = lane; x < TIL_KEYS; x += 32) {
              const int i = j * TIL_BLOCKS + x / OPS_BLOCK;
              const int at = (i < t.span.sinks ? i : t.span.from + i - t.span.sinks) * OPS_BLOCK + x % OPS_BLOCK;
              if (at <= t.last && (a.window == 0 || at > t.pos - a.window || at < a.sinks)) continue;
              char* to = v + (x / 8) * S::GROUP + (x % 8) * 128;
#pragma unroll
              for (int c = 0; c < HD / 8; ++c) *reinterpret_cast<uint4*>(to + (c >> 3) * 1024 + ((c + lane) & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            til_proxy_fence();
            __syncwarp();
            if (lane == 0) til_arrive(&sh.v_full[slot]);
          }
        }
        n_tile += (uint32_t)tiles;
      }
    }
  }
  // copies that are still on their way after a wait has run out land before the shared memory is given up
  if (!ok) {
    const long long t0 = clock64();
    while (clock64() - t0 < 200000ll) {}
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  til_fence_before();
  __syncthreads();
  if (w == TIL_SOFT) {
    til_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
  if (sh.dead) til_give_up(a, &sh.first);
}

typedef CUresult (*TilEncode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                              CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static TilEncode til_encode() {
  static const TilEncode f = [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult how;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &how) != cudaSuccess || how != cudaDriverEntryPointSuccess) return (TilEncode) nullptr;
    return reinterpret_cast<TilEncode>(fn);
  }();
  return f;
}

// The kernel before the tiles where there are no requests for the other kernels: a status, and the counter of units.
__global__ void blink_attn_begin_kernel(int* ws) {
  ops_begin();
  if (threadIdx.x < 2) ws[threadIdx.x] = 0;
}

template <int HD>
static int tiles_run(const AttnArgs& a, int sms, int64_t most_units, void* stream) {
  using S = TilShape<HD>;
  // (first of all: a host thread that comes here before it has used the device has no context for the tensor map until something is launched)
  if (a.few == 0) {
    const int rc = ops_launch(blink_attn_begin_kernel, 1, 32, 0, stream, 0, reinterpret_cast<int*>(a.ws));
    if (rc != BLINK_OK) return rc;
  }
  const TilEncode encode = til_encode();
  if (!encode) return BLINK_ECUDA;
  // the layer's keys and values as {64 dims, 8 keys, slabs of dims, groups of 8 keys, keys | values}; a copy brings two groups
  const cuuint64_t groups = (cuuint64_t)a.pool.n_blocks * a.pool.Hkv * 2;
  const cuuint64_t dims[5] = {64, 8, HD / 64, groups, 2}, strides[4] = {HD * 2, 128, 8 * HD * 2, groups * 8 * HD * 2};
  const cuuint32_t box[5] = {64, 8, HD / 64, 2, 1}, one[5] = {1, 1, 1, 1, 1};
  CUtensorMap map;
  if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, a.pool.k, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return BLINK_ECUDA;
  const size_t fixed = (size_t)S::END + 1024 + TIL_UNITS * sizeof(TilUnit);
  const OpsShared smem(fixed + (size_t)(a.n + 1) * 4, fixed + (size_t)(OPS_MAX_REQUESTS + 1) * 4);
  const int64_t grid = most_units < sms ? most_units : sms;
  return ops_launch(blink_attn_tiles_kernel<HD>, grid, TIL_THREADS, smem, stream, 0, a, map);
}

int attn_tiles(const AttnArgs& a, int sms, void* stream) {
  const int64_t most_units = ((int64_t)a.rows * a.pool.rep / 128 + a.n) * a.pool.Hkv;   // of one stream each
  return a.pool.hd == 128 ? tiles_run<128>(a, sms, most_units, stream) : tiles_run<64>(a, sms, most_units, stream);
}

}  // namespace blink
