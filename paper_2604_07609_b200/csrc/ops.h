// What the operators that can be called alone (ops_*.cu) share on the host: checks of their arguments and launches.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/blink.h"

namespace blink {

constexpr int OPS_BLOCK = 16;            // tokens of a KV block
constexpr int OPS_MAX_REQUESTS = 4096;   // their prefix sums are kept in shared memory

// blink_verify_drafts; with `clear` rows that belong to nobody get the token -1 (for tokens in memory that nobody has written yet).
int verify_drafts(const float* logits, int64_t logits_stride, int rows, int vocab, const int32_t* row_start, int n_requests, const int32_t* draft_tokens,
                  const float* draft_probs, int64_t probs_stride, const float* temperature, const float* u_accept, const float* u_pick, int32_t* out_tokens,
                  int32_t* n_accepted, void* workspace, uint64_t workspace_bytes, bool clear, void* stream);

// One layer of a paged KV pool, [2][n_blocks][Hkv][16][hd] each, as the kernels address it.
struct OpsPool {
  char* k;           // block 0 of the layer's keys
  char* v;
  int64_t n_blocks;
  int Hq, Hkv, rep, hd, dtype;
};

inline bool ops_aligned(const void* p, uintptr_t to) { return p != nullptr && ((uintptr_t)p & (to - 1)) == 0; }

inline int ops_pool(const blink_model_cfg* m, const blink_kv_pool* kv, int layer, OpsPool* out) {
  if (!m || !kv || kv->size != sizeof(blink_kv_pool) || kv->block_size != OPS_BLOCK) return BLINK_EINVAL;
  const int64_t nb = blink_kv_blocks_for_bytes(m, OPS_BLOCK, kv->bytes);   // (refuses a bad model)
  if (nb < 0) return BLINK_EINVAL;
  if (nb == 0) return BLINK_ENOMEM;
  if (layer < 0 || layer >= m->n_layers || !ops_aligned(kv->base, 256)) return BLINK_EINVAL;
  // slots and rows of 64 elements are counted in 32 bits
  if (nb * OPS_BLOCK * m->n_kv_heads > 0x7fffffffll) return BLINK_ETOOBIG;
  const int64_t esz = m->dtype == BLINK_DTYPE_BF16 ? 2 : 4;
  const int64_t plane = nb * m->n_kv_heads * OPS_BLOCK * m->head_dim * esz;
  out->k = static_cast<char*>(kv->base) + 2 * layer * plane;
  out->v = out->k + plane;
  out->n_blocks = nb;
  out->Hq = m->n_q_heads;
  out->Hkv = m->n_kv_heads;
  out->rep = m->n_q_heads / m->n_kv_heads;
  out->hd = m->head_dim;
  out->dtype = m->dtype;
  return BLINK_OK;
}

// A launch reports its own error.  What it left behind of it is taken away, so that no later call reports it; what another call of the library
// left (memory that was not to be had) is none of this one's.
inline int ops_launched(cudaError_t e) {
  if (e == cudaSuccess) return BLINK_OK;
  (void)cudaGetLastError();
  return BLINK_ECUDA;
}

// Dynamic shared memory of a launch, and the most that the same kernel is ever launched with.  The limit of a kernel is the device's, whoever calls: were
// it set to what one call needs, the launch of another host thread that needs more could come right behind that and be refused.
struct OpsShared {
  size_t bytes, most;
  OpsShared(size_t always) : bytes(always), most(always) {}
  OpsShared(size_t now, size_t at_most) : bytes(now), most(at_most) {}
};

// cluster > 0: CTAs of a cluster.  Kernels are set up while the one before them in the stream still runs (1 to 2 us less a launch) and wait for
// it themselves, in all of their threads and before they read or write anything that others do: only behind a kernel's own wait is what came before it
// sure to be seen, and a kernel that is done says that all before it are.  (With the later kernels of a call reading its inputs before their wait: one row behind
// 8000 keys beside two prompts of 2000 99 us, 105 so; one beside a prompt of 500 48 and 51; calls without rows for two kernels the same.)
template <typename... P, typename... A>
inline int ops_launch(void (*kernel)(P...), int64_t grid, int threads, OpsShared smem, void* stream, int cluster, A... args) {
  if (grid < 1) return BLINK_OK;
  if (grid > 0x7fffffffll) return BLINK_ETOOBIG;
  if (smem.bytes > 40 * 1024) {   // (48 KB are free to a kernel, its static shared memory among them, of which none that takes dynamic memory has more than 8 KB)
    const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem.most);
    if (e != cudaSuccess) return ops_launched(e);
  }
  if (cluster > 8) {   // more than every device takes
    const cudaError_t e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return ops_launched(e);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem.bytes;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute at[2];
  int n = 0;
  if (cluster > 0) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = (unsigned)cluster;
    at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
    ++n;
  }
  at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[n].val.programmaticStreamSerializationAllowed = 1;
  ++n;
  cfg.attrs = at;
  cfg.numAttrs = (unsigned)n;
  return ops_launched(cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...));
}

#ifdef __CUDACC__
__device__ __forceinline__ void ops_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// What came before is done, and what comes next may be set up.
__device__ __forceinline__ void ops_begin() {
  ops_wait();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
__device__ __forceinline__ void ops_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
#endif

}  // namespace blink
