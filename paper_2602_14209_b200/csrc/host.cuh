// Host-side helpers shared by the entry points: argument validation, the device view of a cache description, launches,
// shared-memory opt-in and the tensor-map encoder.
#pragma once
#include <cuda.h>

#include <atomic>
#include <cstdio>
#include <mutex>

#include "common.cuh"

namespace mage {

inline std::atomic<uint64_t> g_launches{0};

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline bool valid_kv(const mage_kv_t *kv, mage_status *why) {
    auto fail = [&](mage_status s) { if (why) *why = s; return false; };
    if (!kv) return fail(MAGE_ERR_INVALID_ARG);
    if (kv->P < 1 || kv->H_q < 1 || kv->H_kv < 1 || kv->H_q % kv->H_kv != 0 || kv->B < 1 || kv->N_max < 0 || kv->d < 1)
        return fail(MAGE_ERR_INVALID_ARG);
    if (kv->d != kD || kv->B > 64) return fail(MAGE_ERR_UNSUPPORTED);
    if (kv->N_max > 0 && (!kv->k_cache || !kv->v_cache)) return fail(MAGE_ERR_INVALID_ARG);
    if (kv->page_size < 0) return fail(MAGE_ERR_INVALID_ARG);
    if (kv->page_size == 0) {
        if (kv->stride_n < kD || kv->stride_n % 8 || kv->stride_h % 8 || kv->stride_p % 8 || kv->stride_h < 0 || kv->stride_p < 0)
            return fail(MAGE_ERR_INVALID_ARG);
    } else {
        if (kv->page_size < 16 || (kv->page_size & (kv->page_size - 1))) return fail(MAGE_ERR_UNSUPPORTED);
        if (kv->N_max > 0 && (!kv->block_table || kv->num_pages < 1)) return fail(MAGE_ERR_INVALID_ARG);
        if ((int64_t)kv->max_pages * kv->page_size < kv->N_max) return fail(MAGE_ERR_INVALID_ARG);
    }
    if ((int64_t)kv->P * kv->H_kv > 65535) return fail(MAGE_ERR_UNSUPPORTED);      // (problem, KV head) pairs are one grid dimension
    return true;
}

inline KvView make_view(const mage_kv_t *kv) {
    KvView v;
    v.k = static_cast<const __nv_bfloat16 *>(kv->k_cache);
    v.v = static_cast<const __nv_bfloat16 *>(kv->v_cache);
    v.stride_p = kv->stride_p; v.stride_h = kv->stride_h; v.stride_n = kv->stride_n;
    v.block_table = kv->block_table; v.seq_lens = kv->seq_lens;
    v.max_pages = kv->max_pages; v.num_pages = kv->num_pages; v.page_size = kv->page_size;
    v.N_max = kv->N_max;
    v.P = kv->P; v.H_q = kv->H_q; v.H_kv = kv->H_kv; v.B = kv->B; v.G = kv->H_q / kv->H_kv; v.M = v.G * kv->B;
    return v;
}

// Launch with the programmatic-serialization attribute: the kernel may be scheduled while its predecessor in the stream is
// still running; every kernel launched this way begins with griddepcontrol.wait, so it touches no global memory before
// the predecessor has completed.  What is saved is the launch gap between dependent kernels (a few microseconds each,
// which is most of a single-layer reuse step).
template <typename... KArgs, typename... Args>
inline cudaError_t launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args &&...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

inline mage_status launch_check() {
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) {
        std::fprintf(stderr, "libmage: kernel launch failed: %s\n", cudaGetErrorString(e));
        return MAGE_ERR_CUDA;
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return MAGE_OK;
}

// Raise a kernel's dynamic shared memory limit; done once per kernel and device, remembered afterwards.
inline mage_status opt_in_smem_impl(const void *kernel, size_t bytes) {
    static std::mutex mu;
    static const void *seen[32];
    static unsigned long long seen_devs[32];
    static int n_seen = 0;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return MAGE_ERR_CUDA;
    const unsigned long long bit = 1ull << (dev & 63);
    std::lock_guard<std::mutex> lock(mu);
    int slot = -1;
    for (int i = 0; i < n_seen; ++i)
        if (seen[i] == kernel) slot = i;
    if (slot >= 0 && (seen_devs[slot] & bit)) return MAGE_OK;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return MAGE_ERR_CUDA;
    if (slot < 0 && n_seen < 32) { slot = n_seen++; seen[slot] = kernel; seen_devs[slot] = 0; }
    if (slot >= 0) seen_devs[slot] |= bit;
    return MAGE_OK;
}
template <typename K>
inline mage_status opt_in_smem(K kernel, size_t bytes) { return opt_in_smem_impl(reinterpret_cast<const void *>(kernel), bytes); }

namespace tc {

using EncodeTiledFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                   const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver entry point is looked up through the runtime, so the library does not link against libcuda.
inline EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiledFn>(p);
    }();
    return fn;
}

}  // namespace tc
}  // namespace mage
