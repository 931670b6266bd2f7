// Shared by the operators on a caller's own paged cache and logits (xsm_append.cu, xsm_attend.cu, xsm_logprob.cu).
#pragma once
#include "xsm_host.h"

#include <stddef.h>
#include <stdint.h>

struct xsm_kv {
    xsm_kv_config cfg;
    void *k, *v;
    // boxes of 16 or 32 positions of a head, as many elements wide as fill 128 (d_head 32 and 96 of 16 bits: 64) bytes, swizzled
    xsm::TensorMap k_map, v_map;
    int box_rows, sms;
    unsigned tries;      // of a barrier of xsm_kv_attend, before a wait gives up
    int starve;          // xsm_debug_kv_waits
};

namespace xsm {

// leaves the text for xsm_last_error(NULL) and hands the status back
xsm_status op_failed(xsm_status st, const char *msg) noexcept;

inline xsm_status launched(cudaError_t e) noexcept {
    if (e == cudaSuccess) return XSM_OK;
    (void)cudaGetLastError();      // reported here: the next call starts clean
    return op_failed(XSM_ERR_CUDA, cudaGetErrorString(e));
}
inline int element_size(int dtype) { return dtype == XSM_F32 ? 4 : 2; }
inline bool is_dtype(int dtype) { return dtype == XSM_F32 || dtype == XSM_BF16 || dtype == XSM_F16; }

// The pools as the kernels see them.
struct Pages {
    char *k, *v;
    const int *table;
    long long page, head, row, table_ld;      // strides in elements
    int n_pages, size, kv_heads, max_pages;
};
inline Pages pages_of(const xsm_kv &kv, const int32_t *table, int64_t table_ld, int max_pages) {
    const xsm_kv_config &c = kv.cfg;
    return Pages{(char *)kv.k, (char *)kv.v, table, c.page_stride, c.head_stride, c.row_stride, table_ld, c.n_pages, c.page_size, c.n_kv_heads, max_pages};
}

// ------------------------------------------------------------------------------------------- elements

// rounding to the type, once: to the nearest, what is too large becomes infinite
template <typename T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 rounded<bf16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half rounded<__half>(float v) { return __float2half_rn(v); }
// the same for an element of a pool: fp16 saturates, as the cache of this library's own models does; NaN stays NaN
template <typename T> __device__ __forceinline__ T to_stored(float v) { return rounded<T>(v); }
template <> __device__ __forceinline__ __half to_stored<__half>(float v) {
    return __float2half_rn(fabsf(v) > 65504.f ? copysignf(65504.f, v) : v);
}

// Launches a kernel that may start while the one before it on the stream still runs: it calls chain_wait before its first access to
// memory, and chain_go to let the next one do the same.
template <typename... P, typename... X>
inline cudaError_t launch_early(void (*fn)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const X &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, fn, args...);
}

// calls f with a value of the element type that `dtype` names
template <typename F> inline void with_dtype(int dtype, F &&f) {
    if (dtype == XSM_F32) f(float());
    else if (dtype == XSM_BF16) f(bf16());
    else f(__half());
}

}  // namespace xsm
