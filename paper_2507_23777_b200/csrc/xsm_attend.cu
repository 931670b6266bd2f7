// Attention of the newest tokens of each sequence over a caller's paged pools (xsm_kv).
#include "xsm_ops.h"

#include <limits.h>
#include <math.h>

namespace xsm {

struct AttendArgs {
    const void *q;
    void *out;
    float *lse;
    const int *lengths, *counts;
    long long qs[3], os[3];
    int m, heads, group, causal, window;
    float scale;
};

// One block for every query row of every head: its four warps take keys in turn, a lane holds every 32nd element of the row; the online
// softmax of a warp is joined with the others' at the end.
template <typename TQ, typename TC, int DH>
__global__ void __launch_bounds__(128) attend_kernel(const __grid_constant__ AttendArgs A, const __grid_constant__ Pages P) {
    constexpr int E = DH / 32;
    __shared__ float s_o[4][DH], s_m[4], s_l[4];
    const int h = blockIdx.x % A.heads, j = (blockIdx.x / A.heads) % A.m, b = blockIdx.x / (A.heads * A.m);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n_q = A.counts ? min(A.counts[b], A.m) : A.m;
    const long long n = min((long long)A.lengths[b], (long long)P.max_pages * P.size);
    long long end = j < n_q ? n : 0, begin = 0;
    if (A.causal) end = min(end, n - n_q + j + 1);
    if (A.causal && A.window > 0) begin = max(0LL, end - A.window);
    float q[E], o[E], mx = -INFINITY, l = 0.f;
    const TQ *qp = reinterpret_cast<const TQ *>(A.q) + b * A.qs[0] + j * A.qs[1] + h * A.qs[2];
#pragma unroll
    for (int e = 0; e < E; ++e) { q[e] = to_f(qp[lane + 32 * e]) * A.scale; o[e] = 0.f; }
    for (long long t = begin + warp; t < end; t += 4) {
        const int page = P.table[b * P.table_ld + t / P.size];
        if (page < 0 || page >= P.n_pages) continue;
        const long long at = page * P.page + (h / A.group) * P.head + (t % P.size) * P.row;
        const TC *kp = reinterpret_cast<const TC *>(P.k) + at, *vp = reinterpret_cast<const TC *>(P.v) + at;
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s += q[e] * to_f(kp[lane + 32 * e]);
        s = warp_sum(s);
        const float top = fmaxf(mx, s), f = mx == top ? 1.f : expf(mx - top), p = expf(s - top);
        l = l * f + p;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * f + p * to_f(vp[lane + 32 * e]);
        mx = top;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[warp][lane + 32 * e] = o[e];
    if (lane == 0) { s_m[warp] = mx; s_l[warp] = l; }
    __syncthreads();
    const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
    float total = 0.f, f[4];
    for (int w = 0; w < 4; ++w) { f[w] = s_l[w] == 0.f ? 0.f : expf(s_m[w] - top); total += s_l[w] * f[w]; }
    TQ *op = reinterpret_cast<TQ *>(A.out) + b * A.os[0] + j * A.os[1] + h * A.os[2];
    for (int e = threadIdx.x; e < DH; e += 128) {
        float v = 0.f;
        for (int w = 0; w < 4; ++w) v += f[w] == 0.f ? 0.f : s_o[w][e] * f[w];
        op[e] = rounded<TQ>(total == 0.f ? 0.f : v / total);
    }
    if (A.lse && threadIdx.x == 0) A.lse[((long long)b * A.m + j) * A.heads + h] = total == 0.f ? -INFINITY : top + logf(total);
}

}  // namespace xsm

using namespace xsm;

size_t xsm_kv_attend_workspace(const xsm_kv *kv, int batch, int m, int n_heads) {
    if (!kv || batch < 1 || m < 1 || m > XSM_MAX_DRAFT || n_heads < 1) return 0;
    return 16;
}

xsm_status xsm_kv_attend(const xsm_kv *kv, const xsm_kv_attend_args *a, void *cuda_stream) {
    if (!kv || !a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    const xsm_kv_config &c = kv->cfg;
    if (a->batch < 0 || a->max_pages < 0) return op_failed(XSM_ERR_INVALID_ARG, "batch and max_pages must not be negative");
    if (a->m < 1 || a->m > XSM_MAX_DRAFT) return op_failed(XSM_ERR_INVALID_ARG, "m must be in [1, 16]");
    if (a->n_heads < 1 || a->n_heads > 4096 || a->n_heads % c.n_kv_heads) return op_failed(XSM_ERR_INVALID_ARG, "n_heads must be a multiple of n_kv_heads, at most 4096");
    if (!is_dtype(a->q_dtype) || (a->q_dtype != c.dtype && c.dtype != XSM_F16))
        return op_failed(XSM_ERR_INVALID_ARG, "q_dtype must be the pools' type (over an fp16 pool: any)");
    if (a->window < 0 || (a->window && !a->causal)) return op_failed(XSM_ERR_INVALID_ARG, "window must not be negative, and needs causal");
    if (!(fabsf(a->scale) < INFINITY)) return op_failed(XSM_ERR_INVALID_ARG, "scale must be finite");
    if (a->batch == 0) return XSM_OK;
    if (!a->q || !a->out || !a->block_table || !a->lengths || !a->workspace) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (a->workspace_bytes < (int64_t)xsm_kv_attend_workspace(kv, a->batch, a->m, a->n_heads)) return op_failed(XSM_ERR_CAPACITY, "the workspace is too small");
    const int per16 = 16 / element_size(a->q_dtype);
    for (int i = 0; i < 3; ++i)
        if (a->q_stride[i] % per16 || a->out_stride[i] % per16) return op_failed(XSM_ERR_INVALID_ARG, "strides of q and out must be multiples of 16 bytes");
    if (((uintptr_t)a->q | (uintptr_t)a->out | (uintptr_t)a->workspace) % 16) return op_failed(XSM_ERR_INVALID_ARG, "q, out and workspace must be 16-byte aligned");
    const long long rows = (long long)a->batch * a->m * a->n_heads;
    if (rows > INT_MAX) return op_failed(XSM_ERR_INVALID_ARG, "more than 2^31 - 1 rows");
    AttendArgs A;
    A.q = a->q; A.out = a->out; A.lse = a->lse; A.lengths = a->lengths; A.counts = a->counts;
    for (int i = 0; i < 3; ++i) { A.qs[i] = a->q_stride[i]; A.os[i] = a->out_stride[i]; }
    A.m = a->m; A.heads = a->n_heads; A.group = a->n_heads / c.n_kv_heads; A.causal = a->causal != 0; A.window = a->window; A.scale = a->scale;
    const Pages P = pages_of(*kv, a->block_table, a->table_stride, a->max_pages);
    with_dtype(a->q_dtype, [&](auto q) {
        with_dtype(c.dtype, [&](auto s) {
            using TQ = decltype(q);
            using TC = decltype(s);
            const cudaStream_t st = (cudaStream_t)cuda_stream;
            if (c.d_head == 32) attend_kernel<TQ, TC, 32><<<(unsigned)rows, 128, 0, st>>>(A, P);
            else if (c.d_head == 64) attend_kernel<TQ, TC, 64><<<(unsigned)rows, 128, 0, st>>>(A, P);
            else if (c.d_head == 96) attend_kernel<TQ, TC, 96><<<(unsigned)rows, 128, 0, st>>>(A, P);
            else if (c.d_head == 128) attend_kernel<TQ, TC, 128><<<(unsigned)rows, 128, 0, st>>>(A, P);
            else attend_kernel<TQ, TC, 256><<<(unsigned)rows, 128, 0, st>>>(A, P);
        });
    });
    return launched(cudaGetLastError());
}
