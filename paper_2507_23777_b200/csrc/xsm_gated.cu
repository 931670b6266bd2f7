// The gated feed-forward part of a block: out = act(x . w_gate) * (x . w_up), both projections, the activation and the product in one kernel, and its gradients.
//
// A tile's columns are as many of gate as of up, so that both sums of an output lie in the same thread's tensor memory.  Backward: gate and up are computed
// again and turned into their gradients where the products leave them (gate's and up's, rounded to the operands' type, of few rows in two parts), then
// dx = d_gate . w_gate + d_up . w_up is one product over both, d_w_gate = d_gate^T . x and d_w_up = d_up^T . x: one launch for all three.  (Gate and up kept in 16 bits
// would spare a quarter of the work and double the gradients' error; kept in fp32 they cost as much to move as to compute.)
//
// What bounds it.  8192 rows, 4096 of 1024: forward 91 us = 1.51 PFLOP/s, gradient 307 = 1.34: 104 us for gate and up again, 190 for 256 tiles of 74 at a time, which
// leave the last round half empty.  4001 rows, 8192 of 2048: 191 us, 1.41 PFLOP/s.  Five rows, 4096 of 1024: 8 us, of which the weights' bytes are 2.6.
#include "xsm_product.cuh"

namespace xsm {

static size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

struct GatedGradPlan {
    ProductCut cut;
    SumsPlan sums;
    int ld;
    long long low;
    size_t amax, all, scale, bounds, x, d_gate, d_up, part, bytes;
};
static GatedGradPlan plan_gated_grad(int rows, int ff, int d, bool x, bool w) {
    GatedGradPlan p;
    const bool few = product_few(PR_GATED_GRAD, rows, ff);
    p.cut = product_cut(PR_GATED_GRAD, rows, ff, d);
    p.sums = plan_sums(rows, ff, d, 2, x, w, true, few);
    p.ld = (ff + 7) / 8 * 8;
    p.amax = 0;
    p.all = up(2 * kAmaxBlocks * 4);
    p.scale = p.all + 256;
    p.bounds = p.scale + up((size_t)rows * 4);
    p.x = p.bounds + up((size_t)rows * 4);
    p.d_gate = p.x + (w ? up((size_t)rows * d * 2) : 0);
    const size_t one = up((size_t)rows * p.ld * 2);
    p.low = few ? (long long)one : 0;        // (in elements: behind both)
    p.d_up = p.d_gate + one;
    p.part = p.d_up + (few ? 3 : 1) * one;
    p.bytes = p.part + up(p.sums.bytes);
    return p;
}

static const char *wrong_shape(int rows, int ff, int d, int dtype, int activation) {
    if (dtype != XSM_BF16 && dtype != XSM_F16) return "dtype must be 1 (bf16) or 2 (fp16)";
    if (rows < 0 || ff < 1 || d < 8 || d % 8) return "rows must not be negative, ff positive, d a positive multiple of 8";
    if (rows > kMostRows || ff > kMostRows || d > kMostRows) return "rows, ff and d must not exceed 2^30";
    if (activation != ACT_SILU && activation != ACT_GELU) return "activation must be 0 (silu) or 1 (gelu)";
    return nullptr;
}
static bool rows_fit(const void *p, int64_t ld, int d) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && ld >= d; }

}  // namespace xsm

using namespace xsm;

xsm_status xsm_gated_ff(const xsm_gated_ff_args *a, void *cuda_stream) {
    if (!a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (const char *w = wrong_shape(a->rows, a->ff, a->d, a->dtype, a->activation)) return op_failed(XSM_ERR_INVALID_ARG, w);
    if (a->rows == 0) return XSM_OK;
    if (!a->x || !a->w_gate || !a->w_up || !a->out || !a->status) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (!rows_fit(a->x, a->x_stride, a->d) || !rows_fit(a->w_gate, a->w_gate_stride, a->d) || !rows_fit(a->w_up, a->w_up_stride, a->d))
        return op_failed(XSM_ERR_INVALID_ARG, "rows of x, w_gate and w_up must be 16-byte aligned and must not overlap");
    if ((uintptr_t)a->out % 2 || a->out_stride < a->ff || (uintptr_t)a->status % 4) return op_failed(XSM_ERR_INVALID_ARG, "out and status must be aligned to their elements, rows of out must not overlap");
    ProductArgs A = {};
    A.status = a->status; A.activation = a->activation;
    A.out[0] = a->out; A.out_ld = a->out_stride;
    const Operand x = {a->x, a->rows, a->d, a->x_stride}, w[2] = {{a->w_gate, a->ff, a->d, a->w_gate_stride}, {a->w_up, a->ff, a->d, a->w_up_stride}};
    return launched(launch_product(PR_GATED, a->dtype, product_cut(PR_GATED, a->rows, a->ff, a->d), A, a->rows, a->ff, x, w, (cudaStream_t)cuda_stream));
}

size_t xsm_gated_ff_grad_workspace(int rows, int ff, int d) {
    if (rows < 1 || ff < 1 || d < 1 || rows > kMostRows || ff > kMostRows || d > kMostRows) return 0;
    const size_t a = plan_gated_grad(rows, ff, d, true, true).bytes, b = plan_gated_grad(rows, ff, d, true, false).bytes, c = plan_gated_grad(rows, ff, d, false, true).bytes;
    return a > b ? (a > c ? a : c) : b > c ? b : c;
}

xsm_status xsm_gated_ff_grad(const xsm_gated_ff_grad_args *a, void *cuda_stream) {
    if (!a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (const char *w = wrong_shape(a->rows, a->ff, a->d, a->dtype, a->activation)) return op_failed(XSM_ERR_INVALID_ARG, w);
    if (!a->d_x && !a->d_w_gate && !a->d_w_up) return XSM_OK;
    if (!a->d_w_gate != !a->d_w_up) return op_failed(XSM_ERR_INVALID_ARG, "d_w_gate and d_w_up go together");
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    if (a->d_w_gate && (!rows_fit(a->d_w_gate, a->d_w_stride, a->d) || !rows_fit(a->d_w_up, a->d_w_stride, a->d)))
        return op_failed(XSM_ERR_INVALID_ARG, "rows of d_w_gate and d_w_up must be 16-byte aligned and must not overlap");
    if (a->rows == 0) {
        cudaError_t e = cudaSuccess;
        if (a->d_w_gate) e = cudaMemset2DAsync(a->d_w_gate, (size_t)a->d_w_stride * 2, 0, (size_t)a->d * 2, (size_t)a->ff, st);
        if (a->d_w_gate && e == cudaSuccess) e = cudaMemset2DAsync(a->d_w_up, (size_t)a->d_w_stride * 2, 0, (size_t)a->d * 2, (size_t)a->ff, st);
        return launched(e);
    }
    if (!a->x || !a->w_gate || !a->w_up || !a->g_out || !a->workspace || !a->status || !a->counters) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (!rows_fit(a->x, a->x_stride, a->d) || !rows_fit(a->w_gate, a->w_gate_stride, a->d) || !rows_fit(a->w_up, a->w_up_stride, a->d) || (a->d_x && !rows_fit(a->d_x, a->d_x_stride, a->d)))
        return op_failed(XSM_ERR_INVALID_ARG, "rows of x, w_gate, w_up and d_x must be 16-byte aligned and must not overlap");
    if ((uintptr_t)a->g_out % 2 || a->g_out_stride < 0 || ((uintptr_t)a->status | (uintptr_t)a->counters) % 4 || (uintptr_t)a->workspace % 16)
        return op_failed(XSM_ERR_INVALID_ARG, "g_out, status and counters must be aligned to their elements, workspace to 16 bytes");
    const GatedGradPlan p = plan_gated_grad(a->rows, a->ff, a->d, a->d_x, a->d_w_gate);
    if (a->workspace_bytes < (int64_t)p.bytes) return op_failed(XSM_ERR_CAPACITY, "the workspace is too small");
    char *ws = (char *)a->workspace;
    ProductArgs A = {};
    A.status = a->status; A.activation = a->activation;
    A.g_y = a->g_out; A.g_y_ld = a->g_out_stride;
    A.out[0] = ws + p.d_gate; A.out[1] = ws + p.d_up; A.out_ld = p.ld; A.low = p.low;
    cudaError_t e = cudaSuccess;
    const Operand x = {a->x, a->rows, a->d, a->x_stride}, w[2] = {{a->w_gate, a->ff, a->d, a->w_gate_stride}, {a->w_up, a->ff, a->d, a->w_up_stride}};
    Sums S = {};
    S.pairs = 2; S.low = p.low;
    S.h = x;
    if (a->dtype == XSM_F16) {        // fp16 has no numbers below 2^-24 and none above 65504: a row's largest possible gradient by gate or up is taken to 2^13 and more
        S.row_scale = A.row_scale = (float *)(ws + p.scale);
        S.all_scale = A.all_scale = (float *)(ws + p.all);
        A.bounds = (const float *)(ws + p.bounds);
        A.amax = (const float *)(ws + p.amax);
        if (a->d_w_gate) {
            A.h = a->x; A.h_ld = a->x_stride; A.h_out = ws + p.x; A.h_out_ld = A.d = a->d;
            S.h = {ws + p.x, a->rows, a->d, a->d};
        }
        e = launch_gated_sizes({x, {a->g_out, a->rows, a->ff, a->g_out_stride}, {w[0], w[1]}, (float *)(ws + p.bounds), (float *)(ws + p.amax)}, st);
    }
    if (e == cudaSuccess) e = launch_product(PR_GATED_GRAD, a->dtype, p.cut, A, a->rows, a->ff, x, w, st);
    for (int i = 0; i < 2; ++i) { S.g[i] = {A.out[i], a->rows, a->ff, p.ld}; S.w[i] = w[i]; }
    S.x = a->d_x; S.x_ld = a->d_x_stride;
    S.y[0] = a->d_w_gate; S.y[1] = a->d_w_up; S.y_ld = a->d_w_stride;
    S.end = 1;
    S.partial = ws + p.part;
    S.counters = a->counters; S.status = a->status;
    if (e == cudaSuccess) e = launch_sums(a->dtype, p.sums, S, st);
    return launched(e);
}
