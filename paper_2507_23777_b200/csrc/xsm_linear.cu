// Log probabilities of given tokens straight from hidden states and the weights of an output projection, and their gradients: the logits of a tile are
// worked on where the products leave them and are never in memory.
//
// Forward: z = hidden . weight / T; every tile of 256 (few rows: a CTA's tiles) tokens of the vocabulary gives a row two pairs (maximum, sum of exponentials), which a second
// kernel joins, or, of few rows, the CTA that ends last: lse = max + log sum.  Backward, in pieces of the vocabulary: the logits once more, p = exp(z - lse),
// d = ([token] g - p (g - g_lse)) / T rounded to the operands' type, then d_hidden = d . weight and d_weight = d^T . hidden in one launch.  d in 16 bits: these products
// are two thirds of the work; it doubles the square of the gradients' error (a rounding before the sum next to the one behind it).  Few rows, where the weights' bytes are the
// time and single elements of d the gradient, also have what the rounding left.
//
// What bounds it.  8192 rows, 32003 tokens, 2048 wide: 3.3 ms for four products of 1.07 TFLOP (three without the logits again), 1.31 PFLOP/s under the power limit, 93 % of what the
// library's own product sustains.  4096 x 4096 x 1024: 29 + 76 us, three launches' beginnings and ends in it.  1999 x 5003 x 768: 21 + 46, in fp16 with its scales 49.
#include "xsm_product.cuh"

#include <math.h>

namespace xsm {

constexpr long long kPieceBytes = 256ll << 20;      // of a piece's gradients by the logits
constexpr int kRowsLookedThrough = 8192;            // so many rows every CTA looks through for the largest gradient, beside its first products

// Eight rows a block; thread (row, y) joins parts y, y + 32, ...  (32 rows a block, eight threads a row: 145 us for 96 rows of 4096 parts.)
__global__ void __launch_bounds__(256) join_stats_kernel(const float2 *parts, const float *token_z, const void *tokens, long long token_ld, int token_bytes, int rows, int vocab,
                                                         int n, float c, double to_lse, float *logprob, float *lse, float *kept) {
    chain_go();
    chain_wait();
    __shared__ float2 s[32][9];
    const int x = threadIdx.x & 7, y = threadIdx.x >> 3, row = blockIdx.x * 8 + x;
    RowSums r;
    if (row < rows) {
#pragma unroll 4
        for (int i = y; i < n; i += 32) r.take(parts[(long long)i * rows + row]);
    }
    s[y][x] = make_float2(r.m, r.sum);
    __syncthreads();
    // (a warp takes a row: lane = y)
    const int lane = threadIdx.x & 31, at = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (at >= rows) return;
    r.m = s[lane][threadIdx.x >> 5].x;
    r.sum = s[lane][threadIdx.x >> 5].y;
    r.across_lanes();
    if (lane == 0) r.finish(tokens, token_ld, token_bytes, vocab, at, token_z, c, to_lse, logprob, lse, kept);
}

// One tile of rows: a CTA joins what its tiles find in its registers, and there are two parts for each CTA.
struct LinearPlan { ProductCut cut; bool carry; int parts; };
static LinearPlan plan_linear(int rows, int vocab, int d) {
    LinearPlan p;
    p.cut = product_cut(PR_STATS, rows, vocab, d);
    p.carry = rows <= p.cut.tm();
    const long long tiles = p.cut.tiles(p.cut.tm(), vocab, false);
    p.parts = 2 * (p.carry ? product_ctas(tiles, p.cut.wide) / (p.cut.wide ? 2 : 1) : (int)tiles);
    return p;
}

static size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

struct LinearGradPlan {
    ProductCut cut_z;
    SumsPlan sums;
    int piece, pieces;
    long long low;
    size_t amax, all, scale, hidden, dz, part, acc, bytes;      // offsets in the workspace
};
static LinearGradPlan plan_linear_grad(int rows, int vocab, int d, bool h, bool w) {
    LinearGradPlan p;
    const bool few = product_few(PR_DLOGITS, rows, vocab);
    const int each = few ? 4 : 2;
    long long piece = kPieceBytes / each / rows / 256 * 256;
    if (piece < 1024) piece = 1024;
    p.pieces = (int)((vocab + piece - 1) / piece);
    p.piece = (int)(((vocab + p.pieces - 1) / p.pieces + 255) / 256 * 256);
    if (p.piece > vocab) p.piece = (vocab + 63) / 64 * 64;
    p.pieces = (vocab + p.piece - 1) / p.piece;
    p.cut_z = product_cut(PR_DLOGITS, rows, p.piece, d);
    p.sums = plan_sums(rows, p.piece, d, 1, h, w, p.pieces == 1, few);
    p.amax = 0;
    p.all = up(kAmaxBlocks * 4);
    p.scale = p.all + 256;
    p.hidden = p.scale + up((size_t)rows * 4);
    p.dz = p.hidden + (w ? up((size_t)rows * d * 2) : 0);
    const size_t dz = up((size_t)rows * p.piece * 2);
    p.low = few ? (long long)(dz / 2) : 0;
    p.part = p.dz + (few ? 2 : 1) * dz;
    p.acc = p.part + up(p.sums.bytes);
    p.bytes = p.acc + (p.pieces > 1 && h ? up(sums_bytes(p.sums.cut, rows, d)) : 0);
    return p;
}

static const char *wrong_shape(int rows, int vocab, int d, int dtype, int token_bytes, float temperature) {
    if (dtype != XSM_BF16 && dtype != XSM_F16) return "dtype must be 1 (bf16) or 2 (fp16)";
    if (rows < 0 || vocab < 1 || d < 8 || d % 8) return "rows must not be negative, vocab positive, d a positive multiple of 8";
    if (rows > kMostRows || vocab > kMostRows || d > kMostRows) return "rows, vocab and d must not exceed 2^30";
    if (token_bytes != 4 && token_bytes != 8) return "token_bytes must be 4 or 8";
    if (!(temperature > 0.f) || !(temperature < INFINITY) || !((float)(1.4426950408889634 / temperature) < INFINITY)) return "temperature must be positive and finite, and log2(e) times its reciprocal finite";
    return nullptr;
}
static bool rows_fit(const void *p, int64_t ld, int d) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && ld >= d; }

}  // namespace xsm

using namespace xsm;

size_t xsm_linear_logprobs_workspace(int rows, int vocab, int d) {
    if (rows < 1 || vocab < 1 || d < 1 || rows > kMostRows || vocab > kMostRows || d > kMostRows) return 0;
    return up((size_t)plan_linear(rows, vocab, d).parts * rows * 8) + up((size_t)rows * 4);
}

xsm_status xsm_linear_logprobs(const xsm_linear_logprobs_args *a, void *cuda_stream) { return xsm_linear_logprobs_keep(a, nullptr, cuda_stream); }

xsm_status xsm_linear_logprobs_keep(const xsm_linear_logprobs_args *a, float *kept, void *cuda_stream) {
    if (!a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (const char *w = wrong_shape(a->rows, a->vocab, a->d, a->dtype, a->token_bytes, a->temperature)) return op_failed(XSM_ERR_INVALID_ARG, w);
    if (a->rows == 0) return XSM_OK;
    if (!a->hidden || !a->weight || !a->tokens || !a->logprob || !a->lse || !a->workspace || !a->status) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (!rows_fit(a->hidden, a->hidden_stride, a->d) || !rows_fit(a->weight, a->weight_stride, a->d))
        return op_failed(XSM_ERR_INVALID_ARG, "rows of hidden and weight must be 16-byte aligned and must not overlap");
    if ((uintptr_t)a->tokens % a->token_bytes || ((uintptr_t)a->logprob | (uintptr_t)kept | (uintptr_t)a->lse | (uintptr_t)a->status | (uintptr_t)a->counters) % 4 || (uintptr_t)a->workspace % 16)
        return op_failed(XSM_ERR_INVALID_ARG, "tokens, logprob, lse, status and counters must be aligned to their elements, workspace to 16 bytes");
    if (a->workspace_bytes < (int64_t)xsm_linear_logprobs_workspace(a->rows, a->vocab, a->d)) return op_failed(XSM_ERR_CAPACITY, "the workspace is too small");
    const LinearPlan p = plan_linear(a->rows, a->vocab, a->d);
    ProductArgs A = {};
    A.status = a->status;
    A.tokens = a->tokens; A.token_ld = a->token_stride; A.token_bytes = a->token_bytes; A.vocab = a->vocab;
    A.inv_t = 1.f / a->temperature;
    A.c = (float)(1.4426950408889634 / a->temperature);
    A.to_lse = 1.0 / ((double)A.c * a->temperature);
    A.parts = (float2 *)a->workspace;
    A.carry = p.carry;
    // (few rows: the last CTA joins the parts itself, 5 x 4096 7.8 -> 7.3 us and a launch less; of 96 rows that takes one CTA 15 us)
    if (p.carry && !p.cut.wide && a->rows <= 16) A.counter = a->counters;
    A.logprob = a->logprob; A.lse_out = a->lse; A.kept = kept;
    A.token_z = (float *)((char *)a->workspace + up((size_t)p.parts * a->rows * 8));
    const Operand h = {a->hidden, a->rows, a->d, a->hidden_stride}, w[2] = {{a->weight, a->vocab, a->d, a->weight_stride}, {}};
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e = launch_product(PR_STATS, a->dtype, p.cut, A, a->rows, a->vocab, h, w, st);
    if (e == cudaSuccess && !A.counter)
        e = launch_early(join_stats_kernel, dim3((unsigned)((a->rows + 7) / 8)), dim3(256), 0, st, (const float2 *)A.parts, (const float *)A.token_z, a->tokens, (long long)a->token_stride,
                         (int)a->token_bytes, (int)a->rows, (int)a->vocab, (int)p.parts, A.c, A.to_lse, a->logprob, a->lse, kept);
    return launched(e);
}

size_t xsm_linear_logprobs_grad_workspace(int rows, int vocab, int d) {
    if (rows < 1 || vocab < 1 || d < 1 || rows > kMostRows || vocab > kMostRows || d > kMostRows) return 0;
    const size_t a = plan_linear_grad(rows, vocab, d, true, true).bytes, b = plan_linear_grad(rows, vocab, d, true, false).bytes, c = plan_linear_grad(rows, vocab, d, false, true).bytes;
    return a > b ? (a > c ? a : c) : b > c ? b : c;
}

xsm_status xsm_linear_logprobs_grad(const xsm_linear_logprobs_grad_args *a, void *cuda_stream) { return xsm_linear_logprobs_grad_near(a, nullptr, cuda_stream); }

xsm_status xsm_linear_logprobs_grad_near(const xsm_linear_logprobs_grad_args *a, const float *logprob, void *cuda_stream) {
    if (!a) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (const char *w = wrong_shape(a->rows, a->vocab, a->d, a->dtype, a->token_bytes, a->temperature)) return op_failed(XSM_ERR_INVALID_ARG, w);
    if (!a->d_hidden && !a->d_weight) return XSM_OK;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    if (a->d_weight && !rows_fit(a->d_weight, a->d_weight_stride, a->d)) return op_failed(XSM_ERR_INVALID_ARG, "rows of d_weight must be 16-byte aligned and must not overlap");
    if (a->rows == 0)
        return a->d_weight ? launched(cudaMemset2DAsync(a->d_weight, (size_t)a->d_weight_stride * 2, 0, (size_t)a->d * 2, (size_t)a->vocab, st)) : XSM_OK;
    if (!a->hidden || !a->weight || !a->tokens || !a->lse || !a->workspace || !a->status || !a->counters) return op_failed(XSM_ERR_INVALID_ARG, "null argument");
    if (!rows_fit(a->hidden, a->hidden_stride, a->d) || !rows_fit(a->weight, a->weight_stride, a->d) || (a->d_hidden && !rows_fit(a->d_hidden, a->d_hidden_stride, a->d)))
        return op_failed(XSM_ERR_INVALID_ARG, "rows of hidden, weight and d_hidden must be 16-byte aligned and must not overlap");
    if ((uintptr_t)a->tokens % a->token_bytes || ((uintptr_t)a->lse | (uintptr_t)logprob | (uintptr_t)a->g_logprob | (uintptr_t)a->g_lse | (uintptr_t)a->status | (uintptr_t)a->counters) % 4 || (uintptr_t)a->workspace % 16)
        return op_failed(XSM_ERR_INVALID_ARG, "tokens, lse, logprob, g_logprob, g_lse, status and counters must be aligned to their elements, workspace to 16 bytes");
    const LinearGradPlan p = plan_linear_grad(a->rows, a->vocab, a->d, a->d_hidden, a->d_weight);
    if (a->workspace_bytes < (int64_t)p.bytes) return op_failed(XSM_ERR_CAPACITY, "the workspace is too small");
    char *ws = (char *)a->workspace;
    ProductArgs Z = {};
    Z.status = a->status;
    Z.tokens = a->tokens; Z.token_ld = a->token_stride; Z.token_bytes = a->token_bytes; Z.vocab = a->vocab;
    Z.inv_t = 1.f / a->temperature;
    Z.c = (float)(1.4426950408889634 / a->temperature);
    Z.lse = a->lse; Z.given = logprob; Z.g = a->g_logprob; Z.g_ld = a->g_logprob_stride; Z.g_lse = a->g_lse; Z.g_lse_ld = a->g_lse_stride;
    Z.out[0] = ws + p.dz; Z.out_ld = p.piece; Z.low = p.low;
    Sums S = {};
    S.pairs = 1; S.low = p.low;
    const Operand hidden = {a->hidden, a->rows, a->d, a->hidden_stride};
    S.h = hidden;
    S.x = a->d_hidden; S.x_ld = a->d_hidden_stride; S.y_ld = a->d_weight_stride;
    S.x_sums = p.pieces > 1 ? (float *)(ws + p.acc) : nullptr;
    S.partial = ws + p.part;
    S.counters = a->counters; S.status = a->status;
    cudaError_t e = cudaSuccess;
    if (a->dtype == XSM_F16) {        // fp16 has no numbers below 2^-24: a row's largest possible gradient by a logit is taken to 2^13 and more
        S.row_scale = Z.row_scale = (float *)(ws + p.scale);
        S.all_scale = Z.all_scale = (float *)(ws + p.all);
        if (a->d_weight) {
            Z.h = a->hidden; Z.h_ld = a->hidden_stride; Z.h_out = ws + p.hidden; Z.h_out_ld = Z.d = a->d;
            S.h = {ws + p.hidden, a->rows, a->d, a->d};
        }
        Z.look = a->rows <= kRowsLookedThrough;
        if (!Z.look) {
            Z.amax = (const float *)(ws + p.amax);
            e = launch_amax_losses(Z, a->rows, (float *)(ws + p.amax), st);
        }
    }
    for (int i = 0; i < p.pieces && e == cudaSuccess; ++i) {
        const int v0 = i * p.piece, v = a->vocab - v0 < p.piece ? a->vocab - v0 : p.piece;
        const Operand w[2] = {{(const char *)a->weight + (long long)v0 * a->weight_stride * 2, v, a->d, a->weight_stride}, {}};
        Z.vocab0 = v0;
        e = launch_product(PR_DLOGITS, a->dtype, p.cut_z, Z, a->rows, v, hidden, w, st);
        Z.h_out = nullptr;        // (the first one's stay)
        S.g[0] = {ws + p.dz, a->rows, v, p.piece};
        S.w[0] = w[0];
        S.y[0] = a->d_weight ? (char *)a->d_weight + (long long)v0 * a->d_weight_stride * 2 : nullptr;
        S.go_on = i > 0;
        S.end = i == p.pieces - 1;
        if (e == cudaSuccess) e = launch_sums(a->dtype, p.sums, S, st);
    }
    return launched(e);
}
