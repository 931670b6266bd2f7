// Tiled matrix products of the operators on a caller's own activations and weights, on tcgen05: one persistent kernel, several things that it
// can do with a finished tile (xsm_product.cu, xsm_linear.cu, xsm_gated.cu).
#pragma once
#include "xsm_chain.cuh"
#include "xsm_ops.h"

#include <cuda.h>

namespace xsm {

enum ProductEpi {
    PR_STATS,        // maximum and sum of exponentials of a row's logits, the token's logit
    PR_DLOGITS,      // gradient by the logits
    PR_GATED,        // act(gate) * up
    PR_GATED_GRAD,   // gradients by gate and up
    PR_OUT           // the sums themselves: one or two products of B whose rows run along the summed axis
};
enum Activation { ACT_SILU = 0, ACT_GELU = 1 };

constexpr int kAmaxBlocks = 256;
constexpr int kMostRows = 1 << 30;      // of an operand, and elements of one: a tile's last row and column are then ints too

constexpr int kSumCounters = 2048;      // words that PR_OUT counts in

// One product of a launch.
struct ProductPart {
    int m, n;                       // rows and columns of the result (PR_GATED*: n columns of gate and of up)
    int first, tiles;               // number of its first tile, tiles of it
    int tiles_m, group_m;           // tiles of rows, how many of them are worked on side by side
    int jobs, splits;
    int kb0, kb;                    // stages along the summed axis: of the first pair of operands, of all
    int kb_each, kb_more;           // stages of a split, and how many splits have one more
    Divisor by_plane, by_group, by_rows, by_last_rows, by_splits;      // tiles of a split, of a group, rows of a group, of the last one
    int a_rows;                     // rows of a box of A (whose rows lie across the summed axis)
    uint32_t stage_tx;              // bytes of a stage of all CTAs of a tile

    // PR_OUT
    int rows_a;                     // A's rows run along the summed axis
    int map_a, map_b, map_out;      // the first of its descriptions
    float *partial;                 // where there are splits: their sums
    int apart;                      // so many splits that a kernel of its own adds them up
    float *sums;                    // where the result is made in several launches: fp32 sums so far, NULL: made in this one
    int go_on, end;                 // add to them; this is the last
    unsigned counters;              // the first of its counters
    void *out[2];                   // of each job
    long long out_ld;
};
struct __align__(64) ProductMaps { CUtensorMap a[4], b[4], out[3]; };      // (stages of several blocks: a[1], b[2], b[3] are what is left of the rows)

struct ProductArgs {
    ProductPart part[2];
    int tiles;
    int chunks;                     // blocks of 64 that a stage holds
    int tail;                       // with several: the last stage holds what is left of the rows behind whole blocks
    int stages;                     // of the ring
    uint32_t stage, stage_b;        // bytes of a CTA's stage, where B begins in it
    int tma_out;                    // wide tiles: results leave by TMA
    int round;                      // PR_STATS, PR_DLOGITS, one CTA a tile: stages after which the sums so far are added up outside the tensor core
    long long low;                  // elements from a gradient (PR_OUT: from A) to what its rounding left, of few rows; 0: that is let go
    unsigned tries;                 // of a barrier, before a wait gives up
    int starve;                     // fetch nothing (xsm_debug_product_waits)
    int *status;

    // PR_STATS, PR_DLOGITS
    const void *tokens;
    long long token_ld;
    int token_bytes, vocab0, vocab; // first token of this piece of the vocabulary, all tokens
    float c, inv_t;                 // log2(e) / T, 1 / T
    double to_lse;                  // 1 / (c T)
    float2 *parts;                  // [part][m]: maximum, sum
    int carry;                      // one tile of rows: a CTA's parts are joined in its registers, parts are the CTAs'
    unsigned *counter;              // with carry: the CTA that comes last joins the CTAs' parts, [m][part], itself
    float *logprob, *lse_out, *kept;        // kept: logprob once more, may be NULL
    float *token_z;                 // [m], the token's sum
    const float *lse, *g, *g_lse;
    const float *given;             // PR_DLOGITS: the forward pass' logprob, may be NULL
    long long g_ld, g_lse_ld;

    // PR_GATED_GRAD reads g_y, PR_GATED* and PR_DLOGITS write 16-bit rows
    int activation;
    const void *g_y;
    long long g_y_ld;
    void *out[2];                   // PR_GATED_GRAD: gate's, up's
    long long out_ld;
    // fp16, whose smallest number is 2^-24: a power of two of every row's gradients, [m], and one of all; NULL: none.  PR_DLOGITS and PR_GATED_GRAD leave them for PR_OUT, and the operand
    // of the weights' gradients with rows scaled by the power of all over their own (h_out; NULL: nobody needs it).
    float *row_scale, *all_scale;
    const float *bounds;            // PR_GATED_GRAD: [m], times the largest of amax's second kAmaxBlocks numbers no less than any element of a row's gradients
    const float *amax;              // the largest of rows' bounds is that of the first kAmaxBlocks
    int look;                       // PR_DLOGITS: it is looked for here instead
    const void *h;                  // [m][d]
    void *h_out;
    long long h_ld, h_out_ld;
    int d;
};

// A row's maximum (times log2(e) / T) and sum of exponentials, joined part by part.
struct RowSums {
    float m = -INFINITY, sum = 0.f;
    __device__ __forceinline__ void take(float2 p) {
        const float was = m;
        m = fmaxf(m, p.x);
        const float base = m == -INFINITY ? 0.f : m;
        sum = sum * ex2(was - base) + p.y * ex2(p.x - base);
    }
    __device__ __forceinline__ void across_lanes() {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) take(make_float2(__shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, sum, o)));
    }
    // The maximum and the sums share what rounding c x maximum left, and all logits what they have in common: the token's logit less the maximum, less the logarithm of the sum, is off by
    // its own size's rounding.  (z - lse is off by that of the logits: 3e-5 at 300, and above zero as often as below.)
    __device__ __forceinline__ void finish(const void *tokens, long long token_ld, int token_bytes, int vocab, int row, const float *token_z, float c, double to_lse, float *logprob, float *lse, float *kept) const {
        const float s = log2f(sum), l = m == -INFINITY && sum == 0.f ? -INFINITY : (float)(((double)m + s) * to_lse);
        const long long t = token_bytes == 8 ? reinterpret_cast<const long long *>(tokens)[row * token_ld] : (long long)reinterpret_cast<const int *>(tokens)[row * token_ld];
        lse[row] = l;
        float p = 0.f;
        if (t >= 0 && t < vocab) {
            p = l == -INFINITY ? l : (fmaf(__ldcg(token_z + row), c, -m) - s) * 0.69314718056f;
            if (p > 0.f) p = 0.f;
        }
        logprob[row] = p;
        if (kept) kept[row] = p;
    }
};

// How a product is cut: `wide`: two CTAs share tiles of 256 x 256; otherwise a CTA has tiles of 128 x bn.  gated: half of the columns are gate's, half up's, and a
// tile is half as wide.
struct ProductCut {
    bool wide;
    int bn;
    int tm() const { return wide ? 256 : 128; }
    int tn(bool gated) const { return gated ? bn / 2 : bn; }
    long long tiles(long long m, long long n, bool gated) const { return ((m + tm() - 1) / tm()) * ((n + tn(gated) - 1) / tn(gated)); }
};
// few rows, or few columns: gradients by logits, gate and up are held in two parts
bool product_few(ProductEpi epi, long long m, long long n);
// out [m][n] over rows of d; epi: what is done with it (not PR_OUT: plan_sums)
ProductCut product_cut(ProductEpi epi, long long m, long long n, long long d);

// An operand in memory: `rows` rows of `row` elements, ld elements apart.
struct Operand { const void *p; long long rows, row, ld; };

// CTAs that a product of so many tiles runs on
int product_ctas(long long tiles, bool wide);
// Fills in the cut (tiles, boxes, descriptions) of A and launches: a . b^T [m][n], or with both b (PR_GATED*).
cudaError_t launch_product(ProductEpi epi, int dtype, ProductCut cut, ProductArgs A, int m, int n, const Operand &a, const Operand (&b)[2], cudaStream_t st);

// Two products in one launch, of each the results that are wanted:  x = sum over pairs of g[i] . w[i]  [rows][d],  y[i] = g[i]^T . h  [cols][d].
struct SumsPlan {
    ProductCut cut;
    int splits_x, splits_y;
    size_t partial_x, partial_y, bytes;      // fp32 sums of splits, in bytes from the beginning of their place
};
struct Sums {
    int pairs;
    Operand g[2], w[2], h;
    long long low;                  // elements from g to what its rounding left, 0: nothing
    void *x, *y[2];
    long long x_ld, y_ld;
    float *x_sums;                  // fp32 sums of x over several launches, NULL: one launch
    int go_on, end;
    char *partial;
    unsigned *counters;             // kSumCounters words
    float *row_scale, *all_scale;   // of g's rows, fp16; h's rows are scaled by the latter over the former
    int *status;
};
SumsPlan plan_sums(long long rows, long long cols, long long d, int pairs, bool x, bool y, bool once, bool low);      // once: x is made in one launch; low: g in two parts
size_t sums_bytes(const ProductCut &cut, long long rows, long long d);      // of x_sums
cudaError_t launch_sums(int dtype, const SumsPlan &p, const Sums &s, cudaStream_t st);

// What the gradients by rows' logits may be at most; [kAmaxBlocks].
cudaError_t launch_amax_losses(const ProductArgs &A, int rows, float *amax, cudaStream_t st);

// What gate's and up's gradients of fp16 rows may be at most, infinities and NaN apart: |up act'(gate)| <= 1.13 |x| |w_up|, |act(gate)| <= |x| |w_gate| (Cauchy and Schwarz; no derivative of silu or
// gelu is above 1.13).
struct GatedSizes {
    Operand x, g, w[2];             // w: gate's, up's
    float *bounds;                  // [rows]: the largest |g| times |x|
    float *amax;                    // [2][kAmaxBlocks]: of bounds, of the weights' factor
};
cudaError_t launch_gated_sizes(const GatedSizes &s, cudaStream_t st);

int product_sms();
void product_waits(unsigned *tries, int *starve);

}  // namespace xsm
