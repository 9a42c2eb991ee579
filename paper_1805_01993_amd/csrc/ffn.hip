// The gated feed-forward block, forward and backward: what is launched, and in which order.
#include "product.hpp"

namespace {
using namespace ccdc;

struct SideArgs {
    const void *from;
    uint16_t *to;
    int64_t rows, columns, ld, to_ld, plane;
    uint32_t packs, blocks;               // of a row; workgroups up to the end of this matrix
};
constexpr int kMostSides = 4;
struct SidesArgs {
    SideArgs of[kMostSides];
    int count;
};

// Matrices as sides of products: fp32 numbers as their three parts, 16-bit ones that begin anywhere as rows of whole packs,
// zeros past their ends.  A work item makes a pack; all matrices of a call in one launch (56 files of 37 tokens, 515 x 1333 bf16, four
// launches of 4 us each).  Bound by memory (fp32: four bytes read and six written an element).
template <class T>
__global__ __launch_bounds__(kBlock) void k_sides(const SidesArgs all)
{
    int which = 0;
    while (which + 1 < all.count && blockIdx.x >= all.of[which].blocks) which++;
    const SideArgs &a = all.of[which];
    const uint32_t first = which ? all.of[which - 1].blocks : 0;
    const uint64_t p = (uint64_t)(blockIdx.x - first) * kBlock + threadIdx.x, row = p / a.packs;
    const uint32_t c = (uint32_t)(p - row * a.packs) * 8;
    if (row >= (uint64_t)a.rows) return;
    const Eight v = load_eight<T>((const typename T::elem *)a.from + row * a.ld + c, (int)min(a.columns - c, (int64_t)8));
    store_side<T>(a.to + row * a.to_ld + c, a.plane, v);
}

template <class T>
int run_sides(const SidesArgs &a, hipStream_t st)
{
    k_sides<T><<<a.of[a.count - 1].blocks, kBlock, 0, st>>>(a);
    return launched();
}

constexpr int64_t kSideStride = (int64_t)1 << 24;

// The caller's matrices as sides of products: as they are where rows of 16-bit numbers are whole packs of 16 bytes, no further apart than
// 64 rows' offsets have bits for, else made in the workspace by one launch.
class Sides {
public:
    Sides(const ccdc_block_t *b, hipStream_t st) : b_(b), st_(st) {}
    Side add(const void *p, int64_t ld, int64_t rows, int64_t columns, size_t room)
    {
        if (b_->planes == 1 && columns % 8 == 0 && ld % 8 == 0 && ld <= kSideStride && aligned(p, 16)) return {(const uint16_t *)p, ld, 0, 0, (int32_t)columns};
        const int64_t wide = padded(columns);
        uint16_t *to = inside_of<uint16_t>(b_->d_workspace, room);
        const uint32_t packs = (uint32_t)(wide / 8);
        if (rows > 0) {
            blocks_ += cdiv((uint64_t)rows * packs, kBlock);
            sides_.of[sides_.count++] = {p, to, rows, columns, ld, wide, rows * wide, packs, (uint32_t)blocks_};
        }
        return {to, wide, rows * wide, 0, (int32_t)wide};
    }
    int make()
    {
        if (sides_.count == 0) return CCDC_OK;
        if (!fits_launch(blocks_ * kBlock)) return CCDC_ESIZE;
        const auto run = [&]() -> int { CCDC_BY_ELEM(b_, (run_sides<T>(sides_, st_))); };
        return run();
    }

private:
    const ccdc_block_t *b_;
    hipStream_t st_;
    SidesArgs sides_{};
    uint64_t blocks_ = 0;
};

struct PartsArgs {
    const float *parts;
    void *y;
    int64_t part, ld, ldy;
    int32_t count, width;
    uint32_t rows, packs;
};

// y from its ranges of k, added in their order.
template <class T>
__global__ __launch_bounds__(kBlock) void k_parts(const PartsArgs a)
{
    const uint32_t p = blockIdx.x * kBlock + threadIdx.x, row = p / a.packs, c = (p - row * a.packs) * 8;
    if (row >= a.rows) return;
    const float *from = a.parts + (int64_t)row * a.ld + c;
    Eight sum = load_eight<ElemF32>(from, 8);         // (rows of the ranges are whole packs)
    for (int i = 1; i < a.count; i++) {
        const Eight v = load_eight<ElemF32>(from + i * a.part, 8);
#pragma unroll
        for (int e = 0; e < 8; e++) sum.v[e] += v.v[e];
    }
    store_eight<T>((typename T::elem *)a.y + (int64_t)row * a.ldy + c, sum, a.width - (int)c);
}

template <class T>
int run_parts(const PartsArgs &a, hipStream_t st)
{
    k_parts<T><<<cdiv((uint64_t)a.rows * a.packs, kBlock), kBlock, 0, st>>>(a);
    return launched();
}

// What every product of the block is given.
ProductArgs common(const ccdc_block_t *b)
{
    ProductArgs a{};
    a.segments = a.files = a.halves = 1;
    a.ldh = b->hidden_ld;
    a.plane_h = b->M * b->hidden_ld;
    a.row_of = b->d_row_of;
    a.activation = b->c.activation;
    return a;
}

// The block's own matrix of hidden values.
Side hidden_side(const ccdc_block_t *b, const uint16_t *h)
{
    return {h, b->hidden_ld, b->M * b->hidden_ld, 0, (int32_t)b->hidden_ld};
}

int forward(const ccdc_block_t *b, int64_t rows, const void *x, int64_t ldx, const void *W_in, const void *W_out, void *y, int64_t ldy,
            void *saved, uint64_t seed, hipStream_t st)
{
    const int64_t d = b->c.width, F = b->c.hidden;
    const Dropout drop = make_dropout(b->c.dropout_hidden, 2 * b->c.layer, seed);
    if (!saved && rows <= kFewRows)
        return few_forward(b, rows, x, ldx, W_in, W_out, y, ldy, inside_of(b->d_workspace, b->at_h), drop, st);
    Sides sides(b, st);
    const Side in = sides.add(W_in, d, 2 * F, d, b->at_in), px = sides.add(x, ldx, rows, d, b->at_x);
    const Side out = sides.add(W_out, F, d, F, b->at_out);
    int rc = sides.make();
    if (rc != CCDC_OK) return rc;
    uint16_t *h = saved ? inside_of<uint16_t>(saved, b->saved_h) : inside_of<uint16_t>(b->d_workspace, b->at_h);
    ProductArgs a = common(b);
    a.n = in, a.m = px;
    a.rows_n = (int32_t)F, a.rows_m = (int32_t)rows, a.K = (int32_t)padded(d);
    a.h = h;
    a.P = saved ? inside_of<float>(saved, b->saved_p) : nullptr;
    a.Q = saved ? inside_of<float>(saved, b->saved_q) : nullptr;
    a.drop = drop;
    rc = run_product(b->c.mode, Product::gated, a, st);
    if (rc != CCDC_OK) return rc;
    a = common(b);
    a.n = out, a.m = hidden_side(b, h);
    a.rows_n = (int32_t)d, a.rows_m = (int32_t)rows, a.K = (int32_t)padded(F);
    const int parts = saved ? 1 : forward_parts(d, b->hidden_ld, rows);
    if (parts == 1) {
        a.c = y, a.ldc = ldy;
        return run_product(b->c.mode, Product::plain, a, st);
    }
    float *made = inside_of<float>(b->d_workspace, b->at_parts);
    const int64_t steps = (padded(F) + 63) / 64;
    a.part_k = (int32_t)((steps + parts - 1) / parts * 64);
    a.files = (int32_t)cdiv(padded(F), a.part_k);
    a.c = made, a.ldc = b->width_ld, a.file_c = rows * b->width_ld;
    if ((rc = run_product(b->c.mode, Product::parts, a, st)) != CCDC_OK) return rc;
    const PartsArgs p{made, y, a.file_c, a.ldc, ldy, a.files, (int32_t)d, (uint32_t)rows, (uint32_t)(b->width_ld / 8)};
    CCDC_BY_ELEM(b, (run_parts<T>(p, st)));
}

int backward(const ccdc_block_t *b, const void *x, int64_t ldx, const void *W_in, const void *W_out, const void *saved, const void *dy,
             int64_t lddy, void *dx, int64_t lddx, void *dW_in, int64_t ld_in, void *dW_out, int64_t ld_out, hipStream_t st)
{
    const int64_t d = b->c.width, F = b->c.hidden, M = b->M, Fp = b->hidden_ld;
    Sides sides(b, st);
    const Side out = sides.add(W_out, F, d, F, b->at_out), pdy = sides.add(dy, lddy, M, d, b->at_dy);
    Side in{}, px{};
    if (dx) in = sides.add(W_in, d, 2 * F, d, b->at_in);
    if (dW_in) px = sides.add(x, ldx, M, d, b->at_x);
    int rc = sides.make();
    if (rc != CCDC_OK) return rc;
    // gradients of a and u, side by side: as one range of 2 F where F is whole packs, else as two of F
    const bool one = F == Fp;
    uint16_t *dau = inside_of<uint16_t>(b->d_workspace, b->at_dau);
    ProductArgs a = common(b);
    a.n = out, a.m = pdy;
    a.rows_n = (int32_t)F, a.rows_m = (int32_t)M, a.K = (int32_t)d;
    a.h = dau, a.plane_h = M * 2 * Fp, a.second_h = Fp;
    a.P = inside_of<float>(saved, b->saved_p), a.Q = inside_of<float>(saved, b->saved_q);
    rc = run_product(b->c.mode, Product::gated_gradient, a, st);
    if (rc != CCDC_OK) return rc;
    const Side both{dau, 2 * Fp, M * 2 * Fp, Fp, (int32_t)(one ? 2 * Fp : Fp)};
    if (dW_in) {
        // side N: x or h, side M: gradients, both with the tokens of a file as k
        a = common(b);
        a.first = b->d_first, a.files = b->N, a.file_c = ld_in;
        a.K = (int32_t)(M / b->N);
        a.n = px, a.m = both;
        a.halves = one ? 1 : 2, a.half_c = F * d;
        a.rows_n = (int32_t)d, a.rows_m = (int32_t)(one ? 2 * F : F);
        a.c = dW_in, a.ldc = d;
        if ((rc = run_product(b->c.mode, Product::weight_gradient, a, st)) != CCDC_OK) return rc;
        a.n = hidden_side(b, inside_of<uint16_t>(saved, b->saved_h)), a.m = pdy;
        a.halves = 1;
        a.rows_n = (int32_t)F, a.rows_m = (int32_t)d;
        a.c = dW_out, a.ldc = F, a.file_c = ld_out;
        if ((rc = run_product(b->c.mode, Product::weight_gradient, a, st)) != CCDC_OK) return rc;
    }
    if (!dx) return CCDC_OK;
    a = common(b);
    a.n = in, a.m = both;
    a.n.segment = F * in.ld;
    a.segments = one ? 1 : 2;
    a.rows_n = (int32_t)d, a.rows_m = (int32_t)M, a.K = (int32_t)(one ? 2 * F : F);
    a.c = dx, a.ldc = lddx;
    return run_product(b->c.mode, Product::input_gradient, a, st);      // last: dx may be dy
}

}  // namespace

extern "C" {

int ccdc_ffn_forward(const ccdc_block_t *b, int64_t rows, const void *x, int64_t ldx, const void *W_in, const void *W_out, void *y,
                     int64_t ldy, void *saved, uint64_t seed, void *stream)
{
    const int rc = ready(b);
    if (rc != CCDC_OK) return rc;
    if (rows < 0 || rows > b->M || (saved && rows != b->M) || ldx < b->c.width || ldy < b->c.width) return CCDC_EINVAL;
    if (rows == 0) return CCDC_OK;
    if (!fits(b, x) || !fits(b, W_in) || !fits(b, W_out) || !fits(b, y) || !aligned(saved, 16)) return CCDC_EINVAL;
    WorkspaceOrder order(b, (hipStream_t)stream, true);
    return forward(b, rows, x, ldx, W_in, W_out, y, ldy, saved, seed, (hipStream_t)stream);
}

int ccdc_ffn_backward(const ccdc_block_t *b, const void *x, int64_t ldx, const void *W_in, const void *W_out, const void *saved,
                      const void *dy, int64_t lddy, void *dx, int64_t lddx, void *dW_in, int64_t ld_in, void *dW_out,
                      int64_t ld_out, void *stream)
{
    const int rc = ready(b);
    if (rc != CCDC_OK) return rc;
    const int64_t d = b->c.width, F = b->c.hidden;
    if ((!dx && !dW_in && b->M > 0) || !dW_in != !dW_out || ldx < d || lddy < d || (dx && lddx < d)) return CCDC_EINVAL;
    if (dW_in && b->N > 1 && (ld_in < 2 * F * d || ld_out < d * F)) return CCDC_EINVAL;
    const bool empty = b->M == 0;                 // a batch without tokens has no rows to point at; its gradients are zeros
    if (!fits(b, x, empty) || !fits(b, W_in) || !fits(b, W_out) || !aligned(saved, 16) || (!saved && !empty) || !fits(b, dy, empty) ||
        !fits(b, dx, true) || !fits(b, dW_in, true) || !fits(b, dW_out, true))
        return CCDC_EINVAL;
    if (dx && dx == dy && lddx != lddy) return CCDC_EINVAL;
    WorkspaceOrder order(b, (hipStream_t)stream, true);
    return backward(b, x, ldx, W_in, W_out, saved, dy, lddy, dx, lddx, dW_in, ld_in, dW_out, ld_out,
                    (hipStream_t)stream);
}

}  // extern "C"
