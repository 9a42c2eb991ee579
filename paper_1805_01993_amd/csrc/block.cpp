// The host side of a block: configuration, batch and the sizes of what its calls keep.  No GPU code.
#include "block.hpp"

#include <cmath>
#include <new>

namespace ccdc {
namespace {

constexpr int64_t kMostWidth = (int64_t)1 << 20, kMostRows = INT32_MAX, kMostBytes = (int64_t)1 << 40;

bool probability(float p) { return p >= 0.0f && p <= 1.0f; }

int check(const ccdc_block_config &c)
{
    if (c.width < 1 || c.width > kMostWidth || c.hidden < 1 || c.hidden > kMostWidth) return CCDC_EINVAL;
    if (c.mode != CCDC_F32_SUM && c.mode != CCDC_F32_SUM_XOR && c.mode != CCDC_BF16_SUM_XOR && c.mode != CCDC_F16_SUM_XOR)
        return CCDC_EINVAL;
    if (c.activation < CCDC_ACT_SILU || c.activation > CCDC_ACT_RELU) return CCDC_EINVAL;
    if (c.norm != CCDC_NORM_RMS && c.norm != CCDC_NORM_CENTRED) return CCDC_EINVAL;
    if (c.layer > (uint32_t)INT32_MAX || !(c.eps > 0.0f) || !std::isfinite(c.eps) || !std::isfinite(c.residual_scale))
        return CCDC_EINVAL;
    return probability(c.dropout_hidden) && probability(c.dropout_out) ? CCDC_OK : CCDC_EINVAL;
}

// Takes bytes of a buffer, whole cache lines of them.
size_t take(size_t *at, int64_t bytes)
{
    const size_t from = *at;
    *at += ((size_t)bytes + 255) / 256 * 256;
    return from;
}

}  // namespace

int bind_block(ccdc_block_t *b, int files, const int64_t *tokens, const int32_t *ids)
{
    if (files < 1 || !tokens) return CCDC_EINVAL;
    int64_t M = 0;
    for (int n = 0; n < files; n++) {
        if (tokens[n] < 0 || (ids && ids[n] < 0)) return CCDC_EINVAL;
        if (tokens[n] > kMostRows || (M += tokens[n]) > kMostRows) return CCDC_ESIZE;
    }
    const int64_t width_ld = padded(b->c.width), hidden_ld = padded(b->c.hidden), operand = 2 * b->planes;
    // (each factor is below 2^31 and 2^21, so nothing here passes 63 bits)
    if (M * hidden_ld * 8 + M * hidden_ld * operand > kMostBytes || M * width_ld * operand > kMostBytes ||
        hidden_ld * width_ld * 2 * operand > kMostBytes)
        return CCDC_ESIZE;

    std::vector<int32_t> first(1, 0), chunk_first(1, 0);
    std::vector<RowOf> row_of;
    std::vector<Chunk> chunks;
    row_of.reserve((size_t)M);
    for (int n = 0; n < files; n++) {
        const int32_t id = ids ? ids[n] : n, rows = (int32_t)tokens[n];
        for (int32_t t = 0; t < rows; t++) row_of.push_back({id, t, n});
        each_chunk(rows, [&](int32_t t, int32_t of) { chunks.push_back({n, first[n] + t, of}); });
        first.push_back(first[n] + rows);
        chunk_first.push_back((int32_t)chunks.size());
    }

    size_t at = 0;
    b->saved_h = take(&at, M * hidden_ld * operand);
    b->saved_p = take(&at, M * hidden_ld * 4);
    b->saved_q = take(&at, M * hidden_ld * 4);
    b->saved_bytes = at;
    at = 0;
    b->at_h = take(&at, M * hidden_ld * operand);
    b->at_dau = take(&at, M * 2 * hidden_ld * operand);
    b->at_x = take(&at, M * width_ld * operand);
    b->at_dy = take(&at, M * width_ld * operand);
    b->at_in = take(&at, 2 * b->c.hidden * width_ld * operand);
    b->at_out = take(&at, b->c.width * hidden_ld * operand);
    b->at_parts = take(&at, (M * width_ld < kPartElements / 256 ? M * width_ld * 256 : kPartElements) * 4);
    size_t sums = 0;
    if (b->c.width <= kJoinWidth) take(&sums, (int64_t)chunks.size() * 2 * width_ld * 4);
    b->workspace_bytes = at > sums ? at : sums;

    b->M = M;
    b->N = files;
    b->width_ld = width_ld;
    b->hidden_ld = hidden_ld;
    b->first = std::move(first);
    b->row_of = std::move(row_of);
    b->chunks = std::move(chunks);
    b->chunk_first = std::move(chunk_first);
    b->bound = true;
    return CCDC_OK;
}

}  // namespace ccdc

extern "C" {

int ccdc_block(const ccdc_block_config *config, ccdc_block_t **out)
{
    if (!config || !out) return CCDC_EINVAL;
    const int rc = ccdc::check(*config);
    if (rc != CCDC_OK) return rc;
    ccdc_block_t *b = new (std::nothrow) ccdc_block_s;
    if (!b) return CCDC_ENOMEM;
    b->c = *config;
    b->elem = config->mode == CCDC_BF16_SUM_XOR || config->mode == CCDC_F16_SUM_XOR ? 2 : 4;
    b->planes = b->elem == 2 ? 1 : 3;
    *out = b;
    return CCDC_OK;
}

int ccdc_block_query(const ccdc_block_t *b, int what, void *out, size_t out_bytes)
{
    if (!b || !out) return CCDC_EINVAL;
    if (what < CCDC_BLOCK_Q_TOKENS || what > CCDC_BLOCK_Q_WORKSPACE_BYTES || out_bytes < sizeof(int64_t)) return CCDC_EINVAL;
    if (!b->bound) return CCDC_ESTATE;
    const int64_t of[] = {b->M, b->N, (int64_t)b->saved_bytes, (int64_t)b->workspace_bytes};
    *static_cast<int64_t *>(out) = of[what];
    return CCDC_OK;
}

}  // extern "C"
