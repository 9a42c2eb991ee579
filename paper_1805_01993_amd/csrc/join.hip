// The join of two blocks (norm, gate, dropout, residual, next norm) with its gradient, and dropout by itself.
#include <algorithm>

#include "element.hpp"

namespace {
using namespace ccdc;

constexpr int kJoinWaves = 4;         // wavefronts of a workgroup where a row has fewer
// Rows that a workgroup of the gradient has at a time.  A row is a chain of four sums over it and three waits for memory, 9 us of them
// at 2048 columns, so a chunk's rows go several abreast: 14336 x 2048 bf16 one at a time 298 us, four 117 (3.0 TB/s); 14348 x 1001 fp32
// four at a time 117 us, eight 86.
constexpr int teams(int waves) { return waves < 8 ? 8 / waves : 1; }

struct JoinArgs {
    const void *x, *f, *w_post, *gate, *w_pre;    // forward; backward: x is dr
    const void *dn, *y_in;
    void *y, *n;                                  // forward; backward: dx, df
    float *sums;                                  // backward: [chunks][2][sum_ld]
    const RowOf *row_of;
    const Chunk *chunks;
    int64_t ld, ld_gate, sum_ld;
    int32_t rows, width;
    float eps, rho;
    Dropout drop;
};

// Sums over the threads of a row: a wavefront's in registers, wavefronts by LDS in their order.  Two halves of the LDS in
// turn, so that one barrier a sum is enough: who writes the first half again has met the others since they read it.
template <int WAVES>
struct RowSums {
    float *part;                                  // [2][2 * WAVES] of the row
    int at = 0;

    template <int COUNT>
    __device__ __forceinline__ void add(float (&v)[COUNT])
    {
#pragma unroll
        for (int c = 0; c < COUNT; c++) v[c] = wave_sum(v[c]);
        if constexpr (WAVES > 1) {
            float *slot = part + at;
            at = 2 * WAVES - at;
            if (fresh(threadIdx.x) % 64 == 0)
#pragma unroll
                for (int c = 0; c < COUNT; c++) slot[threadIdx.x / 64 % WAVES * COUNT + c] = v[c];
            __syncthreads();
#pragma unroll
            for (int c = 0; c < COUNT; c++) v[c] = slot[c];
#pragma unroll
            for (int i = 1; i < WAVES; i++)
#pragma unroll
                for (int c = 0; c < COUNT; c++) v[c] += slot[i * COUNT + c];
        }
    }
    __device__ __forceinline__ float add(float v)
    {
        float one[1] = {v};
        add(one);
        return one[0];
    }
};

// What a thread holds of a row: packs (threadIdx in the row) + i * (threads of the row).
template <int WAVES, int PACKS>
struct Share {
    Eight p[PACKS];
};

template <int WAVES>
__device__ __forceinline__ int pack_of(int i)
{
    return i * (WAVES * 64) + (int)threadIdx.x % (WAVES * 64);
}

// v becomes v hat = (v - mean, where centred) * rstd; returns rstd.  Statistics of the held row: the mean first, then
// the squares of what is left, as the formula says (no difference of large sums).
template <bool CENTRED, int WAVES, int PACKS>
__device__ __forceinline__ float normalise(Share<WAVES, PACKS> &v, int width, float eps, RowSums<WAVES> &sums)
{
    if constexpr (CENTRED) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < PACKS; i++)
#pragma unroll
            for (int e = 0; e < 8; e++) sum += v.p[i].v[e];          // past the row's end: zeros
        const float mean = sums.add(sum) / (float)width;
#pragma unroll
        for (int i = 0; i < PACKS; i++) {
            const int valid = fresh(width - pack_of<WAVES>(i) * 8);
#pragma unroll
            for (int e = 0; e < 8; e++)
                v.p[i].v[e] = __int_as_float(__float_as_int(v.p[i].v[e] - mean) & -inside(valid, e));
        }
    }
    float square = 0.0f;
#pragma unroll
    for (int i = 0; i < PACKS; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) square += v.p[i].v[e] * v.p[i].v[e];
    const float rstd = 1.0f / sqrtf(sums.add(square) / (float)width + eps);
#pragma unroll
    for (int i = 0; i < PACKS; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) v.p[i].v[e] *= rstd;
    return rstd;
}

// e becomes the gradient of v from that of v hat: rstd (e - v hat mean(e v hat) [- mean(e)]).
template <bool CENTRED, int WAVES, int PACKS>
__device__ __forceinline__ void norm_gradient(Share<WAVES, PACKS> &e, const Share<WAVES, PACKS> &hat, float rstd, int width,
                                              RowSums<WAVES> &sums)
{
    float dot = 0.0f, sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PACKS; i++)
#pragma unroll
        for (int k = 0; k < 8; k++) {
            dot += e.p[i].v[k] * hat.p[i].v[k];
            if constexpr (CENTRED) sum += e.p[i].v[k];
        }
    if constexpr (CENTRED) {
        float both[2] = {dot, sum};
        sums.add(both);
        dot = both[0], sum = both[1];
    } else {
        dot = sums.add(dot);
    }
    dot /= (float)width;
    sum /= (float)width;
#pragma unroll
    for (int i = 0; i < PACKS; i++) {
        const int valid = fresh(width - pack_of<WAVES>(i) * 8);
#pragma unroll
        for (int k = 0; k < 8; k++) {
            e.p[i].v[k] = rstd * (e.p[i].v[k] - hat.p[i].v[k] * dot - sum);
            // zeros stay past the row's end, where the next sum over the row takes them
            if constexpr (CENTRED) e.p[i].v[k] = __int_as_float(__float_as_int(e.p[i].v[k]) & -inside(valid, k));
        }
    }
}

// A row as loaded: 16-bit elements are half the registers that they are widened.
template <class T, int WAVES, int PACKS>
struct RawShare {
    Raw8<T> p[PACKS];
};

template <class T, int WAVES, int PACKS>
__device__ __forceinline__ RawShare<T, WAVES, PACKS> load_raw_row(const void *base, int64_t at, int width)
{
    RawShare<T, WAVES, PACKS> s;
#pragma unroll
    for (int i = 0; i < PACKS; i++) {
        const int c = fresh(pack_of<WAVES>(i) * 8);
        if (c < width) s.p[i] = load_raw<T>((const typename T::elem *)base + at + c, width - c);
        else s.p[i] = {};
    }
    return s;
}

template <class T, int WAVES, int PACKS>
__device__ __forceinline__ Share<WAVES, PACKS> widen_row(const RawShare<T, WAVES, PACKS> &raw)
{
    Share<WAVES, PACKS> s;
#pragma unroll
    for (int i = 0; i < PACKS; i++) s.p[i] = widen(raw.p[i]);
    return s;
}

template <class T, int WAVES, int PACKS>
__device__ __forceinline__ Share<WAVES, PACKS> load_row(const void *base, int64_t at, int width)
{
    return widen_row(load_raw_row<T, WAVES, PACKS>(base, at, width));
}

template <class T, int WAVES, int PACKS>
__device__ __forceinline__ void store_row(void *base, int64_t at, int width, const Share<WAVES, PACKS> &s)
{
#pragma unroll
    for (int i = 0; i < PACKS; i++) {
        const int c = fresh(pack_of<WAVES>(i) * 8);
        if (c < width) store_eight<T>((typename T::elem *)base + at + c, s.p[i], width - c);
    }
}

// Multiplies by a vector of the parameters (null: ones).
template <class T, int WAVES, int PACKS>
__device__ __forceinline__ void times(Share<WAVES, PACKS> &v, const void *w, int64_t at, int width)
{
    if (!w) return;
    const Share<WAVES, PACKS> s = load_row<T, WAVES, PACKS>(w, at, width);
#pragma unroll
    for (int i = 0; i < PACKS; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) v.p[i].v[e] *= s.p[i].v[e];
}

template <int WAVES, int PACKS>
__device__ __forceinline__ void drop(Share<WAVES, PACKS> &v, const Dropout &d, const RowOf &row, int width)
{
    if (d.threshold == 0) return;
#pragma unroll
    for (int i = 0; i < PACKS; i++) {
        const int unit = pack_of<WAVES>(i);
        if (unit * 8 >= width) continue;
        drop_eight(v.p[i], d, row.id, row.token, unit);
    }
}

// One row a wavefront (WAVES = 1) or a workgroup: x and f are read once, y and n written once; the row's statistics are
// taken from registers, and n from y before it is rounded.
template <class T, bool CENTRED, int WAVES, int PACKS>
__global__ __launch_bounds__(64 * (WAVES > 1 ? WAVES : kJoinWaves)) void k_join(const JoinArgs a)
{
    __shared__ float part[WAVES > 1 ? 4 * WAVES : 1];
    RowSums<WAVES> sums{part};
    const int row = WAVES > 1 ? (int)blockIdx.x : (int)(blockIdx.x * kJoinWaves + threadIdx.x / 64);
    if (row >= a.rows) return;
    const int64_t at = row * a.ld;
    Share<WAVES, PACKS> y = load_row<T, WAVES, PACKS>(a.x, at, a.width);
    if (a.f) {
        Share<WAVES, PACKS> z = load_row<T, WAVES, PACKS>(a.f, at, a.width);
        const RowOf of = a.row_of[row];
        normalise<CENTRED>(z, a.width, a.eps, sums);
        times<T>(z, a.w_post, 0, a.width);
        times<T>(z, a.gate, of.file * a.ld_gate, a.width);
        drop(z, a.drop, of, a.width);
#pragma unroll
        for (int i = 0; i < PACKS; i++)
#pragma unroll
            for (int e = 0; e < 8; e++) y.p[i].v[e] = a.rho * y.p[i].v[e] + z.p[i].v[e];
    } else {
#pragma unroll
        for (int i = 0; i < PACKS; i++)
#pragma unroll
            for (int e = 0; e < 8; e++) y.p[i].v[e] *= a.rho;
    }
    if (a.y) store_row<T>(a.y, at, a.width, y);
    if (a.n) {
        normalise<CENTRED>(y, a.width, a.eps, sums);
        times<T>(y, a.w_pre, 0, a.width);
        store_row<T>(a.n, at, a.width, y);
    }
}

// The gradients of a chunk of one file's rows.  The gate and the norms' weights are one for a file's rows, so two sums over them make
// all three gradients: with S = sum D(dy) fhat, dw_post = gate S and dgate = w_post S; dw_pre = sum dn yhat.  A thread keeps its
// columns' sums over the chunk's rows in registers; k_learned adds the chunks.
template <class T, bool CENTRED, int WAVES, int PACKS>
__global__ __launch_bounds__(64 * WAVES * teams(WAVES)) void k_join_gradient(const JoinArgs a)
{
    using E = typename T::elem;
    constexpr int TEAMS = teams(WAVES), ROW = 64 * WAVES;     // rows at a time, threads of a row
    __shared__ float part[TEAMS][WAVES > 1 ? 4 * WAVES : 1];
    __shared__ float add[TEAMS > 1 ? TEAMS * ROW * 8 : 1];
    const Chunk chunk = a.chunks[blockIdx.x];
    const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / ROW);
    RowSums<WAVES> sums{part[team]};
    // a workgroup of sixteen wavefronts has 128 registers a lane: its sums are in LDS, each lane's its own
    constexpr bool in_lds = WAVES == 16;
    __shared__ float lds_sum[in_lds ? 2 * PACKS * 8 * 64 * WAVES : 1];
    Share<WAVES, in_lds ? 1 : PACKS> sum[2] = {};
    const auto sum_at = [&](int s, int i, int k) -> float & {
        if constexpr (in_lds) return lds_sum[((s * PACKS + i) * 8 + k) * (64 * WAVES) + threadIdx.x];
        else return sum[s].p[i].v[k];
    };
    if constexpr (in_lds)
        for (int i = 0; i < 2 * PACKS * 8; i++) lds_sum[i * (64 * WAVES) + threadIdx.x] = 0.0f;
    const auto *args = (const __attribute__((address_space(4))) JoinArgs *)__builtin_amdgcn_kernarg_segment_ptr();
    for (int r = team; r - team < chunk.rows; r += TEAMS) {
        const bool own = r < chunk.rows;          // else with the others to the barriers, on the last row
        // The arguments, and the parameters that they point to, are asked for again in every row: kept over the rows they are more
        // scalar registers than there are, and the vector registers of other wavefronts.
        const auto &a = *fresh_uniform(args);
        const int width = a.width;
        const int64_t row = chunk.first + (own ? r : chunk.rows - 1), at = row * a.ld;
        // 16-bit rows are all asked for at once; those of fp32 would be the registers of half the wavefronts
        constexpr bool early = sizeof(E) == 2;
        RawShare<T, WAVES, PACKS> raw_dr, raw_f;
        if (early && a.x) raw_dr = load_raw_row<T, WAVES, PACKS>(a.x, at, width);
        if (early && a.f) raw_f = load_raw_row<T, WAVES, PACKS>(a.f, at, width);
        Share<WAVES, PACKS> dy = {};
        if (a.dn) {
            dy = load_row<T, WAVES, PACKS>(a.dn, at, width);
            Share<WAVES, PACKS> hat = load_row<T, WAVES, PACKS>(a.y_in, at, width);
            const float rstd = normalise<CENTRED>(hat, width, a.eps, sums);
            if (own)
#pragma unroll
                for (int i = 0; i < PACKS; i++)
#pragma unroll
                    for (int k = 0; k < 8; k++) sum_at(1, i, k) += dy.p[i].v[k] * hat.p[i].v[k];
            times<T>(dy, a.w_pre, 0, width);
            norm_gradient<CENTRED>(dy, hat, rstd, width, sums);
        }
        if (a.x) {
            const Share<WAVES, PACKS> dr = early ? widen_row(raw_dr) : load_row<T, WAVES, PACKS>(a.x, at, width);
#pragma unroll
            for (int i = 0; i < PACKS; i++)
#pragma unroll
                for (int k = 0; k < 8; k++) dy.p[i].v[k] += dr.p[i].v[k];
        }
        if (a.y && own) {
#pragma unroll
            for (int i = 0; i < PACKS; i++) {
                const int c = fresh(pack_of<WAVES>(i) * 8);
                if (c >= width) continue;
                Eight dx;
#pragma unroll
                for (int k = 0; k < 8; k++) dx.v[k] = a.rho * dy.p[i].v[k];
                store_eight<T>((E *)a.y + at + c, dx, width - c);
            }
        }
        if (a.f) {
            Share<WAVES, PACKS> hat = early ? widen_row(raw_f) : load_row<T, WAVES, PACKS>(a.f, at, width);
            const RowOf of = a.row_of[row];
            const Dropout drop{{a.drop.key[0], a.drop.key[1]}, a.drop.site, a.drop.threshold, a.drop.scale};
            const float rstd = normalise<CENTRED>(hat, width, a.eps, sums);
#pragma unroll
            for (int i = 0; i < PACKS; i++) {
                const int unit = fresh(pack_of<WAVES>(i));
                if (drop.threshold && unit * 8 < width) drop_eight(dy.p[i], drop, of.id, of.token, unit);
                if (own)
#pragma unroll
                    for (int k = 0; k < 8; k++) sum_at(0, i, k) += dy.p[i].v[k] * hat.p[i].v[k];
            }
            times<T>(dy, a.w_post, 0, width);
            times<T>(dy, a.gate, of.file * a.ld_gate, width);
            norm_gradient<CENTRED>(dy, hat, rstd, width, sums);
            if (a.n && own) store_row<T>(a.n, at, width, dy);
        }
    }
    if (!a.sums) return;
    float *to = a.sums + (int64_t)blockIdx.x * 2 * a.sum_ld;
#pragma unroll
    for (int s = 0; s < 2; s++)
#pragma unroll
        for (int i = 0; i < PACKS; i++) {
            const int c = fresh(pack_of<WAVES>(i) * 8);
            Eight v;
#pragma unroll
            for (int k = 0; k < 8; k++) v.v[k] = sum_at(s, i, k);
            if constexpr (TEAMS > 1) {            // all teams have the same columns: added in their order
                const int in_row = threadIdx.x % ROW;
#pragma unroll
                for (int k = 0; k < 8; k++) add[(team * 8 + k) * ROW + in_row] = v.v[k];
                __syncthreads();
                if (team == 0) {
#pragma unroll
                    for (int k = 0; k < 8; k++)
                        for (int o = 1; o < TEAMS; o++) v.v[k] += add[(o * 8 + k) * ROW + in_row];
                }
                __syncthreads();
                if (team > 0) continue;
            }
            if (c >= a.width) continue;           // (rows of sums are whole packs)
#pragma unroll
            for (int k = 0; k < 8; k++) to[s * a.sum_ld + c + k] = v.v[k];
        }
}

struct LearnedArgs {
    const float *sums;
    void *w_post, *gate, *w_pre;                  // gradients; null: not wanted
    const void *by_gate, *by_post;                // what the sum is multiplied by for the first two; null: ones
    const int32_t *chunk_first;
    int64_t sum_ld, ld_file, ld_gate;
    int32_t width;
};

// The chunks of a file are added in their order, from four beginnings so that four are asked for together; a file without
// rows has none and gets zeros.
template <class T>
__global__ __launch_bounds__(kBlock) void k_learned(const LearnedArgs a)
{
    const int c = (int)(blockIdx.x * kBlock + threadIdx.x), file = (int)blockIdx.y, which = (int)blockIdx.z;
    using E = typename T::elem;
    if (c >= a.width || (which == 0 ? !a.w_post && !a.gate : !a.w_pre)) return;
    const int from = a.chunk_first[file], end = a.chunk_first[file + 1];
    const float *p = a.sums + which * a.sum_ld + c;
    const int64_t step = 2 * a.sum_ld, at = file * a.ld_file + c;
    float v[4] = {};
    int k = from;
    for (; k + 4 <= end; k += 4)
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] += p[(k + i) * step];
    for (; k < end; k++) v[0] += p[k * step];
    const float sum = (v[0] + v[1]) + (v[2] + v[3]);
    if (which == 1) {
        ((E *)a.w_pre)[at] = narrow<T>(sum);
        return;
    }
    if (a.w_post) ((E *)a.w_post)[at] = narrow<T>(a.by_gate ? sum * T::widen(((const E *)a.by_gate)[file * a.ld_gate + c]) : sum);
    if (a.gate) ((E *)a.gate)[at] = narrow<T>(a.by_post ? sum * T::widen(((const E *)a.by_post)[c]) : sum);
}

struct DropoutArgs {
    const void *x, *residual;
    void *y;
    const RowOf *row_of;
    int64_t ldx, ld_residual, ldy, columns;
    uint32_t items, units;                        // packs in all, and of a row
    uint32_t factor, shift;                       // pack / units = pack * factor >> shift
    Dropout drop;
};

// A work item makes eight columns of a row; the rows' packs follow one another without a gap (4160 columns are 520 packs, and
// workgroups that begin with a row left a third of their lanes without any).
template <class T>
__global__ __launch_bounds__(kBlock) void k_dropout(const DropoutArgs a)
{
    using E = typename T::elem;
    const uint32_t p = blockIdx.x * kBlock + threadIdx.x;
    if (p >= a.items) return;
    const uint32_t row = (uint32_t)((uint64_t)p * a.factor >> a.shift), unit = p - row * a.units;
    const int64_t c = (int64_t)unit * 8, left = a.columns - c;
    const int valid = left < 8 ? (int)left : 8;
    Eight v = load_eight<T>((const E *)a.x + (int64_t)row * a.ldx + c, valid), res = {};
    if (a.residual) res = load_eight<T>((const E *)a.residual + (int64_t)row * a.ld_residual + c, valid);
    const RowOf of = a.row_of[row];
    drop_eight(v, a.drop, of.id, of.token, unit);
    if (a.residual)
#pragma unroll
        for (int i = 0; i < 8; i++) v.v[i] += res.v[i];
    store_eight<T>((E *)a.y + (int64_t)row * a.ldy + c, v, valid);
}

// Wavefronts and packs of a lane that hold a row.  With four packs a lane one wavefront has 2048 columns and meets no other, but the
// registers leave half as many rows on their way: 14336 x 2048 bf16 forward 71 us, with two wavefronts of two packs 58 (4.1 TB/s).
template <class F>
void by_width(int64_t width, F launch)
{
    const int64_t packs = (width + 7) / 8;
    if (packs <= 64) launch(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
    else if (packs <= 128) launch(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
    else if (packs <= 256) launch(std::integral_constant<int, 2>(), std::integral_constant<int, 2>());
    else if (packs <= 512) launch(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
    else if (packs <= 1024) launch(std::integral_constant<int, 8>(), std::integral_constant<int, 2>());
    else launch(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
}

inline int row_threads(int64_t width) { return width <= 1024 ? 64 : width <= 2048 ? 128 : width <= 4096 ? 256 : width <= 8192 ? 512 : 1024; }

template <class T, bool CENTRED>
int run_join(const JoinArgs &a, hipStream_t st)
{
    by_width(a.width, [&](auto waves, auto packs) {
        constexpr int W = decltype(waves)::value, P = decltype(packs)::value;
        k_join<T, CENTRED, W, P><<<W > 1 ? a.rows : cdiv(a.rows, kJoinWaves), 64 * (W > 1 ? W : kJoinWaves), 0, st>>>(a);
    });
    return launched();
}

template <class T, bool CENTRED>
int run_gradient(const ccdc_block_t *b, const JoinArgs &a, const LearnedArgs &l, hipStream_t st)
{
    if (!b->chunks.empty()) {
        by_width(a.width, [&](auto waves, auto packs) {
            constexpr int W = decltype(waves)::value, P = decltype(packs)::value;
            k_join_gradient<T, CENTRED, W, P><<<(uint32_t)b->chunks.size(), 64 * W * teams(W), 0, st>>>(a);
        });
        const int rc = launched();
        if (rc != CCDC_OK) return rc;
    }
    if (!a.sums) return CCDC_OK;
    for (int from = 0; from < b->N; from += 65535) {        // files a launch can number
        LearnedArgs part = l;
        const auto move = [&](auto *p, int64_t ld) { return p ? (decltype(p))((typename T::elem *)p + from * ld) : p; };
        part.chunk_first += from;
        part.w_post = move(l.w_post, l.ld_file), part.gate = move(l.gate, l.ld_file), part.w_pre = move(l.w_pre, l.ld_file);
        part.by_gate = move(l.by_gate, l.ld_gate);
        k_learned<T><<<dim3(cdiv(a.width, kBlock), std::min(b->N - from, 65535), 2), kBlock, 0, st>>>(part);
    }
    return launched();
}

template <class T>
int run_dropout(const DropoutArgs &a, hipStream_t st)
{
    k_dropout<T><<<cdiv(a.items, kBlock), kBlock, 0, st>>>(a);
    return launched();
}

}  // namespace

extern "C" {

int ccdc_join_forward(const ccdc_block_t *b, int64_t rows, const void *x, const void *f, const void *w_post, const void *gate,
                      int64_t ld_gate, const void *w_pre, void *y, void *n, int64_t ld, uint64_t seed, void *stream)
{
    const int rc = ready(b);
    if (rc != CCDC_OK) return rc;
    if (rows < 0 || rows > b->M || ld < b->c.width || (ld_gate != 0 && ld_gate < b->c.width)) return CCDC_EINVAL;
    if (rows == 0) return CCDC_OK;
    if (!y && !n) return CCDC_EINVAL;
    if (!fits(b, x) || !fits(b, f, true) || !fits(b, w_post, true) || !fits(b, gate, true) || !fits(b, w_pre, true) ||
        !fits(b, y, true) || !fits(b, n, true))
        return CCDC_EINVAL;
    if (b->c.width > kJoinWidth || !fits_launch((uint64_t)rows * row_threads(b->c.width))) return CCDC_ESIZE;
    JoinArgs a{};
    a.x = x, a.f = f, a.w_post = w_post, a.gate = gate, a.w_pre = w_pre, a.y = y, a.n = n;
    a.row_of = b->d_row_of;
    a.ld = ld, a.ld_gate = ld_gate, a.rows = (int32_t)rows, a.width = (int32_t)b->c.width;
    a.eps = b->c.eps, a.rho = b->c.residual_scale;
    a.drop = make_dropout(b->c.dropout_out, 2 * b->c.layer + 1, seed);
    if (b->c.norm == CCDC_NORM_CENTRED) CCDC_BY_ELEM(b, (run_join<T, true>(a, (hipStream_t)stream)));
    CCDC_BY_ELEM(b, (run_join<T, false>(a, (hipStream_t)stream)));
}

int ccdc_join_backward(const ccdc_block_t *b, const void *dn, const void *dr, const void *y, const void *f, const void *w_post,
                       const void *gate, int64_t ld_gate, const void *w_pre, void *dx, void *df, int64_t ld, void *dw_post,
                       void *dgate, void *dw_pre, int64_t ld_file, uint64_t seed, void *stream)
{
    const int rc = ready(b);
    if (rc != CCDC_OK) return rc;
    const bool learned = dw_post || dgate || dw_pre;
    // (a batch without tokens has no rows to point at; its gradients are zeros)
    if (b->M > 0 && ((!dn && !dr) || (dn && !y) || (!f && (df || dw_post || dgate)) || (!dn && dw_pre))) return CCDC_EINVAL;
    if (ld < b->c.width || (ld_gate != 0 && ld_gate < b->c.width) || (learned && b->N > 1 && ld_file < b->c.width)) return CCDC_EINVAL;
    for (const void *p : {dn, dr, y, f, w_post, gate, w_pre, (const void *)dx, (const void *)df, (const void *)dw_post,
                          (const void *)dgate, (const void *)dw_pre})
        if (!fits(b, p, true)) return CCDC_EINVAL;
    if (b->c.width > kJoinWidth || !fits_launch((uint64_t)b->chunks.size() * std::max(row_threads(b->c.width), 512)))
        return CCDC_ESIZE;
    JoinArgs a{};
    a.x = dr, a.dn = dn, a.y_in = y, a.f = f, a.w_post = w_post, a.gate = gate, a.w_pre = w_pre, a.y = dx, a.n = df;
    a.sums = learned ? (float *)b->d_workspace : nullptr;
    a.row_of = b->d_row_of, a.chunks = b->d_chunks;
    a.ld = ld, a.ld_gate = ld_gate, a.sum_ld = b->width_ld, a.width = (int32_t)b->c.width;
    a.eps = b->c.eps, a.rho = b->c.residual_scale;
    a.drop = make_dropout(b->c.dropout_out, 2 * b->c.layer + 1, seed);
    LearnedArgs l{a.sums, dw_post, dgate, dw_pre, gate, w_post, b->d_chunk_first, b->width_ld, ld_file, ld_gate, a.width};
    hipStream_t st = (hipStream_t)stream;
    WorkspaceOrder order(b, st, learned);
    if (b->c.norm == CCDC_NORM_CENTRED) CCDC_BY_ELEM(b, (run_gradient<T, true>(b, a, l, st)));
    CCDC_BY_ELEM(b, (run_gradient<T, false>(b, a, l, st)));
}

int ccdc_dropout(const ccdc_block_t *b, int64_t rows, int64_t columns, double p, uint32_t site, uint64_t seed, const void *x,
                 int64_t ldx, const void *residual, int64_t ld_residual, void *y, int64_t ldy, void *stream)
{
    const int rc = ready(b);
    if (rc != CCDC_OK) return rc;
    if (rows < 0 || rows > b->M || columns < 1 || !(p >= 0.0 && p <= 1.0)) return CCDC_EINVAL;
    if (ldx < columns || ldy < columns || (residual && ld_residual < columns)) return CCDC_EINVAL;
    if (rows == 0) return CCDC_OK;
    if (!fits(b, x) || !fits(b, y) || !fits(b, residual, true)) return CCDC_EINVAL;
    const uint64_t units = ((uint64_t)columns + 7) / 8;
    if (units > kMaxLaunchItems || !fits_launch(cdiv((uint64_t)rows * units, kBlock) * (uint64_t)kBlock)) return CCDC_ESIZE;
    // exact for numbers below 2^31: with 2^bits >= units the factor is at most units - 1 too large times 2^-(31 + bits) of them
    uint32_t bits = 0;
    while (((uint64_t)1 << bits) < units) bits++;
    const uint64_t factor = (((uint64_t)1 << (31 + bits)) + units - 1) / units;
    const DropoutArgs a{x, residual, y, b->d_row_of, ldx, ld_residual, ldy, columns, (uint32_t)((uint64_t)rows * units), (uint32_t)units,
                        (uint32_t)factor, 31 + bits, make_dropout(p, site, seed)};
    CCDC_BY_ELEM(b, (run_dropout<T>(a, (hipStream_t)stream)));
}

}  // extern "C"
