// The distance of a student's logits from a teacher's top logits, and its gradient: one pass over the row.
//
// With S the listed columns and e_v = exp((z_v - m) / T), m the largest logit outside S and s the sum of e_v there, all that a row of others
// needs is one number: dz_v = w C e_v with C = exp(m / T - lse) - p_rest / s, lse over the whole row.  So the others' sums are
// their own (a difference of the whole row's and the list's would lose them where the list has nearly everything), and the
// list's k columns are one wavefront's, two a lane.  A bit a column in LDS says which are listed.
//
// The row is held in registers as loaded between the sums and the gradient: read once, written once.
#include "vocabulary.hpp"

namespace {
using namespace ccdc;

struct DistillArgs {
    const void *z;
    const int32_t *index;
    const float *value, *rest, *weight;
    float *loss;
    void *dz;
    int64_t ldz, lddz;
    int32_t columns, k, mask_bytes;
    float per_T, scale;                           // 1 / T
};

constexpr float kLog2e = 1.44269504f;

// What the list's wavefront tells the others.
struct Listed {
    float most, sum;                              // of the listed logits: the largest, sum of exp((z - most) / T)
    float p_rest;
    int count;                                    // entries; 0 too where they and the rest are all -infinity
};

// exp(x) = 2^(x log2 e): rounding the product is off by half a step of it, |x| 2^-24 of the result.
__device__ __forceinline__ float exponential(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

template <class T, int WAVES, int PACKS, int LDS, bool REST>
__global__ __launch_bounds__(64 * WAVES, LDS > 0 ? 8 : 0) void k_distill(const DistillArgs a)
{
    using E = typename T::elem;
    constexpr int THREADS = 64 * WAVES;
    constexpr bool kept = !REST && T::planes == 3;        // fp32: the exponentials take the logits' registers
    extern __shared__ __attribute__((aligned(16))) uint32_t mask[];       // a bit a column, lowest first; then packs of the row
    __shared__ double part[2 * WAVES];
    __shared__ int32_t listed[kMostListed];
    __shared__ Listed shared;
    OverRow<WAVES> over{part};
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x % 64;
    const bool lists = threadIdx.x < 64;          // the list's wavefront
    const float factor = a.weight ? a.weight[row] * a.scale : a.scale;
    const bool counts = !(a.weight && a.weight[row] == 0.0f);
    if (WAVES > 1 || PACKS > 1) __builtin_assume(a.columns >= 8);     // (by_columns; shorter rows' loads are many registers)
    Row<T, WAVES, PACKS, LDS, REST> z;
    z.room = reinterpret_cast<Bytes16 *>(mask + a.mask_bytes / 4) + threadIdx.x;
    if (counts) z.load(a.z, row * a.ldz, a.columns);
    for (int i = threadIdx.x; i < a.mask_bytes / 4; i += THREADS) mask[i] = 0;

    int32_t column[2] = {-1, -1};
    float p[2] = {}, log_p[2] = {}, logit[2] = {-INFINITY, -INFINITY};
    if (lists) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int j = lane + 64 * h;
            if (j < a.k) column[h] = a.index[row * a.k + j];
            if ((uint32_t)column[h] >= (uint32_t)a.columns) column[h] = -1;
            listed[j] = column[h];
        }
    }
    __syncthreads();
    if (lists) {
        // an entry whose column was listed before is none
        bool again = false;
#pragma unroll
        for (int h = 0; h < 2; h++)
            if (column[h] >= 0) again |= atomicOr(&mask[column[h] / 32], 1u << (column[h] % 32)) >> (column[h] % 32) & 1;
        if (__any(again))
            for (int i = 0; i < a.k; i++) {
                const int32_t other = listed[i];
#pragma unroll
                for (int h = 0; h < 2; h++)
                    if (i < lane + 64 * h && other == column[h]) column[h] = -1;
            }
        float t[2] = {-INFINITY, -INFINITY}, most = -INFINITY, count = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; h++)
            if (column[h] >= 0) {
                t[h] = a.value[row * a.k + lane + 64 * h];
                logit[h] = T::widen(((const E *)a.z)[row * a.ldz + column[h]]);
                count += 1.0f;
                most = fmaxf(most, logit[h]);
            }
        // the teacher's p over the list and the rest, all as distances from its largest value there: these by 1 / T round to what counts, where
        // values far from zero would first (10000 / 0.7: p off by 5e-4), or pass fp32's range
        const float value = wave_most(fmaxf(t[0], t[1])), largest = fmaxf(value, kLowest);
#pragma unroll
        for (int h = 0; h < 2; h++) t[h] = (t[h] - largest) * a.per_T;
        float rest = a.rest ? a.rest[row] : -INFINITY;
        if (fabsf(rest) < INFINITY) rest = fminf(fmaf(-largest, a.per_T, rest), -kLowest);
        const float top = fmaxf(fmaxf(value > -INFINITY ? 0.0f : -INFINITY, rest), kLowest);
        float sum = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; h++) sum += exponential(t[h] - top);
        const float of_rest = exponential(rest - top), total = wave_sum(sum) + of_rest, log_total = logf(total);
#pragma unroll
        for (int h = 0; h < 2; h++) p[h] = exponential(t[h] - top) / total, log_p[h] = t[h] - top - log_total;
        most = wave_most(most);
        float own = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; h++)
            if (column[h] >= 0) own += exponential((logit[h] - fmaxf(most, kLowest)) * a.per_T);
        own = wave_sum(own);
        count = wave_sum(count);
        if (lane == 0) shared = {most, own, of_rest / total, total == 0.0f ? 0 : (int)count};
    }
    __syncthreads();
    const Listed list = shared;
    if (!counts || list.count == 0) {             // (the same for all threads)
        if (a.loss && threadIdx.x == 0) a.loss[row] = 0.0f;
        if (a.dz)
            for (int32_t c = (int32_t)threadIdx.x * 8; c < a.columns; c += THREADS * 8) store_eight<T>((E *)a.dz + row * a.lddz + c, Eight{}, a.columns - c);
        return;
    }

    const auto listed_of = [&](int32_t c) { return (uint32_t)((((uint64_t)mask[c / 32 + 1] << 32) | mask[c / 32]) >> (c % 32)) & 0xFFu; };
    const float scale = a.per_T * kLog2e;
    float m = -INFINITY, s = 0.0f;
    if constexpr (!REST) {
        z.template hide_held<false>(listed_of, [&](const Eight &v) {
#pragma unroll
            for (int i = 0; i < 8; i++) m = fmaxf(m, v.v[i]);
        });
        m = over.most(m);
    } else {
        // the largest so far and the sum from it on
        float from = kLowest;
        const auto arrives = [&](const Eight &v) {
            float next = m;
#pragma unroll
            for (int i = 0; i < 8; i++) next = fmaxf(next, v.v[i]);
            if (next > m) {
                s *= __builtin_amdgcn_exp2f((m - next) * scale);
                m = from = next;
            }
#pragma unroll
            for (int i = 0; i < 8; i++) s += __builtin_amdgcn_exp2f((v.v[i] - from) * scale);
        };
        z.template hide_held<false>(listed_of, arrives);
        z.rest(listed_of, [&](const Eight &v, int32_t, uint32_t) { arrives(v); });
        const float own = m;
        m = over.most(m);
        s = over.sum(s * __builtin_amdgcn_exp2f((own - fmaxf(m, kLowest)) * scale));
    }
    const Powers powers(scale, fmaxf(m, kLowest));
    const bool far = REST || kept || powers.far();        // (the same for all threads)
    if constexpr (!REST) {
        PackSum sum;
        const auto add = [&](const Eight &e) {
            sum.add(((e.v[0] + e.v[1]) + (e.v[2] + e.v[3])) + ((e.v[4] + e.v[5]) + (e.v[6] + e.v[7])));
        };
        const auto sums = [&](auto &row, auto term) {
            row.each(listed_of, [&](const Eight &v, int32_t, uint32_t) {
                Eight e;
#pragma unroll
                for (int i = 0; i < 8; i++) e.v[i] = term(v.v[i]);
                add(e);
            });
        };
        if constexpr (kept) {
#pragma unroll
            for (int i = 0; i < PACKS; i++) {
                if (!z.some(i)) continue;
                Eight e;
#pragma unroll
                for (int k = 0; k < 8; k++) {
                    e.v[k] = powers.difference(__uint_as_float(z.held[i][k]));
                    z.held[i][k] = __float_as_uint(e.v[k]);
                }
                add(e);
            }
        } else if (far) {                         // few rows: read again
            auto again = z.again();
            sums(again, [&](float v) { return powers.difference(v); });
        } else {
            sums(z, [&](float v) { return powers(v); });
        }
        s = over.sum(sum) * (far ? 1.0f : powers.lost());
    }

    // all relative to the row's largest logit
    const float from = fmaxf(m, kLowest), top = fmaxf(fmaxf(m, list.most), kLowest);
    const float others = (from - top) * a.per_T, others_exp = m > -INFINITY ? exponential(others) : 0.0f;
    const float listed_exp = list.most > -INFINITY ? exponential((list.most - top) * a.per_T) : 0.0f;
    const float total = s * others_exp + list.sum * listed_exp, lse = logf(total);
    if (total == 0.0f) {                          // no logit above -infinity: nothing to learn
        if (a.loss && threadIdx.x == 0) a.loss[row] = 0.0f;
        if (a.dz)
            for (int32_t c = (int32_t)threadIdx.x * 8; c < a.columns; c += THREADS * 8) store_eight<T>((E *)a.dz + row * a.lddz + c, Eight{}, a.columns - c);
        return;
    }
    float gradient[2];
    if (lists) {
        float loss = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const float log_q = (logit[h] - top) * a.per_T - lse;
            if (column[h] >= 0 && !(p[h] == 0.0f)) loss += p[h] * (log_p[h] - log_q);
            gradient[h] = factor * a.per_T * (exponential(log_q) - p[h]);
        }
        loss = wave_sum(loss);
        if (lane == 0 && a.loss) {
            if (!(list.p_rest == 0.0f)) loss += list.p_rest * (logf(list.p_rest) - (others + logf(s) - lse));
            a.loss[row] = factor * loss;
        }
    }
    if (!a.dz) return;
    const float of_rest = list.p_rest == 0.0f || s == 0.0f ? 0.0f : list.p_rest / s;
    const float C = factor * a.per_T * (others_exp / total - of_rest) * (far ? 1.0f : powers.lost());
    E *dz = (E *)a.dz + row * a.lddz;
    const auto made = [&](auto &row, auto term) {
        row.each(listed_of, [&](const Eight &v, int32_t c, uint32_t valid) {
            if (!valid) return;
            Eight d;
#pragma unroll
            for (int i = 0; i < 8; i++) d.v[i] = C * term(v.v[i]);
            row.store(dz + c, d, valid);
        });
    };
    if constexpr (REST) {
        made(z, [&](float v) { return powers.difference(v); });
    } else if constexpr (kept) {
        made(z, [](float v) { return v; });
    } else if (far) {
        auto again = z.again();
        made(again, [&](float v) { return powers.difference(v); });
    } else {
        made(z, [&](float v) { return powers(v); });
    }
    __syncthreads();                              // the list's columns are written over
    if (lists)
#pragma unroll
        for (int h = 0; h < 2; h++)
            if (column[h] >= 0) dz[column[h]] = narrow<T>(gradient[h]);
}

// Of rows with more packs none is held: their bits and packs in LDS would leave a compute unit no second workgroup, and from 900000
// columns on not one (16 bits, dz too: 600 x 300000 212 us held, 232 not; 300 x 600000 260 and 253).
constexpr int64_t kMostHeld = 65536;

// launch(wavefronts of a row, packs that a lane holds of it in registers, in LDS, whether the row may be longer).
// Many rows go by wavefronts of few packs and many of them a compute unit, a few rows by as many as shorten their way (us, bf16: 16384 x 2000
// by 2 wavefronts of 2 packs 39.5, by 4 of 2 55, 128 rows 4.5 and 4.3; 16384 x 4000 by 2 of 4 62, by 4 of 2 70, 128 rows 5.1 and 4.5; 7812 x
// 32000 by 8 of 8 210, by 16 of 4 221, not held 241, 128 rows 11.5 and 10.3).
template <class T, class F>
int by_columns(int64_t columns, int64_t rows, F launch)
{
    const auto go = [&](auto waves, auto packs) { return launch(waves, packs, std::integral_constant<int, 0>(), std::false_type()); };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 4> four;
    const std::integral_constant<int, 8> eight;
    const std::integral_constant<int, 16> sixteen;
    const int64_t packs = (columns + 7) / 8;
    const bool few = rows <= 256;
    if (packs <= 64) return go(one, one);
    if (packs <= 128) return go(one, two);
    if (packs <= 256 && !few) return go(two, two);
    if (packs <= 512) return few ? go(four, two) : go(two, four);
    if (packs <= 1024) return go(four, four);
    if (packs <= 2048) return go(eight, four);
    if (packs <= 4096) return few ? go(sixteen, four) : go(eight, eight);
    if constexpr (T::planes == 1) {
        if (packs <= 8192) return launch(sixteen, four, four, std::false_type());
        if (packs <= kMostHeld) return launch(sixteen, four, std::integral_constant<int, 3>(), std::true_type());
    } else {
        if (packs <= 8192) return go(sixteen, eight);
    }
    return launch(sixteen, std::integral_constant<int, 0>(), std::integral_constant<int, 0>(), std::true_type());
}

template <class T>
int run_distill(const DistillArgs &a, int64_t rows, hipStream_t st)
{
    return by_columns<T>(a.columns, rows, [&](auto waves, auto packs, auto lds, auto rest) -> int {
        constexpr int W = decltype(waves)::value, P = decltype(packs)::value, L = decltype(lds)::value;
        if (!fits_launch((uint64_t)rows * 64 * W)) return CCDC_ESIZE;
        k_distill<T, W, P, L, decltype(rest)::value><<<(uint32_t)rows, 64 * W, a.mask_bytes + L * 64 * W * 16, st>>>(a);
        return launched();
    });
}

}  // namespace

extern "C" {

int ccdc_distill(const ccdc_block_t *b, int64_t rows, int64_t columns, const void *z, int64_t ldz, int k, const int32_t *index,
                 const float *value, const float *rest, double temperature, const float *weight, double scale, float *loss, void *dz,
                 int64_t lddz, void *stream)
{
    const int rc = ready(b);
    if (rc != CCDC_OK) return rc;
    if (rows < 0 || columns < 1 || ldz < columns || k < 1 || k > kMostListed || (dz && lddz < columns)) return CCDC_EINVAL;
    const float heat = (float)temperature, per_T = 1.0f / heat;
    if (!(heat > 0.0f) || !std::isfinite(heat) || !std::isfinite(per_T * kLog2e) || !std::isfinite((float)scale)) return CCDC_EINVAL;
    if (rows == 0) return CCDC_OK;
    if (!loss && !dz) return CCDC_EINVAL;
    if (!fits(b, z) || !fits(b, dz, true) || !index || !value || (dz && dz == z && lddz != ldz)) return CCDC_EINVAL;
    for (const void *p : {(const void *)index, (const void *)value, (const void *)rest, (const void *)weight, (const void *)loss})
        if (!aligned(p, 4)) return CCDC_EINVAL;
    if (columns > kMostColumns) return CCDC_ESIZE;
    const DistillArgs a{z, index, value, rest, weight, loss, dz, ldz, lddz, (int32_t)columns, k, (int32_t)((columns / 32 + 2 + 3) / 4 * 16), per_T,
                        (float)scale};
    CCDC_BY_ELEM(b, (run_distill<T>(a, rows, (hipStream_t)stream)));
}

}  // extern "C"
