// Runs the calls that learn from a teacher, compiled for the host against teacher_lanes.hpp, on small shapes under AddressSanitizer /
// UBSan, and checks what they give against the formulas of ccdc.h in 64 bits.  Every matrix is a heap block of exactly its size,
// what lies between its rows is poisoned; results begin as what no result is.  Test infrastructure only.
// Usage: teacher_driver quantise MODE ROWS COLUMNS PAD
//        teacher_driver product MODE ROWS WIDE OUTPUTS PAD TILE       (TILE: shim::force)
//        teacher_driver scales MODE ROWS WIDE OUTPUTS PAD TILE        (scales next to their ends)
//        teacher_driver top MODE ROWS COLUMNS K PAD KIND              (KIND 0 noise, 1 all equal, 2 masked but for few,
//                                                                      10 ... all but the last K that many T below them,
//                                                                      -10 ... one of these, the others 5 T further down)
//        teacher_driver distill MODE ROWS COLUMNS K PAD PLACE         (PLACE 1: dz is z)
#include <sanitizer/asan_interface.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>

#include "teacher_lanes.hpp"
#include "ccdc.h"

namespace {
int mode;
size_t elem() { return mode == CCDC_BF16_SUM_XOR || mode == CCDC_F16_SUM_XOR ? 2 : 4; }
double half_step() { return mode == CCDC_BF16_SUM_XOR ? 0x1p-8 : mode == CCDC_F16_SUM_XOR ? 0x1p-11 : 0x1p-24; }

uint64_t state = 88172645463325252ull;
double uniform()                                      // in (-1, 1)
{
    state ^= state << 13, state ^= state >> 7, state ^= state << 17;
    return (double)(state >> 11) / 4503599627370496.0 - 1.0;
}
void put(void *p, double v)
{
    const float f = (float)v;
    if (mode == CCDC_BF16_SUM_XOR) {
        const uint32_t u = __float_as_uint(f);
        const uint16_t h = (uint16_t)((u + 0x7FFF + (u >> 16 & 1)) >> 16);
        std::memcpy(p, &h, 2);
    } else if (mode == CCDC_F16_SUM_XOR) {
        const _Float16 h = (_Float16)f;
        std::memcpy(p, &h, 2);
    } else {
        std::memcpy(p, &f, 4);
    }
}
double get(const void *p)
{
    if (elem() == 4) {
        float f;
        std::memcpy(&f, p, 4);
        return f;
    }
    uint16_t h;
    std::memcpy(&h, p, 2);
    if (mode == CCDC_BF16_SUM_XOR) return __uint_as_float((uint32_t)h << 16);
    _Float16 f;
    std::memcpy(&f, &h, 2);
    return (double)f;
}

// Rows of `columns` elements of `size` bytes, `pad` elements apart, in a heap block of exactly their size.
struct Room {
    char *p;
    int64_t rows, columns, ld;
    size_t size;
    Room(int64_t r, int64_t c, int64_t pad, size_t s, int fill = 0xAB) : rows(r), columns(c), ld(c + pad), size(s)
    {
        const size_t bytes = (size_t)((rows - 1) * ld + columns) * size;
        if (posix_memalign((void **)&p, 16, bytes)) std::abort();
        std::memset(p, fill, bytes);
        for (int64_t i = 0; i + 1 < rows && pad; i++) ASAN_POISON_MEMORY_REGION(at(i, columns), (size_t)pad * size);
    }
    Room(const Room &) = delete;
    ~Room() { std::free(p); }
    char *at(int64_t i, int64_t j) const { return p + (i * ld + j) * (int64_t)size; }
    template <class V>
    V &as(int64_t i, int64_t j = 0) const { return *reinterpret_cast<V *>(at(i, j)); }
};

long checked = 0;
void near(const char *name, int64_t i, int64_t j, double got, double want, double off)
{
    checked++;
    if (std::fabs(got - want) <= off || got == want) return;
    std::fprintf(stderr, "MISMATCH %s [%lld][%lld]: %.9g, not %.9g\n", name, (long long)i, (long long)j, got, want);
    std::exit(1);
}
void check(int rc, const char *call)
{
    if (rc == CCDC_OK) return;
    std::fprintf(stderr, "%s -> %d\n", call, rc);
    std::exit(2);
}
#define CHECK(call) check(call, #call)

int64_t padded(int64_t columns) { return (columns + 127) / 128 * 128; }
int64_t kept(int64_t columns) { return (padded(columns) / 128 + 3) / 4 * 4; }

ccdc_block_t *make()
{
    ccdc_block_config c{8, 1, mode, 0, 0, 0, 1e-6f, 1.0f, 0.0f, 0.0f};
    ccdc_block_t *b = nullptr;
    const int64_t tokens = 1;
    CHECK(ccdc_block(&c, &b));
    CHECK(ccdc_block_bind(b, 1, &tokens, nullptr));
    CHECK(ccdc_block_upload(b));
    return b;
}

void quantise(ccdc_block_t *b, int64_t rows, int64_t columns, int64_t pad)
{
    Room x(rows, columns, pad, elem()), q(rows, padded(columns), 0, 1), s(rows, kept(columns), 0, 1);
    for (int64_t i = 0; i < rows; i++)
        for (int64_t j = 0; j < columns; j++) put(x.at(i, j), uniform() * std::exp2(6 * uniform()));
    CHECK(ccdc_quantise(b, rows, columns, x.p, x.ld, q.p, s.p, nullptr));
    for (int64_t i = 0; i < rows; i++)
        for (int64_t k = 0; k < kept(columns); k++) {
            double most = 0;
            for (int64_t j = k * 128; j < std::min(columns, k * 128 + 128); j++) most = std::max(most, std::fabs(get(x.at(i, j))));
            int e = 0;
            if (most > 0)
                for (e = -127; most > 448 * std::exp2(e); e++) {}
            near("scale", i, k, s.as<unsigned char>(i, k), e + 127, 0);
            for (int64_t j = k * 128; j < std::min(padded(columns), k * 128 + 128); j++)
                near("q", i, j, q.as<unsigned char>(i, j), j < columns ? shim::to_eight((float)(get(x.at(i, j)) * std::exp2(-e))) : 0, 0);
        }
}

void fill(const Room &q, const Room &s)
{
    for (int64_t i = 0; i < q.rows; i++) {
        for (int64_t j = 0; j < q.columns; j++) q.as<unsigned char>(i, j) = (unsigned char)shim::to_eight((float)(uniform() * 300));
        for (int64_t k = 0; k < s.columns; k++) s.as<unsigned char>(i, k) = k < q.columns / 128 ? (unsigned char)(120 + (i + 3 * k) % 9) : 255;
    }
}

// Scales of a row next to one of ten places of their range, numbers of 8 bits of every size.
void fill_ends(const Room &q, const Room &s, bool back)
{
    static constexpr int places[] = {0, 3, 8, 11, 60, 127, 200, 245, 248, 254};
    for (int64_t i = 0; i < q.rows; i++) {
        for (int64_t j = 0; j < q.columns; j++) q.as<unsigned char>(i, j) = (unsigned char)((int)(63 + 63 * uniform()) | (uniform() < 0 ? 128 : 0));
        const int place = places[back ? 9 - i % 10 : i % 10];
        for (int64_t k = 0; k < s.columns; k++)
            s.as<unsigned char>(i, k) = k < q.columns / 128 ? (unsigned char)std::clamp<int>(place + (int)(i + 3 * k) % 5 - 2, 0, 254) : 255;
    }
}

void product(ccdc_block_t *b, int64_t rows, int64_t wide, int64_t outputs, int64_t pad, bool ends)
{
    Room x(rows, wide, 0, 1), xs(rows, kept(wide), 0, 1), w(outputs, wide, 0, 1), ws(outputs, kept(wide), 0, 1), y(rows, outputs, pad, elem(), 0xFF);
    if (ends) fill_ends(x, xs, false), fill_ends(w, ws, true);
    else fill(x, xs), fill(w, ws);
    CHECK(ccdc_packed_product(b, rows, outputs, wide, x.p, xs.p, w.p, ws.p, y.p, y.ld, nullptr));
    for (int64_t i = 0; i < rows; i++)
        for (int64_t j = 0; j < outputs; j++) {
            double sum = 0, size = 0;
            for (int64_t k = 0; k < wide; k++) {
                const double t = (double)shim::of_eight(x.as<unsigned char>(i, k)) * shim::of_eight(w.as<unsigned char>(j, k)) *
                                 std::exp2(xs.as<unsigned char>(i, k / 128) + ws.as<unsigned char>(j, k / 128) - 254);
                sum += t, size += std::fabs(t);
            }
            // (what no number of the results' type holds, a part of the sum maybe, is not looked at)
            if (ends && !(size < (mode == CCDC_F16_SUM_XOR ? 60000 : 0x1p127))) continue;
            // (next to zero half of the least step: of fp32 in each addition, of the results' type in the rounding)
            const double least = !ends ? 0.0 : (double)wide * 0x1p-150 + (mode == CCDC_F16_SUM_XOR ? 0x1p-25 : mode == CCDC_BF16_SUM_XOR ? 0x1p-134 : 0x1p-150);
            // binary16 has an infinity from 65520 on
            if (mode == CCDC_F16_SUM_XOR && std::fabs(sum) >= 65520) sum = std::copysign(INFINITY, sum);
            near("y", i, j, get(y.at(i, j)), sum, (double)wide * 0x1p-24 * size + half_step() * std::fabs(sum) * 1.01 + least);
        }
}

// K logits of zero at a row's end, the others far below them.
void logits_apart(const Room &z, int kind, int k, double T)
{
    const int64_t above = std::max<int64_t>(z.columns - k, 0);
    for (int64_t i = 0; i < z.rows; i++)
        for (int64_t j = 0; j < z.columns; j++) put(z.at(i, j), j >= above ? 0.0 : -T * (kind > 0 ? kind : j == above / 2 ? -kind : 5 - kind));
}

void logits(const Room &z, int kind)
{
    for (int64_t i = 0; i < z.rows; i++)
        for (int64_t j = 0; j < z.columns; j++) put(z.at(i, j), kind == 1 ? 0.5 : kind == 2 && j % 97 ? -INFINITY : 4 * uniform());
}

void top(ccdc_block_t *b, int64_t rows, int64_t columns, int k, int64_t pad, int kind)
{
    Room z(rows, columns, pad, elem()), index(rows, k, 0, 4), value(rows, k, 0, 4), rest(rows, 1, 0, 4);
    const double T = 1.5;
    const bool apart = std::abs(kind) >= 10;
    if (apart) logits_apart(z, kind, k, T);
    else logits(z, kind);
    CHECK(ccdc_top(b, rows, columns, z.p, z.ld, k, T, (int32_t *)index.p, (float *)value.p, (float *)rest.p, nullptr));
    for (int64_t i = 0; i < rows; i++) {
        std::vector<int32_t> order;
        for (int32_t j = 0; j < columns; j++)
            if (get(z.at(i, j)) > -INFINITY) order.push_back(j);
        std::stable_sort(order.begin(), order.end(), [&](int32_t l, int32_t r) { return get(z.at(i, l)) > get(z.at(i, r)); });
        double sum = 0;
        for (size_t j = 0; j < order.size(); j++) {
            const double v = get(z.at(i, order[j]));
            if ((int)j < k) near("index", i, (int64_t)j, index.as<int32_t>(i, (int64_t)j), order[j], 0), near("value", i, (int64_t)j, value.as<float>(i, (int64_t)j), v, 0);
            else sum += std::exp(v / T);
        }
        for (int j = (int)order.size(); j < k; j++) near("index", i, j, index.as<int32_t>(i, j), -1, 0), near("value", i, j, value.as<float>(i, j), -INFINITY, 0);
        // (far from zero: what is summed from by 1 / T, both rounded, and the logarithm's sum with it)
        near("rest", i, 0, rest.as<float>(i), std::log(sum), 2e-5 + (apart ? 4 * 0x1p-24 * std::fabs(std::log(sum)) : 0.0));
    }
}

void distill(ccdc_block_t *b, int64_t rows, int64_t columns, int k, int64_t pad, bool place)
{
    Room z(rows, columns, pad, elem()), out(rows, columns, pad, elem(), 0xFF), index(rows, k, 0, 4), value(rows, k, 0, 4), rest(rows, 1, 0, 4), weight(rows, 1, 0, 4),
        loss(rows, 1, 0, 4, 0xFF);
    logits(z, 0);
    const double T = 2.0, scale = 3.0;
    std::vector<std::vector<double>> before(rows, std::vector<double>(columns));
    for (int64_t i = 0; i < rows; i++) {
        for (int64_t j = 0; j < columns; j++) before[i][j] = get(z.at(i, j));
        for (int j = 0; j < k; j++) {
            index.as<int32_t>(i, j) = j % 5 == 3 ? -1 : (int32_t)((j * 37 + i * 11) % columns);       // some twice, some none
            value.as<float>(i, j) = (float)(3 * uniform());
        }
        rest.as<float>(i) = (float)uniform(), weight.as<float>(i) = i % 4 == 3 ? 0.0f : 1.5f;
    }
    char *dz = place ? z.p : out.p;
    CHECK(ccdc_distill(b, rows, columns, z.p, z.ld, k, (int32_t *)index.p, (float *)value.p, (float *)rest.p, T, (float *)weight.p, scale, (float *)loss.p, dz, z.ld, nullptr));
    for (int64_t i = 0; i < rows; i++) {
        std::vector<int> of(columns, -1), listed;
        std::vector<double> p;
        double total = std::exp((double)rest.as<float>(i)), all = 0, others = 0;
        for (int j = 0; j < k; j++) {
            const int c = index.as<int32_t>(i, j);
            if (c < 0 || of[c] >= 0) continue;
            of[c] = (int)listed.size();
            listed.push_back(c);
            p.push_back(std::exp(value.as<float>(i, j) / T));
            total += p.back();
        }
        for (int64_t j = 0; j < columns; j++) {
            const double e = std::exp(before[i][j] / T);
            all += e;
            if (of[j] < 0) others += e;
        }
        const bool counts = !listed.empty() && weight.as<float>(i) != 0.0f;
        const double w = counts ? scale * weight.as<float>(i) : 0.0, p_rest = std::exp((double)rest.as<float>(i)) / total;
        double want = others > 0 ? p_rest * std::log(p_rest / (others / all)) : INFINITY;
        for (size_t j = 0; j < listed.size(); j++) want += p[j] / total * std::log(p[j] / total / (std::exp(before[i][listed[j]] / T) / all));
        near("loss", i, 0, loss.as<float>(i), counts ? w * want : 0.0, 1e-4 * (1 + std::fabs(w)));
        for (int64_t j = 0; j < columns; j++) {
            const double q = std::exp(before[i][j] / T) / all, d = w / T * (q - (of[j] >= 0 ? p[of[j]] / total : p_rest * std::exp(before[i][j] / T) / others));
            near("dz", i, j, get(dz + (i * z.ld + j) * (int64_t)elem()), counts ? d : 0.0, half_step() * std::fabs(d) * 1.01 + 3e-5 * w * (q + 1e-3));
        }
    }
}
}  // namespace

int main(int argc, char **argv)
{
    if (argc < 6) return 2;
    const std::string what = argv[1];
    const auto number = [&](int i) { return i < argc ? std::atoll(argv[i]) : 0ll; };
    mode = (int)number(2);
    const bool ends = what == "scales";
    if (what == "product" || ends) shim::force = (int)number(7);
    ccdc_block_t *b = make();
    if (what == "quantise") quantise(b, number(3), number(4), number(5));
    else if (what == "product" || ends) product(b, number(3), number(4), number(5), number(6), ends);
    else if (what == "top") top(b, number(3), number(4), (int)number(5), number(6), (int)number(7));
    else distill(b, number(3), number(4), (int)number(5), number(6), number(7) != 0);
    ccdc_block_destroy(b);
    std::printf("%ld values, %ld launches\n", checked, shim::launches.load());
    return 0;
}
