// Runs the calls of a trained block, compiled for the host against block_lanes.hpp, on small shapes under AddressSanitizer / UBSan,
// and checks what they give against the formulas of ccdc.h in 64 bits.  Every matrix is a heap block of exactly its size, what
// lies between its rows is poisoned; results begin as NaN.  Test infrastructure only.
// Usage: block_driver ffn MODE ACT WIDTH HIDDEN P LD TRAIN ROWS TILE TOKENS...       (TRAIN 0: forward of the first ROWS rows; TILE: shim::force)
//        block_driver join MODE CENTRED WIDTH P LD GATE PARTS TOKENS...             (GATE 0 none, 1 shared, 2 by file; PARTS: of "fnr")
//        block_driver dropout MODE COLUMNS P LD RESIDUAL TOKENS...
#include <sanitizer/asan_interface.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>

#include "block_lanes.hpp"
#include "ccdc.h"

namespace {
using Row = std::vector<double>;
using Matrix = std::vector<Row>;

int mode;
size_t elem() { return mode == CCDC_BF16_SUM_XOR || mode == CCDC_F16_SUM_XOR ? 2 : 4; }
double tolerance() { return mode == CCDC_BF16_SUM_XOR ? 4e-2 : mode == CCDC_F16_SUM_XOR ? 5e-3 : 5e-5; }

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
        const uint16_t h = v != v ? 0x7FC0 : (uint16_t)((u + 0x7FFF + (u >> 16 & 1)) >> 16);
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

// A matrix of the mode's elements with row stride ld, aligned to its elements only.
struct Device {
    char *room = nullptr, *p = nullptr;
    int64_t rows, columns, ld;
    Device(int64_t r, int64_t c, int64_t l = 0, double scale = 0.0) : rows(r), columns(c), ld(l ? l : c)
    {
        const size_t bytes = (rows ? (size_t)(rows - 1) * ld + columns : 0) * elem();
        room = static_cast<char *>(std::malloc(bytes + elem()));
        p = room + (l > c ? elem() : 0);              // strided ones begin where no pack does
        if (p == room) {                              // exactly as large
            std::free(room);
            room = p = static_cast<char *>(std::malloc(bytes ? bytes : 1));
        }
        for (int64_t i = 0; i < rows; i++)
            for (int64_t j = 0; j < columns; j++) put(at(i, j), scale != 0.0 ? uniform() * scale : (double)NAN);
        for (int64_t i = 0; i + 1 < rows; i++)
            if (ld > columns) ASAN_POISON_MEMORY_REGION(at(i, columns), (size_t)(ld - columns) * elem());
    }
    Device(const Device &) = delete;
    ~Device() { std::free(room); }
    char *at(int64_t i, int64_t j) const { return p + (i * ld + j) * (int64_t)elem(); }
    Matrix values() const
    {
        Matrix m(rows, Row(columns));
        for (int64_t i = 0; i < rows; i++)
            for (int64_t j = 0; j < columns; j++) m[i][j] = get(at(i, j));
        return m;
    }
};

long checked = 0;
void compare(const char *name, const Device &got, const Matrix &want, double scale = 1.0)
{
    for (int64_t i = 0; i < got.rows; i++)
        for (int64_t j = 0; j < got.columns; j++, checked++) {
            const double g = get(got.at(i, j)), off = std::fabs(g - want[i][j]);
            if (!(off <= tolerance() * (scale + std::fabs(want[i][j])))) {
                std::fprintf(stderr, "MISMATCH %s [%lld][%lld]: %g, not %g\n", name, (long long)i, (long long)j, g, want[i][j]);
                std::exit(1);
            }
        }
}
void check(int rc, const char *call)
{
    if (rc == CCDC_OK) return;
    std::fprintf(stderr, "%s -> %d\n", call, rc);
    std::exit(2);
}
#define CHECK(call) check(call, #call)

std::vector<int64_t> tokens;
std::vector<int32_t> ids, file_of, token_of;

// Dropout's factor (ccdc.h).
double factor(double p, uint32_t site, uint64_t seed, int64_t row, int64_t column)
{
    const long thr = std::lrint((double)p * 65536.0);
    uint32_t c[4] = {(uint32_t)(column / 8), (uint32_t)token_of[row], (uint32_t)ids[file_of[row]], site}, k[2] = {(uint32_t)seed, (uint32_t)(seed >> 32)};
    for (int r = 0; r < 10; r++) {
        const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
        const uint32_t n[4] = {(uint32_t)(b >> 32) ^ c[1] ^ k[0], (uint32_t)b, (uint32_t)(a >> 32) ^ c[3] ^ k[1], (uint32_t)a};
        std::memcpy(c, n, 16);
        k[0] += 0x9E3779B9u, k[1] += 0xBB67AE85u;
    }
    const long half = c[column % 8 / 2] >> (column % 2 * 16) & 0xFFFF;
    return half >= thr ? 65536.0 / (double)(65536 - thr) : 0.0;
}

ccdc_block_t *bound(ccdc_block_config c)
{
    ccdc_block_t *b = nullptr;
    CHECK(ccdc_block(&c, &b));
    CHECK(ccdc_block_bind(b, (int)tokens.size(), tokens.data(), ids.data()));
    CHECK(ccdc_block_upload(b));
    return b;
}

int64_t batch(int argc, char **argv, int from)
{
    for (int i = from; i < argc; i++) {
        const int n = (int)tokens.size();
        tokens.push_back(std::atoll(argv[i]));
        ids.push_back(5 * n + 2);
        for (int64_t t = 0; t < tokens.back(); t++) file_of.push_back(n), token_of.push_back((int32_t)t);
    }
    return (int64_t)file_of.size();
}

constexpr uint64_t kSeed = 0x9E3779B97F4A7C15ull;

int ffn(int argc, char **argv)
{
    const int act = std::atoi(argv[3]);
    const int64_t d = std::atoll(argv[4]), F = std::atoll(argv[5]), ld = std::atoll(argv[7]);
    const float p = (float)std::atof(argv[6]);
    const bool train = std::atoi(argv[8]);
    const int64_t M = batch(argc, argv, 11), rows = train ? M : std::atoll(argv[9]);
    shim::force = std::atoi(argv[10]);
    ccdc_block_t *b = bound({d, F, mode, act, CCDC_NORM_RMS, 3, 1e-6f, 1.0f, p, 0.0f});
    Device x(rows, d, ld, 1.7), in(2 * F, d, 0, 1.7 / std::sqrt(d)), out(d, F, 0, 1.7 / std::sqrt(F)), y(rows, d, ld), dy(rows, d, ld, 1.0), dx(rows, d, ld);
    int64_t bytes = 0;
    CHECK(ccdc_block_query(b, CCDC_BLOCK_Q_SAVED_BYTES, &bytes, 8));
    void *saved = nullptr;
    if (train && posix_memalign(&saved, 16, bytes ? bytes : 16)) return 2;
    if (train) std::memset(saved, 0xFF, bytes);
    CHECK(ccdc_ffn_forward(b, rows, x.p, x.ld, in.p, out.p, y.p, y.ld, saved, kSeed, nullptr));
    const Matrix vx = x.values(), vi = in.values(), vo = out.values(), vg = dy.values();
    Matrix h(rows, Row(F)), P = h, Q = h, wy(rows, Row(d));
    for (int64_t m = 0; m < rows; m++) {
        for (int64_t f = 0; f < F; f++) {
            double a = 0, u = 0;
            for (int64_t k = 0; k < d; k++) a += vx[m][k] * vi[f][k], u += vx[m][k] * vi[F + f][k];
            const double s = 1 / (1 + std::exp(-a)), cdf = 0.5 * (1 + std::erf(a / std::sqrt(2.0)));
            const double value = act == 0 ? a * s : act == 1 ? a * cdf : a > 0 ? a : 0;
            const double slope = act == 0 ? s + a * s * (1 - s) : act == 1 ? cdf + a * std::exp(-a * a / 2) / std::sqrt(2 * M_PI) : a > 0;
            const double keep = p > 0 ? factor(p, 6, kSeed, m, f) : 1.0;
            h[m][f] = value * u * keep, P[m][f] = slope * u * keep, Q[m][f] = value * keep;
        }
        for (int64_t c = 0; c < d; c++)
            for (int64_t f = 0; f < F; f++) wy[m][c] += h[m][f] * vo[c][f];
    }
    compare("y", y, wy);
    if (train) {
        const int64_t N = (int64_t)tokens.size(), room = 3 * F * d + 3;
        Device V(N, 3 * F * d, room);                 // rows of V: dW_in, then dW_out, and a gap
        char *dout = V.p + 2 * F * d * (int64_t)elem();
        CHECK(ccdc_ffn_backward(b, x.p, x.ld, in.p, out.p, saved, dy.p, dy.ld, dx.p, dx.ld, V.p, room, dout, room, nullptr));
        Matrix wx(rows, Row(d)), wV(N, Row(3 * F * d));
        for (int64_t m = 0; m < rows; m++)
            for (int64_t f = 0; f < F; f++) {
                double dh = 0;
                for (int64_t c = 0; c < d; c++) dh += vg[m][c] * vo[c][f];
                const double da = dh * P[m][f], du = dh * Q[m][f];
                Row &w = wV[file_of[m]];
                for (int64_t k = 0; k < d; k++) {
                    wx[m][k] += da * vi[f][k] + du * vi[F + f][k];
                    w[f * d + k] += da * vx[m][k], w[(F + f) * d + k] += du * vx[m][k];
                    w[2 * F * d + k * F + f] += vg[m][k] * h[m][f];
                }
            }
        compare("dx", dx, wx);
        compare("V", V, wV, 4.0);
    }
    std::free(saved);
    ccdc_block_destroy(b);
    return 0;
}

struct Norm {
    Row hat;
    double rstd;
};
Norm norm(const Row &v, bool centred, double eps)
{
    Norm n{v, 0};
    double mean = 0, square = 0;
    for (double e : v) mean += e / (double)v.size();
    if (centred)
        for (double &e : n.hat) e -= mean;
    for (double e : n.hat) square += e * e / (double)v.size();
    n.rstd = 1 / std::sqrt(square + eps);
    for (double &e : n.hat) e *= n.rstd;
    return n;
}
Row norm_gradient(const Row &e, const Norm &n, bool centred)
{
    double dot = 0, mean = 0;
    for (size_t i = 0; i < e.size(); i++) dot += e[i] * n.hat[i] / (double)e.size(), mean += e[i] / (double)e.size();
    Row g(e.size());
    for (size_t i = 0; i < e.size(); i++) g[i] = n.rstd * (e[i] - n.hat[i] * dot - (centred ? mean : 0));
    return g;
}

int join(int argc, char **argv)
{
    const bool centred = std::atoi(argv[3]);
    const int64_t d = std::atoll(argv[4]), ld = std::atoll(argv[6]);
    const float p = (float)std::atof(argv[5]), eps = 1e-3f, rho = 0.75f;
    const int gating = std::atoi(argv[7]);
    const std::string parts = argv[8];
    const bool with_f = parts.find('f') != parts.npos, with_n = parts.find('n') != parts.npos, with_r = parts.find('r') != parts.npos;
    const int64_t M = batch(argc, argv, 9), N = (int64_t)tokens.size(), stride = ld ? ld : d;
    ccdc_block_t *b = bound({d, 8, mode, CCDC_ACT_SILU, centred ? CCDC_NORM_CENTRED : CCDC_NORM_RMS, 3, eps, rho, 0.0f, p});
    Device x(M, d, ld, 2.0), f(M, d, ld, 1.0), post(1, d, 0, 1.0), gate(gating == 2 ? N : 1, d, gating == 2 ? d + 5 : 0, 1.0), pre(1, d, 0, 1.0);
    Device y(M, d, ld), n(M, d, ld), dn(M, d, ld, 0.5), dr(M, d, ld, 0.5), dx(M, d, ld), df(M, d, ld);
    Device dpost(N, d, d + 3), dgate(N, d, d + 3), dpre(N, d, d + 3);
    const int64_t ld_gate = gating == 2 ? gate.ld : 0;
    void *g = gating ? gate.p : nullptr;
    CHECK(ccdc_join_forward(b, M, x.p, with_f ? f.p : nullptr, post.p, g, ld_gate, pre.p, y.p, with_n ? n.p : nullptr, stride, kSeed, nullptr));
    const Matrix vx = x.values(), vf = f.values(), vp = post.values(), vg = gate.values(), vw = pre.values(), vdn = dn.values(), vdr = dr.values();
    Matrix wy(M, Row(d)), wn = wy, keep(M, Row(d, 1.0));
    for (int64_t m = 0; m < M; m++) {
        const Norm z = norm(vf[m], centred, eps);
        for (int64_t c = 0; c < d; c++) {
            if (p > 0) keep[m][c] = factor(p, 7, kSeed, m, c);
            const double ga = gating ? vg[gating == 2 ? file_of[m] : 0][c] : 1.0;
            wy[m][c] = rho * vx[m][c] + (with_f ? ga * keep[m][c] * z.hat[c] * vp[0][c] : 0.0);
        }
        const Norm next = norm(wy[m], centred, eps);
        for (int64_t c = 0; c < d; c++) wn[m][c] = next.hat[c] * vw[0][c];
    }
    compare("y", y, wy);
    if (with_n) compare("n", n, wn);
    CHECK(ccdc_join_backward(b, with_n ? dn.p : nullptr, with_r ? dr.p : nullptr, with_n ? y.p : nullptr, with_f ? f.p : nullptr, post.p, g, ld_gate,
                             pre.p, dx.p, with_f ? df.p : nullptr, stride, with_f ? dpost.p : nullptr, with_f ? dgate.p : nullptr,
                             with_n ? dpre.p : nullptr, d + 3, kSeed, nullptr));
    const Matrix vy = y.values();
    Matrix wx(M, Row(d)), wf = wx, wpost(N, Row(d)), wgate = wpost, wpre = wpost;
    for (int64_t m = 0; m < M; m++) {
        Row dy = with_r ? vdr[m] : Row(d);
        const int file = file_of[m];
        if (with_n) {
            const Norm yhat = norm(vy[m], centred, eps);
            Row e(d);
            for (int64_t c = 0; c < d; c++) e[c] = vdn[m][c] * vw[0][c], wpre[file][c] += vdn[m][c] * yhat.hat[c];
            const Row back = norm_gradient(e, yhat, centred);
            for (int64_t c = 0; c < d; c++) dy[c] += back[c];
        }
        const Norm z = norm(vf[m], centred, eps);
        Row e(d);
        for (int64_t c = 0; c < d; c++) {
            const double ga = gating ? vg[gating == 2 ? file : 0][c] : 1.0, kd = keep[m][c] * dy[c];
            wx[m][c] = rho * dy[c];
            e[c] = kd * ga * vp[0][c];
            wpost[file][c] += kd * ga * z.hat[c], wgate[file][c] += kd * vp[0][c] * z.hat[c];
        }
        wf[m] = norm_gradient(e, z, centred);
    }
    compare("dx", dx, wx);
    if (with_f) compare("df", df, wf, 2.0), compare("dw_post", dpost, wpost, 8.0), compare("dgate", dgate, wgate, 8.0);
    if (with_n) compare("dw_pre", dpre, wpre, 8.0);
    ccdc_block_destroy(b);
    return 0;
}

int dropout(int argc, char **argv)
{
    const int64_t columns = std::atoll(argv[3]), ld = std::atoll(argv[5]);
    const double p = std::atof(argv[4]);
    const bool residual = std::atoi(argv[6]);
    const int64_t M = batch(argc, argv, 7);
    ccdc_block_t *b = bound({8, 8, mode, CCDC_ACT_SILU, CCDC_NORM_RMS, 3, 1e-6f, 1.0f, 0.0f, 0.0f});
    Device x(M, columns, ld, 1.0), res(M, columns, 0, 1.0), y(M, columns, ld ? ld + 2 : 0);
    CHECK(ccdc_dropout(b, M, columns, p, 9, kSeed, x.p, x.ld, residual ? res.p : nullptr, res.ld, y.p, y.ld, nullptr));
    Matrix want = x.values();
    const Matrix vr = res.values();
    for (int64_t m = 0; m < M; m++)
        for (int64_t c = 0; c < columns; c++) want[m][c] = want[m][c] * factor(p, 9, kSeed, m, c) + (residual ? vr[m][c] : 0.0);
    compare("y", y, want);
    ccdc_block_destroy(b);
    return 0;
}
}  // namespace

int main(int argc, char **argv)
{
    if (argc < 5) return 2;
    mode = std::atoi(argv[2]);
    const std::string what = argv[1];
    const int rc = what == "ffn" ? ffn(argc, argv) : what == "join" ? join(argc, argv) : dropout(argc, argv);
    if (rc == 0) std::printf("%s: %ld values, %ld launches\n", what.c_str(), checked, shim::launches.load());
    return rc;
}
