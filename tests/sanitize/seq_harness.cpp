// Host-only driver for AddressSanitizer / UndefinedBehaviorSanitizer runs, built with g++ (no GPU
// code): the sequence operators' argument checks and plans (seq_host.h).  Every plan must cover
// its problem, fit its launch and size its workspace without overflow, at the largest shapes that
// the checks let through too; the overlap check of outputs is compared with all pairs of rows.
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include <limits>
#include <utility>
#include <vector>

#include "seq_host.h"

using namespace snnlif;

static int failures = 0;

#define CHECK(cond)                                                                       \
    do {                                                                                  \
        if (!(cond)) {                                                                    \
            std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #cond); \
            ++failures;                                                                   \
        }                                                                                 \
    } while (0)

struct Shape {
    int64_t T, B, F;
};

static std::vector<Shape> shapes() {
    std::vector<Shape> all;
    for (int64_t T : {1, 2, 15, 16, 17, 127, 128, 129, 333, 4096, 100000})
        for (int64_t B : {1, 2, 7, 64, 300})
            for (int64_t F : {1, 3, 8, 63, 64, 65, 777, 4096, 8193, 70001}) all.push_back({T, B, F});
    // as large as the checks allow
    const int64_t t = kMaxSeqT, b = kMaxSeqB, f = kMaxSeqF, one = 1;
    for (const Shape& s : {Shape{t, one, one}, {one, b, one}, {one, one, f}, {t / 2, 2, one << 13}, {one, b, one << 20},
                           {1 << 20, 1, f}, {64, b, one << 14}, {one << 6, one << 24, one}, {one, 128, f}})
        all.push_back(s);
    return all;
}

static void check_shapes() {
    const int64_t big = std::numeric_limits<int64_t>::max();
    CHECK(check_seq_shape(0, 0, 0) == SNN_OK);
    for (const Shape& s : {Shape{-1, 1, 1}, {1, -1, 1}, {1, 1, -1}, {kMaxSeqT + 1, 1, 1}, {1, kMaxSeqB + 1, 1},
                           {1, 1, kMaxSeqF + 1}, {big, big, big}, {kMaxSeqT, 4, 1}, {1 << 20, 1 << 10, 1 << 20}})
        CHECK(check_seq_shape(s.T, s.B, s.F) == SNN_E_SHAPE);
    for (const Shape& s : shapes()) CHECK(check_seq_shape(s.T, s.B, s.F) == SNN_OK);
}

static void check_spans() {
    const int64_t big = std::numeric_limits<int64_t>::max();
    alignas(16) static char data[16];
    const auto span = [](int64_t t, int64_t b, int64_t T, int64_t B, int64_t X) {
        const snn_seq s = {data, t, b};
        return seq_span(&s, T, B, X);
    };
    CHECK(span(big, big, 1, 1, 5) == 5);             // steps of axes of length 1 are not used
    CHECK(span(-1, 0, 2, 1, 5) == -1 && span(0, -1, 1, 2, 5) == -1);
    CHECK(span(big, 0, 2, 1, 5) == -1 && span(0, big, 1, 2, 5) == -1);
    CHECK(span(kMaxSpan, kMaxSpan, 2, 2, 5) == -1);
    CHECK(span(0, 0, 7, 7, 5) == 5);
    CHECK(span(30, 10, 4, 3, 10) == 120);
    // outputs: exactly those are taken whose rows do not touch, of layouts with one axis inside
    // the other; no overlapping one may pass
    for (int64_t T = 1; T <= 3; ++T)
        for (int64_t B = 1; B <= 3; ++B)
            for (int64_t X = 1; X <= 3; ++X)
                for (int64_t t = 0; t <= 13; ++t)
                    for (int64_t b = 0; b <= 13; ++b) {
                        const snn_seq s = {data, t, b};
                        bool overlap = false;
                        std::vector<int> hit(size_t((T - 1) * t + (B - 1) * b + X), 0);
                        for (int64_t i = 0; i < T; ++i)
                            for (int64_t j = 0; j < B; ++j)
                                for (int64_t k = 0; k < X; ++k) overlap |= hit[size_t(i * t + j * b + k)]++ > 0;
                        const bool taken = check_out(&s, T, B, X, SNN_IO_F32) == SNN_OK;
                        CHECK(!(taken && overlap));
                        const bool dense = (b == X || B == 1) && (t == B * X || T == 1);
                        const bool batch = (t == X || T == 1) && (b == T * X || B == 1);
                        if (dense || batch) CHECK(taken);
                    }
    const snn_seq none = {nullptr, 1, 1}, odd = {data + 1, 8, 8};
    CHECK(check_in(nullptr, 1, 1, 1, SNN_IO_F32) == SNN_E_NULL && check_in(&none, 1, 1, 1, SNN_IO_F32) == SNN_E_NULL);
    CHECK(check_in(&odd, 1, 1, 1, SNN_IO_BF16) == SNN_E_ALIGN);
    CHECK(first_error({SNN_E_SHAPE, SNN_E_NULL}) == SNN_E_NULL && first_error({SNN_OK, SNN_E_ALIGN}) == SNN_E_ALIGN);
}

static void check_conv() {
    for (const Shape& s : shapes())
        for (int io : {SNN_IO_F32, SNN_IO_BF16})
            for (int w : {1, 4, 8})
                for (bool backward : {false, true}) {
                    const snn_conv_cfg c = {io, w, SNN_ACT_SILU};
                    CHECK(check_conv_cfg(&c) == SNN_OK);
                    const ConvPlan p = conv_plan(&c, s.T, s.B, s.F, backward);
                    const int v = conv_vec(io, backward);
                    CHECK(p.lanes == s.F / v + s.F % v);
                    CHECK(p.steps >= conv_rows(backward) && p.chunks >= 1);
                    CHECK(p.steps * p.chunks >= s.T && p.steps * (p.chunks - 1) < s.T);
                    CHECK(conv_workspace(&c, s.T, s.B, s.F) >= p.chunks && conv_workspace(&c, s.T, s.B, s.F) % 256 == 0);
                }
}

static void check_scan() {
    for (const Shape& s : shapes())
        for (int S : {1, 4, 5, 8, 16, 17, 33, 64})
            for (int G : {1, 3, 7}) {
                if (s.F % G != 0 || s.F > kMaxN / s.B) continue;
                const snn_scan_cfg c = {SNN_IO_BF16, S, G, 1};
                CHECK(check_scan_cfg(&c) == SNN_OK);
                const ScanPlan p = scan_plan(&c, s.T, s.B, s.F);
                CHECK(p.waves * kScanStates >= S && p.waves <= 16 && (p.waves & (p.waves - 1)) == 0);
                CHECK(p.tiles * kWave >= s.F / G && (p.tiles - 1) * kWave < s.F / G);
                CHECK(p.segments >= 1 && p.segments <= kMaxSegments);
                CHECK(p.steps * p.segments >= s.T && p.steps * (p.segments - 1) < s.T);
                // segments start on blocks of either direction and on kept states
                if (p.segments > 1) CHECK(p.steps % 16 == 0 && p.steps % p.keep == 0 && p.steps % kScanBlock == 0);
                CHECK(p.keep == 8 || p.keep == 16);
                for (int64_t n : {scan_saved(&c, s.T, s.B, s.F), scan_part_h(&c, p, s.B, s.F), scan_part_d(p, s.B, s.F),
                                  scan_partial_bc(&c, p, s.T, s.B), scan_forward_workspace(&c, s.T, s.B, s.F),
                                  scan_backward_workspace(&c, s.T, s.B, s.F)})
                    CHECK(n >= 0);
                if (s.T > p.keep) CHECK(scan_saved(&c, s.T, s.B, s.F) > 0);
                CHECK(scan_backward_workspace(&c, s.T, s.B, s.F) > 0);
            }
    for (const snn_scan_cfg& c : {snn_scan_cfg{2, 8, 1, 1}, {0, 0, 1, 1}, {0, 65, 1, 1}, {0, 8, 0, 1}, {0, 8, 1, 2}})
        CHECK(check_scan_cfg(&c) == SNN_E_PARAM);
}

static void check_norm() {
    for (const Shape& s : shapes()) {
        const int lanes = norm_lanes(s.F);
        CHECK(lanes % kWave == 0 && lanes <= 1024);
        CHECK(s.F > kNormRegs || lanes * kNormLane >= s.F);
        for (bool backward : {false, true}) {
            const int64_t g = norm_groups(s.T, s.B, s.F, backward);
            CHECK(g >= 1 && g <= s.T * s.B && g <= 256 * 32);
        }
        CHECK(norm_workspace(s.T, s.B, s.F) >= 3 * s.F * 4);
    }
    const float nan = std::numeric_limits<float>::quiet_NaN(), inf = std::numeric_limits<float>::infinity();
    for (float e : {0.0f, -1.0f, nan, inf}) {
        const snn_norm_cfg c = {SNN_IO_F32, e};
        CHECK(check_norm_cfg(&c) == SNN_E_PARAM);
    }
}

int main() {
    check_shapes();
    check_spans();
    check_conv();
    check_scan();
    check_norm();
    if (failures != 0) return 1;
    std::puts("all checks passed");
    return 0;
}
