// Host-only driver for AddressSanitizer / UndefinedBehaviorSanitizer runs, built with g++ (no GPU
// code): what the sequence operators' plans (seq_host.h) decide, at the shapes that the GPU tests
// use to reach a path.
#include <chrono>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include <limits>

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

static ScanPlan plan_of(int64_t T, int64_t B, int64_t F, int S, int G = 1) {
    const snn_scan_cfg c = {SNN_IO_F32, S, G, 1};
    return scan_plan(&c, T, B, F);
}

// A state updated in place: written by the last segment's workgroups while others may still start
// from it, unless those read it before the scan starts.
static void check_states_in_place() {
    float states[2] = {};
    float *h = &states[0], *other = &states[1];
    bool several = false, many = false;
    for (int64_t T : {1, 2, 127, 128, 270, 333, 442, 3300, 4096, 131072})
        for (int64_t B : {1, 2, 7})
            for (int64_t F : {1, 64, 777, 2928})
                for (int S : {1, 7, 16, 47, 64}) {
                    const ScanPlan p = plan_of(T, B, F, S);
                    several |= p.segments > 1 && p.segments <= kWalkSegments;
                    many |= p.segments > kWalkSegments;
                    CHECK(scan_walks(p, h, h) == (p.segments == 1));
                    for (const float* from : {static_cast<const float*>(nullptr), static_cast<const float*>(other)}) {
                        CHECK(scan_walks(p, from, h) == (p.segments <= kWalkSegments));
                        CHECK(scan_walks(p, from, nullptr) == (p.segments <= kWalkSegments));
                    }
                }
    CHECK(several && many);
    // more workgroups of 16 waves than CUs, in several segments
    const ScanPlan p = plan_of(442, 2, 2928, 47);
    CHECK(p.waves == 16 && p.segments > 1 && p.segments <= kWalkSegments && p.tiles * 2 * p.segments > 256);
}

// Every launch that the checks let through has fewer than 2^32 threads along x and workgroups for
// all of its work, at the header's limits too.
static void check_launches() {
    const auto fits = [](const dim3& g, int64_t blocks, int threads) {
        return int64_t(g.x) * threads < (int64_t(1) << 32) && g.y <= 65535 && g.z <= 65535 &&
               int64_t(g.x) * g.z >= blocks && int64_t(g.x) * g.z <= std::numeric_limits<unsigned>::max() &&
               int64_t(g.x) * (g.z - 1) < blocks;
    };
    for (int threads : {64, 128, 256, 512, 1024})
        for (int64_t blocks : {int64_t(1), int64_t(2), int64_t(255), (int64_t(1) << 21) - 1, int64_t(1) << 21,
                               (int64_t(1) << 21) + 1, (int64_t(1) << 26) + 7, kMaxBlocks - 1, kMaxBlocks}) {
            const dim3 g = layered_grid(blocks, threads);
            CHECK(fits(g, blocks, threads));
            if (blocks * threads <= int64_t(1) << 31) CHECK(g.z == 1 && g.x == blocks);
        }
    const int64_t K = 1024, M = K * K;
    struct Shape {
        int64_t T, B, F;
        int G;
    };
    for (const Shape& s : {Shape{4096, 1024, 512, 8}, {64, 65536, 8, 8}, {2, 16384, 4096, 4096}, {2, 65536, 4096, 1},
                           {1, 16384, 65536, 1}, {1, 128, 16 * M, 1}, {1, 1, 16 * M, 16 * int(M)}, {K * M, 1, 1, 1},
                           {1, 16 * M, 128, 1}, {32, 16 * M, 2, 2}})
        for (int S : {1, 4, 16, 64}) {
            const snn_scan_cfg c = {SNN_IO_BF16, S, s.G, 1};
            CHECK(check_seq_shape(s.T, s.B, s.F) == SNN_OK);
            const ScanPlan p = scan_plan(&c, s.T, s.B, s.F);
            const int64_t blocks = p.tiles * s.G * s.B;
            CHECK(blocks <= kMaxBlocks && s.T * s.B * s.G <= kMaxBlocks);
            CHECK(fits(scan_grid(p, s.B, s.G, p.segments), blocks, p.waves * kWave));
            const int64_t join = ceil_div(scan_partial_values(s.F, S), kWave) + ceil_div(s.T * s.B * s.G * 2 * S, 1024);
            CHECK(fits(layered_grid(join, 1024), join, 1024));
            for (int n : {1, 4}) {
                const int64_t token = ceil_div(ceil_div(s.B, n) * s.F * p.waves, 256);
                CHECK(fits(layered_grid(token, 256), token, 256));
            }
            if (p.segments > 1) CHECK(s.B * scan_held_states(S) * s.F <= kMaxThreads - kBlock);
        }
    // the convolution's lanes up to B * F = 2^31, and the sums of partial results
    for (const Shape& s : {Shape{1, 128, 16 * M, 1}, {32, 16 * M, 128, 1}, {K * M, 1, 1, 1}, {64, 16 * M, 16, 1}, {1, 16 * M, 127, 1}})
        for (bool backward : {false, true}) {
            const snn_conv_cfg c = {SNN_IO_F32, 8, SNN_ACT_SILU};
            const ConvPlan p = conv_plan(&c, s.T, s.B, s.F, backward);
            CHECK(p.lanes * s.B * p.chunks <= kMaxThreads - kBlock);
        }
    const snn_conv_cfg widest = {SNN_IO_F32, kMaxTaps, SNN_ACT_SILU};
    CHECK(ceil_div(conv_partial(&widest, kMaxSeqF), kWave) * 1024 <= kMaxThreads);
    CHECK(ceil_div(3 * kMaxSeqF, kWave) * 1024 <= kMaxThreads);
    // the example that a grid of one layer does not take
    CHECK(layered_grid(ceil_div(int64_t(4096) * 1024 * 8 * 2 * 64, 1024), 1024).z > 1);
}

// 33 to 64 states: the segments' length is the cheapest of all multiples of 16 between half and twice
// the one to start from, the shortest of several, and finding it does not take longer with more steps.
static void check_segment_search() {
    int searched = 0;
    for (int64_t T : {128, 129, 333, 442, 1000, 4096, 20000})
        for (int64_t B : {1, 2, 7})
            for (int64_t F : {1, 64, 378, 1152, 2928, 4096})
                for (int S : {33, 47, 64}) {
                    const ScanPlan p = plan_of(T, B, F, S);
                    if (p.segments == 1) continue;
                    const int64_t groups = p.tiles * B, waves = groups * ceil_div(S, 4);
                    const int64_t most = std::min({ceil_div(T, 16), int64_t(std::sqrt(2.0 * double(T))), kMaxSegments});
                    const int64_t want = std::min(std::max<int64_t>(4096 / waves, 2), most);
                    const auto cost = [&](int64_t n) { return ceil_div(groups * ceil_div(T, n), 256) * (n + 16); };
                    const int64_t start = ceil_div(ceil_div(T, want), 16) * 16;
                    int64_t best = start;
                    for (int64_t n = 16; n < T; n += 16)
                        if (n >= start / 32 * 16 && n <= 2 * start && ceil_div(T, n) <= most && cost(n) < cost(best)) best = n;
                    CHECK(p.steps == best);
                    searched += best != start;
                }
    CHECK(searched > 10);
    const auto from = std::chrono::steady_clock::now();
    int64_t sum = 0;
    for (int i = 0; i < 400; ++i) sum += plan_of((1 << 24) + i, 1, 2928, 64).segments;
    CHECK(sum > 400);
    // a search through all lengths takes 3 ms each, and more under the sanitizers
    CHECK(std::chrono::duration<double>(std::chrono::steady_clock::now() - from).count() < 0.4);
}

// The shapes of tests/test_gpu_sequence_long.py.
static void check_paths() {
    CHECK(plan_of(4096, 1, 20, 16).segments > kWalkSegments);
    CHECK(plan_of(3300, 3, 6, 3, 2).segments > kWalkSegments);
    CHECK(plan_of(3200, 2, 40, 33).segments > kWalkSegments);
    const ScanPlan rounds = plan_of(160, 2, 2928, 47);
    CHECK(rounds.waves == 16 && rounds.segments > 1 && rounds.tiles * 2 * rounds.segments > 256);
    struct Conv {
        int io, width;
        int64_t T, B, F;
    };
    for (const Conv& s : {Conv{SNN_IO_BF16, 4, 1003, 16, 2059}, {SNN_IO_F32, 3, 700, 9, 2051}, {SNN_IO_BF16, 8, 2100, 8, 2056}})
        for (bool backward : {false, true}) {
            const snn_conv_cfg c = {s.io, s.width, SNN_ACT_SILU};
            const ConvPlan p = conv_plan(&c, s.T, s.B, s.F, backward);
            CHECK(p.steps > conv_rows(backward) && p.chunks > 1);
        }
    for (const auto& [T, B, F] : {std::tuple<int64_t, int64_t, int64_t>{250, 5, 4097}, {1100, 4, 1030}, {130, 5, 9000}, {3000, 3, 66}})
        for (bool backward : {false, true}) CHECK(norm_groups(T, B, F, backward) < T * B);
}

int main() {
    check_states_in_place();
    check_paths();
    check_segment_search();
    check_launches();
    if (failures != 0) return 1;
    std::puts("all checks passed");
    return 0;
}
