// Host-only driver for AddressSanitizer / UndefinedBehaviorSanitizer runs, built with g++ (no GPU
// code): what the sequence operators' plans (seq_host.h) decide, at the shapes that the GPU tests
// use to reach a path.
#include <cstdint>
#include <cstdio>
#include <initializer_list>

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
    for (int64_t T : {1, 2, 127, 128, 270, 333, 442, 3072, 4096, 131072})
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

int main() {
    check_states_in_place();
    if (failures != 0) return 1;
    std::puts("all checks passed");
    return 0;
}
