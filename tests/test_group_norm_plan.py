"""The group norm's plans for samples that clusters of blocks hold, on the CPU: their shared memory, and how many of their blocks the GPU runs at a time."""
from tests._host_program import run_host_program

SWEEP = """
#include <cmath>
#include "block_kernels.h"
int main() {
    std::srand(5);
    auto spread = [](double low, double high) { return (int)std::exp(std::log(low) + std::rand() / (double)RAND_MAX * std::log(high / low)); };
    int bad = 0, held = 0, two = 0;
    auto look = [&](int samples, long long tokens, int channels, int groups, bool backward, bool at_once) {
        const GroupNormPlan p = plan_group_norm(samples, tokens, channels, groups, backward);
        if (!p.cluster) return;
        // what the kernels lay out: the rows' sums of each of 256 threads' channels, the channels' and groups' sums, then the vectors
        const int per_slab = p.slab / (channels / groups);
        const long long floats = backward ? 2 * 256 * p.elems + 4 * p.slab + 2 * per_slab : 256 * (2 * p.elems + 1) + 5 * per_slab, vectors = 4096ll * p.held * (backward ? 2 : 1);
        // blocks of 256 threads of up to 128 registers: two to an SM of 148, of whose 228 KB each takes one for the system
        const long long per_sm = std::min<long long>(2, 228 * 1024 / (p.smem + 1024)), blocks = (long long)p.cluster * samples * p.slabs;
        bool ok = p.smem >= 4 * floats + vectors && p.smem < 4 * floats + vectors + 128 && p.smem <= 227 * 1024;
        ok = ok && p.cluster <= 8 && p.cluster * p.chunk >= tokens && (long long)std::max(1, p.held) * p.rows * (p.held ? 1 : backward ? 4 : 8) >= p.chunk;
        if (p.held) ok = ok && blocks <= (at_once ? 1 : 2) * per_sm * 148 && (blocks <= per_sm * 148 || per_sm == 2);
        held += p.held != 0;
        two += p.held && blocks > per_sm * 148;
        if (!ok && bad++ < 10)
            std::printf("%d x %lld x %d, %d groups, backward %d: clusters of %d, %lld blocks, %lld an SM, %d held, %zu bytes for %lld\\n", samples, tokens, channels, groups, backward,
                        p.cluster, blocks, per_sm, p.held, p.smem, 4 * floats + vectors);
    };
    for (int i = 0; i < 200000; ++i) {
        const int channels = (i % 4 ? 8 : 1) * spread(1, 300), samples = spread(1, 400);
        int groups = spread(1, channels + 1);
        while (channels % groups) --groups;
        look(samples, spread(1, 20000), channels, groups, i & 1, false);
    }
    // fewer blocks to a cluster put these on the GPU at a time
    look(16, 280, 960, 4, true, true);
    look(64, 1178, 56, 1, true, true);
    look(32, 73, 1320, 2, true, true);
    look(3, 4189, 640, 32, false, true);
    look(64, 498, 264, 8, false, true);
    std::printf("%d bad, %d held in shared memory, %d in two turns\\n", bad, held, two);
    return bad != 0 || held < 1000 || two < 100;
}
"""


def test_clusters_fit(tmp_path):
    run_host_program(tmp_path, SWEEP)
