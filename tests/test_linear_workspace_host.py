"""What the products' backward asks for as a workspace, on the CPU: its own sums' parts and no others, and what goes through a gate finds room in as much."""
import pytest

import paper_2608_15211_b200 as terra
from tests._host_program import run_host_program

SWEEP = """
#include <cmath>
#include "block_kernels.h"
int main() {
    std::srand(7);
    auto spread = [](double low, double high) { return (long long)std::exp(std::log(low) + std::rand() / (double)RAND_MAX * std::log(high / low)); };
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    int bad = 0, split = 0;
    for (int i = 0; i < 3000; ++i) {
        const long long rows = spread(1, 1e6);
        const int n_in = 8 * (int)spread(1, 1000), n_out = 8 * (int)spread(1, 1000);      // (rows of whole 16 bytes: no padded copies)
        const terra_linear_desc d = {rows, n_in, n_out, 0, 0};
        const LinearPlan first = plan_linear(kLinearInput, false, rows, n_in, n_out), second = plan_linear(kLinearWeights, false, n_out, n_in, rows);
        size_t parts = 0, bytes = 0;
        if (first.splits > 1) parts = sizeof(float) * first.splits * rows * n_in;
        if (second.splits > 1) parts = std::max<size_t>(parts, sizeof(float) * second.splits * n_out * n_in);
        const size_t sums = sizeof(float) * std::max<size_t>(column_sum_blocks(rows, n_out), second.splits * second.n_tiles) * n_out;
        const int rc = terra_linear_workspace_bytes(&d, TERRA_LINEAR_BWD, &bytes);
        const LinearPlan gated = plan_linear(kLinearGatedInput, false, rows, n_in, n_out, parts);
        const bool fits = gated.splits == 1 || sizeof(float) * gated.splits * rows * n_in <= parts;
        split += gated.splits > 1;
        if ((rc || bytes != up(sums) + up(parts) || !fits) && bad++ < 10)
            std::printf("%lld, %d -> %d: %zu bytes instead of %zu, %d parts through a gate of %zu\\n", rows, n_in, n_out, bytes, up(sums) + up(parts), gated.splits, parts);
    }
    std::printf("%d bad, %d split through a gate\\n", bad, split);
    return bad != 0 || split == 0;
}
"""


def test_a_backward_asks_for_its_own_parts(tmp_path):
    run_host_program(tmp_path, SWEEP)


@pytest.mark.parametrize("rows,n_in,n_out,most", [(487, 2752, 3936, 173312), (79, 152, 704, 8448), (32, 240, 784, 12544)])
def test_sizes_whose_gated_products_would_be_split(rows, n_in, n_out, most):
    assert terra.terra_linear_workspace_bytes(rows, n_in, n_out, "bwd") <= most
