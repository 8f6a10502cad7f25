"""What the products' kernels rely on beyond their arguments, checked without a GPU."""
from tests._host_program import run_host_program


def test_no_bias_may_be_read_as_vectors(tmp_path):
    # products without a bias read zeros from a global of the library, 16 bytes at a time and 16 of 64 columns from any 16th on
    out = run_host_program(tmp_path, """
#include "block_kernels.h"
int main() { std::printf("%zu %zu", alignof(NoBias), sizeof(NoBias::values)); }
""")
    align, size = map(int, out.split())
    assert align % 16 == 0 and size == 64 * 4
