"""What the products' kernels rely on beyond their arguments, checked without a GPU."""
import os
import re

import pytest

from paper_2608_15211_b200 import binding
from paper_2608_15211_b200.build import CSRC, build
from tests._host_program import run_host_program


def test_no_bias_may_be_read_as_vectors(tmp_path):
    # products without a bias read zeros from a global of the library, 16 bytes at a time and 16 of 64 columns from any 16th on
    out = run_host_program(tmp_path, """
#include "block_kernels.h"
int main() { std::printf("%zu %zu", alignof(NoBias), sizeof(NoBias::values)); }
""")
    align, size = map(int, out.split())
    assert align % 16 == 0 and size == 64 * 4


@pytest.mark.parametrize("name", ["linear.cu", "linear_few.cu", "linear_aux.cu", "norm.cu", "rotary.cu"])
def test_dependent_launches_read_by_plain_loads(name):
    # a kernel that may be resident while the launch before it still writes must not promise the compiler that what it reads stays as it is
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert "__ldg" not in code and ".global.nc" not in code
    kernels = re.findall(r"__global__[^;{]*?(\w+_kernel)\s*\(([^{;]*)\)\s*\{", code)
    assert kernels
    for kernel, arguments in kernels:
        assert "__restrict__" not in arguments, kernel


def test_a_missing_workspace_names_every_call_that_asks_for_one():
    build()
    lib = binding.load_library()
    text = lib.terra_strerror(4).decode()
    assert all(n in text for n in binding.EXPORTS if n.endswith("_workspace_bytes"))
