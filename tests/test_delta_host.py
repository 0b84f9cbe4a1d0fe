"""What the gated delta rule's kernels compute about their rows, in a build of their headers for the host."""
import os
import subprocess

import pytest

from paper_2405_04416_amd import build

PROGRAM = r"""
#include "delta_common.h"
#include <cstdio>
#include <cstdlib>
int main(int, char **a)
{
    const dg_delta::Span span = {strtoull(a[1], 0, 0), (uint32_t)strtoull(a[2], 0, 0), atoi(a[3])};
    for (char **t = a + 4; *t; ++t) printf("%llu\n", (unsigned long long)span.row((uint32_t)strtoull(*t, 0, 0)));
}
"""


@pytest.fixture(scope="module")
def rows(tmp_path_factory):
    at = tmp_path_factory.mktemp("delta")
    (at / "rows.hip").write_text(PROGRAM)
    subprocess.run([build.hipcc(), "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-Wno-unused-command-line-argument", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                    str(at / "rows.hip"), "-o", str(at / "rows")], check=True, capture_output=True)
    return lambda *args: [int(x) for x in subprocess.run([str(at / "rows")] + [str(x) for x in args], check=True, capture_output=True, text=True).stdout.split()]


@pytest.mark.parametrize("length", [1, 2, 33, 1 << 20, (1 << 31) - 1, 1 << 31, (1 << 31) + 5, 3 << 30, (1 << 32) - 64])
@pytest.mark.parametrize("begin", [0, 7, 63])
def test_rows_of_a_sequence_of_any_length(rows, begin, length):
    tokens = sorted({t for t in (0, 1, length // 2, (1 << 31) - 1, 1 << 31, (1 << 31) + 1, length - 1) if t < length})
    assert rows(begin, length, 0, *tokens) == [begin + t for t in tokens]
    assert rows(begin, length, -1, *tokens) == [begin + length - 1 - t for t in tokens]
