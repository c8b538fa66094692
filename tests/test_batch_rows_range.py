"""Which rows the batch kernels take for a request's (rows_range.h): never one outside the batch, whatever row_start holds."""
import itertools
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_16162_amd", "csrc")

DRIVER = r'''
#include <cstdio>
#include <cstdlib>
#include "rows_range.h"
int main(int n, char **v) {
    for (int i = 1; i + 2 < n; i += 3) {
        const int row_start[3] = {-1, atoi(v[i]), atoi(v[i + 1])};
        const ks::RowsRange f = ks::rows_of(row_start, 1, atoi(v[i + 2]));
        printf("%d %d\n", f.first, f.n);
    }
}
'''


def test_rows_lie_in_the_batch(tmp_path):
    (tmp_path / "driver.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-I", CSRC, "-o", str(tmp_path / "driver"), str(tmp_path / "driver.cpp")], check=True)
    ends = [-2 ** 31, -2 ** 31 + 1, -2 ** 25, -9, -1, 0, 1, 5, 42, 43, 44, 2 ** 25 - 1, 2 ** 25, 2 ** 30, 2 ** 31 - 2, 2 ** 31 - 1]
    cases = list(itertools.product(ends, ends, (1, 43, 2 ** 25)))
    out = subprocess.run([str(tmp_path / "driver")] + [str(x) for c in cases for x in c], check=True, capture_output=True, text=True).stdout.split()
    got = list(zip(map(int, out[::2]), map(int, out[1::2])))
    assert len(got) == len(cases)
    for (a, b, n_rows), (first, n) in zip(cases, got):
        rows = range(max(a, 0), min(b, n_rows))
        assert n == len(rows), (a, b, n_rows)
        assert 0 <= first <= n_rows and first + n <= n_rows, (a, b, n_rows)
        assert not rows or first == rows[0], (a, b, n_rows)


def test_no_kernel_subtracts_the_starts_itself():
    for name in os.listdir(CSRC):
        text = open(os.path.join(CSRC, name)).read()
        assert name == "rows_range.h" or not re.search(r"row_start\[r \+ 1\]", text), name
