"""The search of a sequence by its first row (csrc/ekv_search.h), compiled for the host with 64 lanes in turn and every access checked:
rows in front of the first entry, entries that do not ascend, one entry to more than two levels of 64."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_21649_amd", "csrc")
PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "ekv_search.h"
int main() {
  int n, v;
  while (std::scanf("%d %d", &n, &v) == 2) {
    std::vector<int> pre(n);
    for (int& x : pre) if (std::scanf("%d", &x) != 1) return 1;
    bool outside = false;
    const int got = ekv::last_at_most_by_64(n, [&](int lo, int left, int step) {
      int count = 0;
      for (int lane = 0; lane < 64; ++lane) {
        const int at = lane * step, i = lo + (at < left - 1 ? at : left - 1);      // every lane reads, as on the GPU
        if (i < 0 || i >= n) { outside = true; continue; }
        count += at < left && pre[i] <= v;
      }
      return count;
    });
    std::printf("%d %d\n", got, (int)outside);
  }
}
"""


@pytest.fixture(scope="module")
def search(tmp_path_factory):
    compiler = shutil.which("g++") or shutil.which("clang++")
    if compiler is None:
        pytest.skip("no host compiler")
    folder = tmp_path_factory.mktemp("search")
    source, program = folder / "search.cpp", folder / "search"
    source.write_text(PROGRAM)
    subprocess.run([compiler, "-std=c++17", "-O1", "-D__device__=", "-D__forceinline__=inline", "-I", CSRC, str(source), "-o", str(program)], check=True)

    def run(questions):
        text = "\n".join(f"{len(pre)} {v} " + " ".join(map(str, pre)) for pre, v in questions)
        out = subprocess.run([str(program)], input=text, capture_output=True, text=True, check=True, timeout=60).stdout.split()
        got = list(map(int, out[::2]))
        assert len(got) == len(questions) and not any(map(int, out[1::2])), "an access outside the entries"
        return got
    return run


SIZES = [1, 2, 3, 63, 64, 65, 127, 128, 200, 4096, 4097, 5000]


@pytest.mark.parametrize("n", SIZES)
def test_values_below_the_first_entry_give_the_first(search, n):
    pre = [18 + 3 * i for i in range(n)]
    assert search([(pre, v) for v in (-1 << 31, -1, 0, 17)] + [([18] * n, 0)]) == [0] * 5


@pytest.mark.parametrize("n", SIZES)
def test_the_last_entry_that_is_not_above_the_value(search, n):
    pre = [7 + 2 * (i // 3) for i in range(n)]               # entries come three times: the last one of them
    values = sorted({7, 8, pre[-1] - 1, pre[-1], pre[-1] + 100, pre[n // 2], pre[n // 3] + 1} & set(range(7, 1 << 20)))
    assert search([(pre, v) for v in values]) == [max(i for i in range(n) if pre[i] <= v) for v in values]


@pytest.mark.parametrize("n", SIZES)
def test_entries_that_do_not_ascend_give_an_entry(search, n):
    down, saw = [5 * (n - i) for i in range(n)], [(7919 * i) % 1009 - 300 for i in range(n)]
    for got in search([(pre, v) for pre in (down, saw) for v in (-1 << 31, -299, 0, 3, 200, 5 * n, (1 << 31) - 1)]):
        assert 0 <= got < n
