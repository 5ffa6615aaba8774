"""How many workgroups the kernels of a stream memory are launched with, without a GPU: rules of sizes, built for the host."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_23317_amd", "csrc")


def built(tmp_path_factory, name, source):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host compiler")
    at = tmp_path_factory.mktemp(name)
    (at / "d.cc").write_text(source)
    cmd = [gxx, "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-static-libubsan",
           "-I", CSRC, str(at / "d.cc"), "-o", str(at / "d")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]

    def run(rows):
        text = "\n".join(" ".join(str(int(x)) for x in r) for r in [[len(rows)], *rows])
        r = subprocess.run([str(at / "d")], input=text, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        return [[int(x) for x in line.split()] for line in r.stdout.splitlines()]

    return run


@pytest.fixture(scope="module")
def advance(tmp_path_factory):
    return built(tmp_path_factory, "advance", """
#include "stream_memory.h"
#include <cstdio>
int main() {
  int n, v[7];
  if (std::scanf("%d", &n) != 1) return 2;
  while (n--) {
    for (int& x : v) if (std::scanf("%d", &x) != 1) return 2;
    const cfdetr::AdvanceLaunch l = cfdetr::advance_launch(v[0], v[1], v[2], v[3], v[4] != 0, v[5] != 0, v[6]);
    std::printf("%d %d\\n", l.chunk, l.grid);
  }
}
""")


def test_steps(advance):
    """Enough workgroups for two rounds of slots' and page numbers each, or one a CU; one where there is little to do."""
    rows = [(n_new, streams, cols, n_pages, forgets, apart, cus)
            for n_new in (0, 1, 512, 513, 10 ** 5, 131_072, 131_073, 2 ** 30) for streams in (1, 300, 4096) for cols in (1, 64, 65_536)
            for n_pages in (1, 4096, 10 ** 6, 2 ** 27) for forgets in (0, 1) for apart in (0, 1) for cus in (80, 256)]
    for (n_new, streams, cols, n_pages, forgets, apart, cus), (chunk, grid) in zip(rows, advance(rows)):
        assert 1 <= grid <= cus and chunk == (4 if n_new > 512 * cus else 1)
        # a table in place keeps what it keeps: only what is given back (at most the pages that there are) has to be done
        numbers = streams * cols if apart else min(streams * cols, n_pages) if forgets else 0
        need = max(-(-n_new // (512 * chunk)), -(-numbers // 1024), 1)
        assert grid == min(cus, need)


def test_pages_given_back_in_place_have_workgroups(advance):
    """One stream of 200,000 tokens in pages of 8, 300 tracks: not one workgroup for tens of rounds."""
    assert [g for _, g in advance([(1, 1, 30_000, 25_100, 1, 0, 256), (300, 300, 64, 13_800, 1, 0, 256), (1024, 1024, 128, 98_256, 1, 0, 256)])] == [25, 14, 96]
    assert [g for _, g in advance([(1, 4, 16, 100_000, 1, 0, 256), (6, 6, 170, 100_000, 1, 0, 256), (300, 300, 64, 13_800, 0, 0, 256)])] == [1, 1, 1]
