"""How many workgroups the kernels of a stream memory are launched with, without a GPU: rules of sizes, built for the host."""
import os
import shutil
import subprocess

import numpy as np
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


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    return built(tmp_path_factory, "cut", """
#include "stream_memory.h"
#include <cstdio>
#include <vector>
using namespace cfdetr;
int main() {
  int n, streams, places, least, whole;
  if (std::scanf("%d", &n) != 1) return 2;
  while (n--) {
    if (std::scanf("%d %d %d %d", &streams, &places, &least, &whole) != 4) return 2;
    std::vector<int> units(streams);
    int total = 0;
    for (int& u : units) {
      int first, held;
      if (std::scanf("%d %d", &first, &held) != 2) return 2;
      u = units_of(first, held);
      total += u;
    }
    const int length = cut_length(total, streams, places, least);
    std::printf("%d %d", most_pieces(streams, places), length);
    for (int u : units) std::printf(" %d %d", u, pieces_of(u, length, 1.0f / (float)length, whole));
    std::printf("\\n");
  }
}
""")


def _lengths(rng, streams, most):
    kind = rng.integers(0, 4)
    if kind == 0:
        return np.full(streams, most)
    if kind == 1:
        return rng.integers(0, most + 1, streams)
    if kind == 2:   # a few long ones among short ones
        return np.where(rng.random(streams) < 0.05, most, rng.integers(0, min(most, 700) + 1, streams))
    return np.exp(rng.uniform(0, np.log(most + 1), streams)).astype(np.int64)


def test_pieces_fit_their_room_and_cover_the_streams(cut):
    """Any streams, numbers of places (CUs over groups of slabs) and least lengths: no more pieces than the launch and the room have,
    every unit in one piece, no empty one, whole streams up to their limit."""
    rng = np.random.default_rng(5)
    rows, spans = [], []
    for streams in (1, 2, 3, 24, 63, 64, 65, 100, 127, 128, 129, 300, 1000, 4096):
        for places in (1, 2, 21, 42, 64, 85, 128, 256, 304):
            for least, whole in ((4, 10), (8, 20), (16, 40), (32, 80)):
                most = int(np.exp(rng.uniform(0, np.log(min(2 ** 29, 2 ** 34 // streams)))))   # (2^30 units in all)
                held = _lengths(rng, streams, most)
                first = rng.integers(0, 2 ** 29, streams)
                spans.append(np.stack([first, held], 1))
                rows.append([streams, places, least, whole, *spans[-1].ravel()])
    for span, row, (room, length, *got) in zip(spans, rows, cut(rows)):
        streams, places, least, whole = row[:4]
        units, pieces = np.asarray(got).reshape(streams, 2).T
        want = [len(range(f // 32, (f + h - 1) // 32 + 1)) if h else 0 for f, h in span]
        assert (units == want).all() and length >= least
        assert pieces.sum() <= room == streams + places
        assert (pieces[units == 0] == 0).all() and (pieces[(units > 0) & (units <= whole)] == 1).all()
        long = units > whole
        assert (pieces[long] * length >= units[long]).all() and ((pieces[long] - 1) * length < units[long]).all()
        if 2 * streams <= places and length > least:
            assert pieces.sum() <= places


def test_the_longest_stream(cut):
    """2^24 units and one more, which 32-bit floats round; every length round a power of two and the largest."""
    rows = []
    for held in (2 ** 29, 2 ** 29 - 1, 2 ** 29 - 31, 2 ** 28 + 1):
        for first in (0, 1, 31, 2 ** 29 - 1):
            for places in list(range(1, 260)) + [304, 1023]:
                rows.append([1, places, 4, 10, first, held])
    for row, (room, length, units, pieces) in zip(rows, cut(rows)):
        assert (pieces - 1) * length < units <= pieces * length and pieces <= room
