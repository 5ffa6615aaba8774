"""The memory of streams without a GPU: the arithmetic of a step, built for the host with the sanitizers and run over random
states in any order of its threads; sizes, tables of rotations and the binding's checks."""
import math
import os
import shutil
import subprocess
import types

import numpy as np
import pytest
import torch

import stream_memory_reference as R
from paper_2505_23317_amd import cfdetr as K

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_23317_amd", "csrc")

# A step as the kernel makes it: sums over the streams, then slots and page numbers one by one, in an order drawn here.
DRIVER = """
#include "stream_memory.h"
#include <cstdio>
#include <random>
#include <vector>
#include <algorithm>
#include <numeric>
using namespace cfdetr;
static int in() { int x; if (std::scanf("%d", &x) != 1) std::exit(2); return x; }
static std::vector<int> ins(size_t n) { std::vector<int> v(n); for (int& x : v) x = in(); return v; }
static void out(const std::vector<int>& v) { for (int x : v) std::printf("%d ", x); std::printf("\\n"); }
int main() {
  int cases = in();
  std::mt19937 order(1);
  while (cases--) {
    const int B = in(), bits = in(), cols = in(), n_pages = in(), apart = in();
    const auto span = ins(2 * B), drop = ins(B), fresh = ins(B);
    auto table = ins((size_t)B * cols);
    const auto pool = ins(2);
    auto free = ins(n_pages);
    std::vector<int> other((size_t)B * cols, -9), cu(B + 1), t0(B), g0(B), w0(B);
    std::vector<int>& to = apart ? other : table;
    std::vector<StreamStep> steps(B);
    int taken = 0, given = 0, work = 0;
    bool bad = false;
    for (int b = 0; b < B; ++b) {
      cu[b + 1] = cu[b] + std::max(0, fresh[b]);
      steps[b] = stream_step(span[2 * b], span[2 * b + 1], drop[b], fresh[b], bits, cols);
      bad |= steps[b].bad;
      t0[b] = taken; g0[b] = given; w0[b] = work;
      if (steps[b].bad) continue;
      taken += steps[b].taken; given += steps[b].given;
      work += steps[b].given + steps[b].taken + (apart ? steps[b].kept : 0);
    }
    const int head = pool[0], n_free = pool[1];
    if (bad || taken > n_free || given > n_pages - n_free) { std::printf("refused\\n"); continue; }
    auto place = [&](int i) { return i >= n_pages ? i - n_pages : i; };
    std::vector<int> slots(cu[B]), todo(cu[B] + work);
    std::iota(todo.begin(), todo.end(), 0);
    std::shuffle(todo.begin(), todo.end(), order);
    for (int i : todo) {
      if (i < cu[B]) {
        const int b = stream_of(cu, B, i);
        const StreamStep& s = steps[b];
        const int p = s.first + s.held + i - cu[b], page = p >> bits;
        const int id = page < s.have ? table.at((size_t)b * cols + ring_column(page, cols)) : free.at(place(head + t0[b] + page - s.have));
        slots.at(i) = (id << bits) | (p & ((1 << bits) - 1));
      } else {
        i -= cu[B];
        const int b = stream_of(w0, B, i);
        const PageWork w = page_work(steps[b], i - w0[b], cols);
        const size_t entry = (size_t)b * cols + w.column;
        if (w.given >= 0) free.at(place(head + n_free + g0[b] + w.given)) = table.at(entry);
        if (w.taken >= 0) to.at(entry) = free.at(place(head + t0[b] + w.taken));
        if (w.kept) to.at(entry) = table.at(entry);
      }
    }
    std::vector<int> spans(2 * B);
    for (int b = 0; b < B; ++b) { spans[2 * b] = steps[b].first; spans[2 * b + 1] = steps[b].held + fresh[b]; }
    std::printf("made\\n");
    out(slots); out(spans); out(to); out(free);
    out({place(head + taken), n_free - taken + given});
  }
}
"""


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host compiler")
    at = tmp_path_factory.mktemp("memory")
    (at / "driver.cc").write_text(DRIVER)
    cmd = [gxx, "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-static-libubsan",
           "-I", CSRC, str(at / "driver.cc"), "-o", str(at / "driver")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]

    def run(cases):
        text = f"{len(cases)} " + " ".join(" ".join(str(int(x)) for part in c for x in np.ravel(part)) for c in cases)
        r = subprocess.run([str(at / "driver")], input=text, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        return r.stdout.splitlines()

    return run


SHAPES = [(1, 8, 3, 2), (3, 8, 20, 4), (7, 16, 40, 6), (20, 8, 60, 1), (5, 1024, 9, 3), (64, 8, 500, 17)]


@pytest.mark.parametrize("streams,page,n_pages,cols", SHAPES)
def test_steps_against_pages_one_by_one(driver, streams, page, n_pages, cols):
    """Random steps in a row, in place and apart: slots, spans, tables, the ring; invariants behind every step."""
    rng = np.random.default_rng(streams)
    s, cases, wants = R.State(streams, page, n_pages, cols), [], []
    bits = page.bit_length() - 1
    for i in range(120):
        drop, new = R.random_step(rng, s, 2 * page)
        got = R.step(s, drop, new)
        cases.append((streams, bits, cols, n_pages, i % 2, s.span, drop, new, s.table, s.pool, s.free))
        if got is None:
            wants.append(None)
            continue
        after, slots = got
        after.check()
        held = [x for b in range(streams) for x in after.slots(b)]
        assert len(set(held)) == len(held) and set(slots) <= set(held)
        for b in range(streams):   # what is kept stays where it was
            left = max(0, int(s.span[b, 1]) - int(drop[b]))
            assert after.slots(b)[:left] == s.slots(b)[int(s.span[b, 1]) - left:]
        wants.append((after, slots, i % 2))
        s = after
    lines = iter(driver(cases))
    for want in wants:
        if want is None:
            assert next(lines) == "refused"
            continue
        after, slots, apart = want
        assert next(lines) == "made"
        got, span, table, free, pool = ([int(x) for x in next(lines).split()] for _ in range(5))
        assert got == slots and span == after.span.ravel().tolist() and pool == after.pool.tolist()
        table = np.asarray(table).reshape(streams, cols)
        for b in range(streams):
            for j in after.pages(b):
                assert table[b, j % cols] == after.table[b, j % cols]
        if apart:
            assert (table != -9).sum() == sum(len(after.pages(b)) for b in range(streams))
        else:
            assert (table == after.table).all()
        assert free == after.free.tolist()
    assert sum(w is not None for w in wants) > 20


@pytest.mark.parametrize("span,drop,fresh", [
    ((-1, 0), 0, 0), ((32, 1), 0, 0), ((0, -1), 0, 0), ((0, 33), 0, 0), ((1, 32), 0, 0), ((0, 8), -1, 0), ((0, 0), 0, -1), ((0, 0), 0, 33),
    ((0, 30), 0, 3), ((5, 27), 0, 1), ((2 ** 31 - 1, 2 ** 31 - 1), 0, 0), ((0, 0), 0, 2 ** 31 - 1), ((-2 ** 31, 2 ** 31 - 1), 2 ** 31 - 1, 1),
])
def test_steps_that_are_none(driver, span, drop, fresh):
    """Spans that no step leaves, and more than a ring of 4 pages of 8 holds: refused, with no number out of range."""
    assert driver([(1, 3, 4, 9, 0, span, [drop], [fresh], [0, 1, 2, 3], [0, 5], range(9))]) == ["refused"]


def test_the_largest_ring(tmp_path):
    """2^29 tokens in pages of 1024: positions go round without leaving 32 bits."""
    src = """
#include "stream_memory.h"
#include <cstdio>
#include <initializer_list>
using namespace cfdetr;
int main() {
  const int bits = 10, cols = (1 << 29) >> bits, ring = cols << bits;
  for (int first : {0, 1, ring / 2, ring - 1})
    for (int held : {0, 1, ring / 2, ring - (first & 1023)})
      for (int drop : {0, 1, held / 2, held, 0x7fffffff}) {
        const StreamStep s = stream_step(first, held, drop, 0, bits, cols);
        const int left = drop >= held ? 0 : held - drop;
        std::printf("%d %d %d %d %d %d %d %d %d\\n", first, held, drop, (int)s.bad, s.first, s.held, left, s.given + s.kept,
                    stream_step(first, held, drop, left + 1023 < ring ? ring - left - 1023 : 0, bits, cols).bad);
      }
}
"""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host compiler")
    (tmp_path / "ring.cc").write_text(src)
    subprocess.run([gxx, "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan", "-I", CSRC,
                    str(tmp_path / "ring.cc"), "-o", str(tmp_path / "ring")], check=True)
    lines = subprocess.run([str(tmp_path / "ring")], capture_output=True, text=True, check=True).stdout.splitlines()
    ring = 1 << 29
    assert len(lines) == 80
    for line in lines:
        first, held, drop, bad, to, now, left, pages, more = (int(x) for x in line.split())
        assert not bad and now == left and not more
        assert to == (0 if left == 0 else (first + drop) % ring)
        assert pages == (0 if held == 0 else (first + held - 1) // 1024 - first // 1024 + 1)


@pytest.mark.parametrize("sizes,good", [
    ((8, 1, 1, 1, 1, 8), True), ((1024, 2097151, 524288, 512, 8, 8), True), ((16, 100, 10, 4096, 2, 12), True),
    ((4, 1, 1, 1, 1, 8), False), ((2048, 1, 1, 1, 1, 8), False), ((24, 1, 1, 1, 1, 8), False), ((0, 1, 1, 1, 1, 8), False), ((-8, 1, 1, 1, 1, 8), False),
    ((8, 0, 1, 1, 1, 8), False), ((8, 1 << 28, 1, 1, 1, 8), False), ((1024, 2097152, 1, 1, 1, 8), False), ((8, 1, 0, 1, 1, 8), False),
    ((8, 1, (1 << 26) + 1, 1, 1, 8), False), ((8, 1, 1, 0, 1, 8), False), ((8, 1, 1, 4097, 1, 8), False), ((8, 1, 1 << 17, 4096, 1, 8), False),
    ((8, 1, 1, 1, 0, 8), False), ((8, 1, 1, 1, 3, 8), False), ((8, 1, 1, 1, 16, 8), False), ((8, 1, 1, 1, -1, 8), False),
])
def test_sizes(tmp_path, sizes, good):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host compiler")
    (tmp_path / "s.cc").write_text('#include "stream_memory.h"\nint main() { return cfdetr::check_memory_sizes(%d, %d, %d, %d, %d, %d) != nullptr; }' % sizes)
    subprocess.run([gxx, "-std=c++17", "-I", CSRC, str(tmp_path / "s.cc"), "-o", str(tmp_path / "s")], check=True)
    assert (subprocess.run([str(tmp_path / "s")]).returncode == 0) == good


@pytest.mark.parametrize("rot_dim,pairs", [(32, (4, 6, 6)), (64, (8, 12, 12)), (16, (8,)), (64, (1, 1, 29, 1)), (48, (12, 12)), (32, (14, 1, 1))])
@pytest.mark.parametrize("in_turn", (False, True))
@pytest.mark.parametrize("shared", (False, True))
def test_tables_of_rotations(rot_dim, pairs, in_turn, shared):
    freq, axis = K.cfdetr_rotary_axes_table(K.rotary_axes_params(rot_dim, pairs, in_turn, shared, base=500.0))
    want_axis, want = R.axes_table(pairs, in_turn, shared, 500.0)
    assert axis == want_axis and np.allclose(freq, want, rtol=1e-15, atol=0)
    if len(pairs) == 1:
        plain = K.cfdetr_rotary_frequencies(K.rotary_params(rot_dim, 1, base=500.0))
        assert np.allclose(freq, plain, rtol=1e-15, atol=0)


def test_tables_that_are_none():
    good = dict(rot_dim=32, pairs=(4, 6, 6))
    for bad in (dict(rot_dim=24), dict(rot_dim=0), dict(rot_dim=80, pairs=(20, 20)), dict(pairs=(4, 6, 5)), dict(pairs=(16, 0)), dict(pairs=(17, -1)),
                dict(pairs=(2 ** 31 - 1, 2 ** 31 - 1, 2)), dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(in_turn=2),
                dict(shared_ladder=3), dict(interleaved=2)):
        with pytest.raises(K.CfdetrError) as e:
            K.cfdetr_rotary_axes_table(K.rotary_axes_params(**dict(good, **bad)))
        assert e.value.status == K.CFDETR_EINVAL
    for pairs in ((), (4, 4, 4, 2, 2)):
        with pytest.raises(ValueError):
            K.rotary_axes_params(32, pairs)
    assert K.load_library().cfdetr_rotary_axes_table(None, None, None) == K.CFDETR_EINVAL


def test_without_a_context():
    lib, mem, axes = K.load_library(), K.CfdetrMemoryConfig(16, 4, 4, 1, 1), K.rotary_axes_params(32, (4, 6, 6))
    assert lib.cfdetr_memory_attach(None, mem) == K.CFDETR_EINVAL
    assert lib.cfdetr_memory_advance(None, 1, *[None] * 2, 0, *[None] * 9) == K.CFDETR_EINVAL
    assert lib.cfdetr_rotary_axes(None, axes, None, None, None, 1, None, 64, None, 64, 1.0, None, 0, None, 0, 0, None) == K.CFDETR_EINVAL
    assert lib.cfdetr_memory_append(None, axes, None, None, None, 1, None, 64, None, 64, None, None, 64, None, 64, None) == K.CFDETR_EINVAL
    assert lib.cfdetr_memory_attention(None, None, 64, 1, None, 64, None, 64, None, None, None, 0.0, None, 64, None) == K.CFDETR_EINVAL


class Tensor:
    """What the binding asks a tensor for."""

    def __init__(self, *shape, dtype=torch.int32, gpu=0, stride=None):
        self.shape, self.dtype, self.gpu = torch.Size(shape), dtype, gpu
        self.steps = stride or ((shape[1], 1) if len(shape) == 2 else (1,))

    def get_device(self):
        return self.gpu

    def is_contiguous(self):
        return len(self.shape) == 1 or self.steps == (self.shape[1], 1)

    def stride(self):
        return self.steps

    def data_ptr(self):
        return 4096


def _context(monkeypatch, calls):
    enc = K.Encoder.__new__(K.Encoder)
    enc.cfg, enc.act, enc.gpu, enc.ctx = types.SimpleNamespace(d=64, d_head=32, heads=2), torch.bfloat16, 0, None
    for name in ("attach", "advance", "append", "attention"):
        monkeypatch.setattr(K, "cfdetr_memory_" + name, lambda *a: calls.append(a))
    monkeypatch.setattr(K, "cfdetr_rotary_axes", lambda *a: calls.append(a))
    monkeypatch.setattr(K.Encoder, "_stream", staticmethod(lambda: 0))
    return enc


def test_the_binding_checks_tensors(monkeypatch):
    """Every argument with another type, shape, device or distance of rows is refused before the library is called."""
    calls = []
    enc = _context(monkeypatch, calls)
    act = torch.bfloat16
    bf = lambda *shape, **kw: Tensor(*shape, dtype=act, **kw)
    params, table = K.rotary_axes_params(32, (4, 6, 6)), dict(freq=Tensor(16, dtype=torch.float64), axis=Tensor(16, dtype=torch.uint8),
                                                              pos=Tensor(3, 3, dtype=torch.float32))
    for call in (lambda: enc.memory_advance(*[Tensor(1)] * 6), lambda: enc.memory_append(*[bf(1, 32)] * 5), lambda: enc.memory_attention(*[bf(1, 64)] * 6),
                 lambda: enc.alloc_memory(1)):
        with pytest.raises(ValueError):   # (no memory yet)
            call()
    enc.attach_memory(16, 10, 4, 5, 1)
    calls.clear()
    good = {
        enc.memory_advance: dict(cu_new=Tensor(4), span=Tensor(3, 2), table=Tensor(3, 4), pool=Tensor(2), free_pages=Tensor(10), slots=Tensor(7),
                                 drop=Tensor(3), span_out=Tensor(3, 2), table_out=Tensor(3, 4), pool_out=Tensor(2)),
        enc.rotary_axes: dict(params=params, **table, q=bf(3, 64), q_out=bf(3, 64), k=bf(3, 32), k_out=bf(3, 32)),
        enc.memory_append: dict(k=bf(3, 32), v=bf(3, 32), slots=Tensor(3), k_cache=bf(160, 32), v_cache=bf(160, 32), params=params, **table),
        enc.memory_attention: dict(q=bf(3, 64), k_cache=bf(160, 32), v_cache=bf(160, 32), span=Tensor(3, 2), table=Tensor(3, 4), out=bf(3, 64),
                                   key_mask=Tensor(160, dtype=torch.uint8)),
    }
    for call, kw in good.items():
        call(**kw)
        assert len(calls) == 1
        for name, t in kw.items():
            if name == "params":
                continue
            shape = tuple(t.shape)
            others = [Tensor(*shape, dtype=torch.float16), Tensor(*shape, dtype=t.dtype, gpu=1), Tensor(*shape, dtype=t.dtype, gpu=-1)]
            if not (call == enc.memory_advance and name == "slots"):
                others.append(Tensor(shape[0] + 1, *shape[1:], dtype=t.dtype))
            if len(shape) == 2:
                others += [Tensor(shape[0], shape[1] + 1, dtype=t.dtype), Tensor(*shape, dtype=t.dtype, stride=(2 * shape[1], 2))]
            for other in others:
                with pytest.raises(ValueError):
                    call(**dict(kw, **{name: other}))
        calls_now = len(calls)
        assert calls_now == 1
        calls.clear()
    with pytest.raises(ValueError):
        enc.rotary_axes(**dict(good[enc.rotary_axes], k_out=None))
    with pytest.raises(ValueError):
        enc.memory_append(**dict(good[enc.memory_append], params=None))
    for empty in ("freq", "axis", "pos"):
        with pytest.raises((ValueError, AttributeError)):
            enc.memory_append(**dict(good[enc.memory_append], **{empty: None}))
    assert not calls
