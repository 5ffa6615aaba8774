"""The cases of a stream memory as a program makes them: contexts for sizes and not for inputs."""
import random
import types

import pytest
import torch

from paper_2505_23317_amd import cfdetr, synth
from perf import more_operators as M


class Context:
    def __init__(self, log, cfg, weights, act_dtype, **kw):
        self.log, self.sizes, self.memory = log, (cfg.d, cfg.heads, act_dtype), None
        log.append(self)

    def attach_memory(self, *a, **kw):
        assert self.memory is None
        self.memory = a + tuple(kw.values())


@pytest.fixture
def made(monkeypatch):
    log = []
    monkeypatch.setattr(cfdetr, "Encoder", lambda cfg, w, **kw: Context(log, cfg, w, **kw))
    monkeypatch.setattr(synth, "make_weights", lambda *a: {})
    monkeypatch.setattr(M, "torch", types.SimpleNamespace(tensor=lambda x, **kw: list(x), float64=0, uint8=1))
    monkeypatch.setattr(cfdetr, "cfdetr_rotary_axes_table", lambda p: (log.append("table"), [1.0], [0])[1:])
    for f in (M._context, M._rotation):
        monkeypatch.setattr(f, "__defaults__", ({},))
    return log


def _state(case, n_pages=100, cols=9):
    s = {"case": case, "input": object()}
    if case["op"] != "rotary":
        s["n_pages"] = n_pages
    if case["op"] in ("advance", "attention"):
        s["cols"] = cols
    return s


def test_inputs_of_one_case_share_a_context(made):
    """... and nothing else: a second set of inputs makes no encoder, no memory, no table, and no state holds another's tensors."""
    for case in M.listed():
        made.clear()
        first, second = _state(case), _state(case)
        M._own_state(case, first)
        count = len(made)
        M._own_state(case, second)
        assert len(made) == count <= 2 and first["enc"] is second["enc"]
        assert first["input"] is not second["input"]
        assert not any(isinstance(x, torch.Tensor) for x in vars(first["enc"]).values())


def test_other_sizes_have_another(made):
    rng = random.Random(3)
    seen = {}
    for case in M.listed() + [M.draw(rng) for _ in range(40)]:
        for pages in (100, 101):
            s = _state(case, pages)
            M._own_state(case, s)
            enc = s["enc"]
            assert enc.sizes == (case.get("width", 256), case.get("heads", 8), case.get("dtype", "bf16"))
            if case["op"] == "rotary":
                assert enc.memory is None
                continue
            assert enc.memory == (case["page"], pages, s.get("cols", 1), case.get("streams", 1), case.get("key_heads"))
            assert seen.setdefault((enc.sizes, enc.memory), enc) is enc
    assert len(set(map(id, seen.values()))) == len(seen)
