"""The binding's checks of what it hands to the library, with tensors that only say what they are (no GPU)."""
import types

import pytest
import torch

from paper_2505_23317_amd import cfdetr as K


class Vector:
    """What the binding asks a tensor for."""

    def __init__(self, *shape, dtype=torch.float32, gpu=0):
        self.shape, self.dtype, self.gpu = torch.Size(shape), dtype, gpu

    def get_device(self):
        return self.gpu

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 4096


def _context(monkeypatch, gpu, d=64):
    enc = K.Encoder.__new__(K.Encoder)
    enc.cfg, enc.act_bf16, enc.act, enc.gpu, enc.ctx = types.SimpleNamespace(d=d), True, torch.bfloat16, gpu, None
    monkeypatch.setattr(K.Encoder, "_stream", staticmethod(lambda: 0))
    return enc


def _rows(gpu, d=64):
    return Vector(8, d, gpu=gpu), Vector(8, d, dtype=torch.bfloat16, gpu=gpu)


def test_vectors_are_checked_for_every_context(monkeypatch):
    """One parameter structure, used by contexts of the same width on two GPUs and by one of another width."""
    calls = []
    monkeypatch.setattr(K, "cfdetr_norm_residual", lambda *a: calls.append(a))
    params = K.norm_residual_params("rms", "none", post_g=Vector(64), gate=Vector(2, 64), cu_seqlens=Vector(3, dtype=torch.int32))
    first, other, wide = _context(monkeypatch, 0), _context(monkeypatch, 1), _context(monkeypatch, 0, 128)
    x, block = _rows(0)
    for _ in range(2):
        first.norm_residual(params, x, block, x)
        assert len(calls) == 1
        calls.clear()
        for enc, gpu, d in ((other, 1, 64), (wide, 0, 128)):
            x2, block2 = _rows(gpu, d)
            with pytest.raises(ValueError):
                enc.norm_residual(params, x2, block2, x2)
            assert not calls
