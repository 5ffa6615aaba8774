"""How exact the operators of a stream memory are, against the formulas in 64 bits: weights of shared key heads, logits of any
size, rotations in the check mode."""
import math

import numpy as np
import pytest

import differential_reference as T
import stream_memory_reference as R
from test_gpu_memory_attention import Case
from test_gpu_memory_rows import _positions, _table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_23317_amd import cfdetr
    cfdetr.load_library()
    return cfdetr


@pytest.mark.parametrize("d,kv,page", [(64, 1, 8), (256, 4, 16), (256, 1, 16), (384, 2, 32), (768, 4, 64), (768, 1, 64), (1024, 8, 64)])
def test_weights_of_shared_key_heads(K, d, kv, page):
    """Values of one sign, so that nothing cancels: a row is off by its own rounding to bf16 and by what 32 bits lose.

    Bound.  A weight w goes into the matrix product as h + l, h = w rounded to bf16 and l = w - h (a number of 32 bits)
    rounded to bf16: off by 2^-8 2^-8 w at most, so a row by 2^-16 sum p |v|.  Two products a token are added in 32 bits where the
    bound of the reference has one: n 2^-24 sum p |v| more.  The rest is that of the reference with weights in 32 bits.
    """
    case = Case(d, kv, [2, 3, 5, 9, 40, 333, 2, 700], page, "bf16")
    case.v.abs_()
    got = case.run()
    want, off = R.attention(case.q, case.k, case.v, case.slots, case.heads, kv, "f32")   # (rows: values are their own size)
    n = max(len(s) for s in case.slots)
    off = off + want * (2.0 ** -16 + n * T.EPS32)
    T.within(got, want, off + T.HALF_STEP["bf16"] * (want + off), "rows")
    case.enc.sync_status()
    case.enc.close()


@pytest.mark.parametrize("d,kv,dtype", [(256, 8, "bf16"), (256, 4, "bf16"), (384, 2, "bf16"), (768, 1, "bf16"), (64, 2, "f32"), (384, 2, "f32"), (768, 2, "f32")])
@pytest.mark.parametrize("exponent", (14, 20, 28))
def test_logits_past_a_billion(K, d, kv, dtype, exponent):
    """Logits of 2^28 to 2^56, thousands and more apart: a row is the value of the token with the largest, bit by bit, wherever that is.

    Queries are 2^exponent and one feature makes the difference: the logit of a key is its first feature times 2^exponent times the
    scale.  The largest key has 3/2 of 2^exponent there, the others -1 to 1 of it: products and sums are exact in 32 bits but for
    the scale, and e to the differences is 0.
    """
    import torch
    lengths = [1, 40, 700, 700, 9000]
    case = Case(d, kv, lengths, 16, dtype, std=1.0)
    dh, group = d // case.heads, case.heads // kv
    big = 2.0 ** exponent
    case.q.zero_()
    case.q[:, ::dh] = big
    top = [0, 39, 0, 350, 8000]
    for b, (slots, t) in enumerate(zip(case.slots, top)):
        at = torch.as_tensor(slots, device="cuda")
        first = (torch.rand(len(slots), kv, generator=torch.Generator(device="cuda").manual_seed(b), device="cuda") * 2 - 1) * big
        first[t] = 1.5 * big
        for h in range(kv):
            case.k[at, h * dh] = first[:, h].to(T.act(dtype))
    got = case.run()
    for b, (slots, t) in enumerate(zip(case.slots, top)):
        want = case.v[slots[t]].view(kv, 1, dh).expand(kv, group, dh).reshape(d)
        assert torch.equal(got[b], want), (b, exponent)
    case.enc.sync_status()
    case.enc.close()


def _in_32_bits(x, pos, axis, freq, heads, interleaved):
    """Features turned by sines and cosines rounded to 32 bits: b s rounded, a c added to it and rounded once."""
    import torch
    rows, n = x.shape[0], len(axis)
    y = x.reshape(rows, heads, -1).clone()
    angle = pos.double()[:, torch.tensor(axis, device=x.device)] * torch.tensor(freq, dtype=torch.float64, device=x.device)
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    i = torch.arange(n, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
    a, b = y[..., ia], y[..., ib]
    y[..., ia], y[..., ib] = (a.double() * c.double() - (b * s).double()).float(), (a.double() * s.double() + (b * c).double()).float()
    return y.reshape(rows, -1)


@pytest.mark.parametrize("d,kv,pairs,interleaved,far", [(64, 1, (4, 6, 6), False, 160), (384, 2, (8, 12, 12), True, 4000), (768, 12, (4, 6, 6), True, 1_000_003),
                                                        (768, 4, (32,), False, 16_000_000)])
def test_rotation_in_the_check_mode(K, d, kv, pairs, interleaved, far):
    """fp32: sine and cosine are those of the angle, rounded to 32 bits; the rest is one product and one fused multiply-add.

    Bound, relative to a pair's length: sine and cosine half a step each, 2^-24 of the length together (|a c| + |b s| is at most the
    length), 2^-24 for the product and 2^-24 for the sum; second orders, a thousandth.  The angle: five roundings in 64
    bits on either side (frequency, product, turns) of at most `far` radians.
    Bits: those of the same two operations on the rounded sines and cosines, which 64 bits hold but for a bit that decides a tie
    in one of 2^28: what differs is what the angle's last 64 bits move over a border of 32, 5 far 2^-53 of 2^-24 radians.
    """
    import torch
    rows = 400
    enc, heads = T.encoder(d, 8, dtype="f32"), T.MODELS[d]
    kd = d // heads * kv
    params = K.rotary_axes_params(2 * sum(pairs), pairs, False, False, interleaved)
    axis, freq = R.axes_table(pairs, False, False)
    pos = _positions(rows, len(pairs), far, 1)
    qk = T.normal(2, rows, d + kd)
    out = torch.empty_like(qk)
    enc.rotary_axes(params, *_table(K, params), pos, qk[:, :d], out[:, :d], qk[:, d:], out[:, d:])
    for x, got, n in ((qk[:, :d], out[:, :d], heads), (qk[:, d:], out[:, d:], kv)):
        want, size = R.turned(x, pos, axis, freq, n, interleaved)
        T.within(got, want, size * (3.003 * T.EPS32 + 5 * far * 2.0 ** -53), "features")
        same = _in_32_bits(x, pos, axis, freq, n, interleaved)
        assert (got != same).double().mean() < 1e-4 + 40 * far * 2.0 ** -29
    cache = torch.empty(rows // 8 * 8, kd, device="cuda"), torch.empty(rows // 8 * 8, kd, device="cuda")
    enc.attach_memory(8, rows // 8, 4, 1, kv)
    slots = torch.arange(rows, dtype=torch.int32, device="cuda")
    enc.memory_append(qk[:, d:], qk[:, d:], slots, *cache, params, *_table(K, params), pos)
    assert torch.equal(cache[0], out[:, d:]) and torch.equal(cache[1], qk[:, d:])   # the same bits as the rotation's
    enc.close()
