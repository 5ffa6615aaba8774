"""Rotary positions against the formula in 64 bits: both layouts, parts of a head, one and two axes, far positions,
rows apart, in place, queries alone; and the refusals."""
import math

import pytest

import differential_reference as T

pytestmark = pytest.mark.gpu

# What a feature may be off, relative to its pair's length: the angle's last 32 bits (half a step of half a turn, in
# radians: 2^-25 2 pi < 2^-22), sine, cosine, two products and a sum in 32 bits (4 units), the scale (1).
PAIR = 2.0 ** -22 + 8 * T.EPS32


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_23317_amd import cfdetr
    cfdetr.load_library()
    return cfdetr


def _positions(rows, axes, far, seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(0, far, (rows, axes), generator=g, device="cuda").float() + (0.5 if far < 1000 else 0.0)


CASES = [
    # d, rows, dtype, rot_dim, axes, interleaved, far
    (64, 1, "bf16", 32, 2, False, 160), (64, 67, "f32", 16, 1, True, 100), (256, 300, "bf16", 32, 2, False, 160),
    (256, 17, "bf16", 16, 2, True, 160), (384, 1001, "bf16", 64, 2, True, 160), (384, 5, "f32", 48, 2, False, 160),
    (768, 129, "bf16", 32, 1, False, 16_000_000), (768, 40, "f32", 64, 1, True, 1_000_003), (1024, 33, "bf16", 48, 1, False, 4000),
    (1024, 9, "f32", 64, 2, False, 160),
]


@pytest.mark.parametrize("d,rows,dtype,rot_dim,axes,interleaved,far", CASES)
def test_against_the_formula(K, d, rows, dtype, rot_dim, axes, interleaved, far):
    import torch
    enc, heads = T.encoder(d, rows, dtype=dtype), T.MODELS[d]
    params = K.rotary_params(rot_dim, axes, interleaved, factor=2.0, trained_len=512.0 if rows % 2 else 0.0)
    freq = torch.tensor(K.cfdetr_rotary_frequencies(params), dtype=torch.float64, device="cuda")
    pos = _positions(rows, axes, far, 1)
    qkv = T.normal(2, rows, 3 * d).to(T.act(dtype))
    q, k = qkv[:, :d], qkv[:, d:2 * d]
    out = torch.full((rows + 2, 2 * d + 64), 7.0, device="cuda").to(T.act(dtype))   # rows apart, others around them
    enc.rotary(params, freq, pos, q, out[1:-1, :d], k, out[1:-1, d:2 * d], q_scale=T.log2e_over(d // heads))
    for x, got, scale in ((q, out[1:-1, :d], T.log2e_over(d // heads)), (k, out[1:-1, d:2 * d], 1.0)):
        want, size = T.turned(x, pos, freq, heads, interleaved)
        T.within(got, want * scale, (want.abs() * T.HALF_STEP[dtype] + size * PAIR) * scale * 1.001, "features")
    assert (out[0] == 7).all() and (out[-1] == 7).all() and (out[:, 2 * d:] == 7).all()
    # features behind the rotated ones are as they were
    if rot_dim < d // heads:
        assert torch.equal(out[1:-1, d:2 * d].view(rows, heads, -1)[..., rot_dim:], k.reshape(rows, heads, -1)[..., rot_dim:])
    # in place, and queries alone, the same bits
    own = qkv.clone()
    enc.rotary(params, freq, pos, own[:, :d], own[:, :d], own[:, d:2 * d], own[:, d:2 * d], q_scale=T.log2e_over(d // heads))
    assert torch.equal(own[:, :2 * d], out[1:-1, :2 * d]) and torch.equal(own[:, 2 * d:], qkv[:, 2 * d:])
    alone = torch.empty(rows, d, device="cuda").to(T.act(dtype))
    enc.rotary(params, freq, pos, q, alone, q_scale=T.log2e_over(d // heads))
    assert torch.equal(alone, out[1:-1, :d])
    enc.close()


def test_many_rows(K):
    """More rows than one round of workgroups, the last one ragged; a row's result does not depend on the others."""
    import torch
    rows, d = 20_011, 256
    enc = T.encoder(d, rows)
    params = K.rotary_params(32)
    freq = torch.tensor(K.cfdetr_rotary_frequencies(params), dtype=torch.float64, device="cuda")
    pos, x = _positions(rows, 2, 160, 5), T.normal(6, rows, d).bfloat16()
    out = torch.empty_like(x)
    enc.rotary(params, freq, pos, x, out)
    want, size = T.turned(x, pos, freq, 8, False)
    T.within(out, want, want.abs() * T.HALF_STEP["bf16"] + size * PAIR)
    part = torch.empty_like(x[:7])
    enc.rotary(params, freq, pos[20_000:20_007], x[20_000:20_007], part)
    assert torch.equal(part, out[20_000:20_007])
    enc.close()


def test_values_that_are_no_numbers_stay_in_their_pair(K):
    import torch
    enc = T.encoder(64, 4)
    params = K.rotary_params(32)
    freq = torch.tensor(K.cfdetr_rotary_frequencies(params), dtype=torch.float64, device="cuda")
    x = T.normal(1, 4, 64).bfloat16()
    x[1, 3], x[2, 40] = math.nan, math.inf
    out = torch.empty_like(x)
    enc.rotary(params, freq, _positions(4, 2, 160, 1), x, out)
    bad = ~torch.isfinite(out)
    assert bad.sum() == 4 and bad[1, 3] and bad[1, 19] and bad[2, 40] and bad[2, 56]
    enc.close()


def test_refusals(K):
    import torch
    enc = T.encoder(64, 8)
    params = K.rotary_params(32)
    freq, pos = torch.ones(16, dtype=torch.float64, device="cuda"), torch.zeros(8, 2, device="cuda")
    x = torch.zeros(8, 80, device="cuda", dtype=torch.bfloat16)
    p, ld = x.data_ptr(), 80

    def call(params=params, freq=freq.data_ptr(), pos=pos.data_ptr(), M=8, q=p, q_ld=ld, qo=p, qo_ld=ld, scale=1.0, k=None, k_ld=0,
             ko=None, ko_ld=0):
        K.cfdetr_rotary(enc.ctx, params, freq, pos, M, q, q_ld, qo, qo_ld, scale, k, k_ld, ko, ko_ld, enc._stream())

    call()
    call(M=0, q=None, qo=None, freq=None, pos=None)
    for kw in (dict(params=K.rotary_params(48)), dict(params=K.rotary_params(8)), dict(params=K.rotary_params(32, 3)), dict(freq=None),
               dict(pos=None), dict(M=-1), dict(q=None), dict(q=p + 2), dict(q_ld=60), dict(qo_ld=84), dict(scale=math.inf), dict(k=p),
               dict(k=p, k_ld=ld, ko=p, ko_ld=ld + 8), dict(k=p, k_ld=63, ko=p, ko_ld=ld), dict(freq=freq.data_ptr() + 4)):
        with pytest.raises(K.CfdetrError) as e:
            call(**kw)
        assert e.value.status == K.CFDETR_EINVAL and K.cfdetr_last_error(enc.ctx)
    for bad in (dict(q=x[:, :64].float()), dict(q=x[:, :60]), dict(pos=pos[:7]), dict(freq=freq.float())):
        kw = dict(dict(freq=freq, pos=pos, q=x[:, :64]), **bad)
        with pytest.raises(ValueError):
            enc.rotary(params, kw["freq"], kw["pos"], kw["q"], x[:, :64])
    enc.sync_status()
    enc.close()
