"""The norm - gate - residual step against its formula in 64 bits: every width, kind of norm, gate and type, ragged frames,
in place; and the refusals."""
import math

import pytest

import differential_reference as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_23317_amd import cfdetr
    cfdetr.load_library()
    return cfdetr


def _norm(v, kind, g, b, err):
    """(norm of the rows, bound of its error when the rows are off by err), 64 bits.

    32-bit sums over d <= 1024 columns go 16 columns a lane and six steps between lanes: 32 roundings at most for the mean,
    as many for the squares, and a few for the root and products.  An error e of the row moves its centred
    values by e and the mean of e, and its root by rms of that."""
    import torch
    if kind == "none":
        return v, err
    e = err + 40 * T.EPS32 * v.abs()
    if kind == "layer":
        e = e + err.mean(1, keepdim=True) + 40 * T.EPS32 * v.abs().mean(1, keepdim=True)
        v = v - v.mean(1, keepdim=True)
    r = torch.sqrt(v.square().mean(1, keepdim=True) + T.LN_EPS)
    e = (e + v.abs() * torch.sqrt(e.square().mean(1, keepdim=True)) / r + 48 * T.EPS32 * v.abs()) / r * g.double().abs()
    v = v / r * g.double()
    return (v + b.double(), e + 2 * T.EPS32 * (v.abs() + b.double().abs())) if b is not None else (v, e)


def _run(K, d, lengths, dtype, post, pre, gate, scale, tail=0):
    import torch
    rows = sum(lengths) + tail
    enc = T.encoder(d, rows, max(1, len(lengths)), dtype, heads=d // 32)
    x, block = T.normal(1, rows, d, std=2.0) + 0.5, (T.normal(2, rows, d, std=0.7) - 0.2).to(T.act(dtype))
    vec = {"post_g": 1 + T.normal(3, d, std=0.1) if post != "none" else None, "post_b": T.normal(4, d, std=0.1) if post == "layer" else None,
           "pre_g": 1 + T.normal(5, d, std=0.1) if pre != "none" else None, "pre_b": T.normal(6, d, std=0.1) if pre == "layer" else None}
    cu = T.offsets(lengths) if gate == "frame" else None
    gt = T.normal(7, len(lengths), d, std=0.3) if gate == "frame" else T.normal(7, d, std=0.3) if gate == "shared" else None
    params = K.norm_residual_params(post, pre, gate=gt, cu_seqlens=cu, res_scale=scale, **vec)
    x_out = torch.full((rows, d), 9.0, device="cuda")
    normed = torch.full((rows, d), 9.0, device="cuda").to(T.act(dtype)) if pre != "none" else None
    enc.norm_residual(params, x, block, x_out, normed)
    enc.sync_status()

    n = sum(lengths)
    zero = torch.zeros(n, d, dtype=torch.float64, device="cuda")
    y, err = _norm(block[:n].double(), post, vec["post_g"], vec["post_b"], zero)
    if gt is not None:
        gg = gt.double() if gate == "shared" else gt.double().repeat_interleave(torch.tensor(lengths, device="cuda"), dim=0)
        y, err = y * gg, err * gg.abs()
    want = scale * x[:n].double() + y
    err = 1.05 * err + 3 * T.EPS32 * (abs(scale) * x[:n].double().abs() + y.abs())
    T.within(x_out[:n], want, err, "x_out")
    if pre != "none":
        a, ea = _norm(want, pre, vec["pre_g"], vec["pre_b"], err)
        T.within(normed[:n], a, 1.05 * ea + T.HALF_STEP[dtype] * a.abs(), "normed")
    if tail:
        # behind the last frame
        assert (x_out[n:] == 9).all() and (normed is None or (normed[n:] == 9).all())
    # in place, the same bits
    x2, b2 = x.clone(), block.clone()
    enc.norm_residual(params, x2, b2, x2, b2 if normed is not None else None)
    assert torch.equal(x2[:n], x_out[:n]) and (normed is None or torch.equal(b2[:n], normed[:n]))
    assert torch.equal(x2[n:], x[n:]) and torch.equal(b2[n:], block[n:])
    enc.close()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("d", range(64, 1025, 64))
def test_every_width(K, d, dtype):
    _run(K, d, [13, 0, 58], dtype, "layer", "layer", "frame", 1.25)


@pytest.mark.parametrize("post", ("none", "layer", "rms"))
@pytest.mark.parametrize("pre", ("none", "layer", "rms"))
@pytest.mark.parametrize("gate", ("none", "shared", "frame"))
def test_every_form(K, post, pre, gate):
    _run(K, 256, [1, 66], "bf16", post, pre, gate, 1.0)


@pytest.mark.parametrize("d,lengths,tail", [(64, [1], 0), (384, [0, 3, 0, 0, 1, 0], 5), (768, [9001, 2, 11_000], 3), (320, [40_003], 0),
                                            (256, [2] * 64, 1), (64, [0, 0], 4)])
def test_rows(K, d, lengths, tail):
    """One row, empty frames in front and behind, more rows than workgroups, every frame there may be, rows behind the last."""
    _run(K, d, lengths, "bf16", "rms", "layer", "frame", 1.0, tail)


def test_no_numbers_stay_in_their_row(K):
    import torch
    enc = T.encoder(256, 64)
    x, block = T.normal(1, 64, 256), T.normal(2, 64, 256).bfloat16()
    block[5, 17], x[9, 0] = math.nan, math.inf
    g = torch.ones(256, device="cuda")
    x_out, normed = torch.empty_like(x), torch.empty_like(block)
    enc.norm_residual(K.norm_residual_params("rms", "rms", post_g=g, pre_g=g), x, block, x_out, normed)
    bad = (~torch.isfinite(normed)).any(1).nonzero().flatten().tolist()
    assert bad == [5, 9] and torch.isfinite(x_out[10:]).all()
    enc.close()


def test_bad_offsets_write_nothing(K):
    import torch
    enc = T.encoder(64, 32, 3)
    x, block = T.normal(1, 32, 64), T.normal(2, 32, 64).bfloat16()
    gate = T.normal(3, 3, 64)
    for cu in ([0, 5, 4, 32], [0, 5, 6, 33], [1, 5, 6, 32], [0, -1, 6, 32]):
        out = torch.full_like(x, 3.0)
        enc.norm_residual(K.norm_residual_params(gate=gate, cu_seqlens=torch.tensor(cu, dtype=torch.int32, device="cuda")), x, block, out)
        with pytest.raises(K.CfdetrError) as e:
            enc.sync_status()
        assert e.value.status == K.CFDETR_ECAPACITY and (out == 3).all()
    enc.sync_status()
    enc.close()


def test_refusals(K):
    import torch
    enc = T.encoder(64, 8, 2)
    x, b, g = torch.zeros(8, 64, device="cuda"), torch.zeros(8, 64, device="cuda").bfloat16(), torch.ones(2, 64, device="cuda")
    cu = torch.tensor([0, 3, 8], dtype=torch.int32, device="cuda")
    vec = torch.ones(64, device="cuda")

    def call(p, x_=x.data_ptr(), block=b.data_ptr(), out=x.data_ptr(), normed=b.data_ptr(), M=8):
        K.cfdetr_norm_residual(enc.ctx, p, x_, block, out, normed, M, enc._stream())

    def params(**kw):
        p = K.norm_residual_params("rms", "layer", post_g=vec, pre_g=vec, pre_b=vec, gate=g, cu_seqlens=cu)
        for k, v in kw.items():
            setattr(p, k, v)
        return p

    call(params())
    call(params(), M=0, x_=None, block=None, out=None, normed=None)
    for p, kw in ((params(post=7), {}), (params(pre=-1), {}), (params(post_g=None), {}), (params(post_b=vec.data_ptr()), {}),
                  (params(pre=0), {}), (params(pre=0, pre_g=None, pre_b=None), {}), (params(gate=None), {}), (params(B=0), {}),
                  (params(res_scale=math.nan), {}), (params(pre_g=vec.data_ptr() + 4), {}), (params(), dict(M=-1)), (params(), dict(x_=None)),
                  (params(), dict(block=None)), (params(), dict(out=None)), (params(), dict(normed=None)),
                  (params(), dict(block=b.data_ptr() + 2)), (params(gate=g.data_ptr() + 8), {})):
        with pytest.raises(K.CfdetrError) as e:
            call(p, **kw)
        assert e.value.status == K.CFDETR_EINVAL
    with pytest.raises(K.CfdetrError) as e:
        call(params(B=3))
    assert e.value.status == K.CFDETR_ECAPACITY
    for kw in (dict(gate=g[0], cu_seqlens=cu), dict(gate=g), dict(post="rms", post_g=vec[:32])):
        p = K.norm_residual_params(**kw)
        with pytest.raises(ValueError):
            enc.norm_residual(p, x, b, x)
    for bad in ((x.bfloat16(), b), (x, x), (x[:7], b), (x[:, ::2], b)):
        with pytest.raises(ValueError):
            enc.norm_residual(K.norm_residual_params(), bad[0], bad[1], x)
    enc.sync_status()
    enc.close()
