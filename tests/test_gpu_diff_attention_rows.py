"""A row of the differential attention belongs to its query alone: the bits of one do not change with the queries beside it."""
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


@pytest.mark.parametrize("d,nq,nk,dtype,level", [
    (256, [40, 7], [2000, 333], "bf16", 0.0), (384, [33], [1500], "bf16", 0.0), (64, [50, 3], [700, 65], "f32", 0.0),
    (384, [20], [900], "f32", 0.0), (256, [1500] * 4, [1500] * 4, "bf16", 400.0), (384, [3000] * 4, [700] * 4, "bf16", 400.0),
])
def test_neighbours_do_not_show(K, d, nq, nk, dtype, level):
    """Every other query is replaced by one whose logits spread over hundreds, so that their largest one moves in many units.
    `level`: about what all logits of the others are before the scale; 400 (144 in powers of two) is past what the kernel of many queries holds
    without a running maximum."""
    import torch
    heads, dh = T.MODELS[d], d // T.MODELS[d]
    q = T.normal(1, sum(nq), d, std=1.5)
    k, v = T.normal(2, sum(nk), d, std=1.5), T.normal(3, sum(nk), d)
    q.view(-1, heads, dh)[:, :, 0], k.view(-1, heads, dh)[:, :, 0] = level / 8.0, 8.0
    q, k, v = (x.to(T.act(dtype)) for x in (q, k, v))
    lam = torch.full((heads // 2,), 0.5, device="cuda")
    enc = T.encoder(d, max(sum(nq), sum(nk)), len(nq), dtype)
    outs = []
    for steep in (False, True):
        x = q.clone()
        if steep:
            x[::2] = 40 * T.normal(4, len(x[::2]), d, std=1.5).to(T.act(dtype))
        out = torch.empty_like(q)
        enc.diff_attention(x, k, v, T.offsets(nq), T.offsets(nk), lam, out, softmax_scale=0.25)
        enc.sync_status()
        outs.append(out[1::2])
    assert torch.isfinite(outs[0]).all()
    differ = int((outs[0] != outs[1]).any(1).sum())
    assert torch.equal(*outs), f"{differ} of {len(outs[0])} rows differ"
    enc.close()


@pytest.mark.parametrize("norm", (False, True))
@pytest.mark.parametrize("d,nq,nk,dtype", [
    (256, [40, 7], [300, 33], "bf16"), (64, [5, 2], [70, 33], "f32"),                    # in one run
    (384, [1], [9000], "bf16"), (64, [3], [6000], "f32"), (256, [3, 2], [4000, 900], "bf16"),   # in several, joined
    (256, [3000] * 2, [300, 77], "bf16"), (384, [6000] * 2, [300, 77], "bf16"),          # many queries
])
def test_lambda_zero_leaves_the_first_map(K, d, nq, nk, dtype, norm):
    """Keys and a query that are no numbers in the second map only: nothing of it is in the rows of a head whose lambda is 0, and
    everything is lost in those of the head that has another."""
    import math
    import torch
    heads, dh = T.MODELS[d], d // T.MODELS[d]
    q, k, v = T.normal(1, sum(nq), d), T.normal(2, sum(nk), d), T.normal(3, sum(nk), d)
    for h in range(heads // 2):
        second = slice((2 * h + 1) * dh, (2 * h + 2) * dh)
        k[3, second], k[20, second], k[nk[0] - 1, second] = math.nan, math.inf, -math.inf
        q[0, second] = math.nan
    q, k, v = (x.to(T.act(dtype)) for x in (q, k, v))
    lam = torch.zeros(heads // 2, device="cuda")
    lam[1:] = 0.5
    g = torch.ones(2 * dh, device="cuda") if norm else None
    out = torch.empty_like(q)
    enc = T.encoder(d, max(sum(nq), sum(nk)), len(nq), dtype)
    enc.diff_attention(q, k, v, T.offsets(nq), T.offsets(nk), lam, out, g)
    enc.sync_status()
    first = [x.clone() for x in (q, k)]
    for x in first:
        x[:, dh:2 * dh] = 0
    want, bound = T.diff_attention(*(x[:, :2 * dh] for x in first), v[:, :2 * dh], nq, nk, 2, lam[:1], g, dtype)
    T.within(out[:, :2 * dh], want, bound, f"{d} {nq} {nk}")
    if heads > 2:
        assert torch.isnan(out[:nq[0], 2 * dh:]).all() and torch.isfinite(out[nq[0]:, 2 * dh:]).all()
    enc.close()


@pytest.mark.parametrize("nq,dtype,level", [(4200, "bf16", 0.0), (4200, "f32", 0.0), (16_400, "bf16", 200.0), (1, "bf16", 0.0)])
def test_sums_at_the_limit_of_values_and_keys(K, nq, dtype, level):
    """Values times keys just below 2^110, and nearly every logit 15.75 above those of the first keys, which is as far as the
    reference of the weights lags: sums of 2^125.  Every value is the same c, so a row is (1 - lambda) c: the weights of either
    map are summed twice, in the row and in the divisor, each n roundings of 2^-24 at most and in bf16 half a step of each weight."""
    import math
    import torch
    nk, c = 70_001, 1.4375 * 2.0 ** 93
    assert 0.5 < nk * c / 2.0 ** 110 < 1.0
    q, k, v = (torch.zeros(n, 64, device="cuda") for n in (nq, nk, nk))
    for first in (0, 32):
        q[:, first:first + 2] = 1.0
        k[:, first], k[256:, first + 1] = level, 15.75
    v[:] = c
    out = torch.empty(nq, 64, device="cuda").to(T.act(dtype))
    enc = T.encoder(64, nk, 1, dtype)
    q, k, v = (x.to(T.act(dtype)) for x in (q, k, v))
    enc.diff_attention(q, k, v, T.offsets([nq]), T.offsets([nk]), torch.full((1,), 0.25, device="cuda"), out, softmax_scale=math.log(2.0))
    enc.sync_status()
    u = T.HALF_STEP["bf16"] if dtype == "bf16" else 0.0
    assert torch.isfinite(out).all()
    off = (out.double() - 0.75 * c).abs().max().item()
    assert off <= 1.25 * (u + 2 * nk * T.EPS32) * c + T.HALF_STEP[dtype] * c, off / c
    enc.close()


@pytest.mark.parametrize("norm", (False, True))
@pytest.mark.parametrize("noise", (0.07, 0.02))
@pytest.mark.parametrize("d,nq,nk,dtype", [
    (384, [300], [1600], "bf16"), (384, [1], [9000], "bf16"), (256, [3000, 2500], [1600, 333], "bf16"), (384, [6000], [1600], "bf16"),
    (384, [40], [1600], "f32"),
])
def test_maps_that_are_nearly_alike(K, d, nq, nk, dtype, noise, norm):
    """The second map's queries and keys are the first's and a little noise, lambda is 0.9: the maps' products with the values are
    many times their difference.  The bound counts the rounding of the weights relative to the products."""
    import torch
    heads, dh = T.MODELS[d], d // T.MODELS[d]
    q, k, v = T.normal(1, sum(nq), d), T.normal(2, sum(nk), d), T.normal(3, sum(nk), d)
    for x, seed in ((q, 4), (k, 5)):
        maps = x.view(len(x), heads // 2, 2, dh)
        maps[:, :, 1] = maps[:, :, 0] + noise * T.normal(seed, len(x), heads // 2, dh)
    q, k, v = (x.to(T.act(dtype)) for x in (q, k, v))
    lam, g = torch.full((heads // 2,), 0.9, device="cuda"), torch.ones(2 * dh, device="cuda") if norm else None
    out = torch.empty_like(q)
    enc = T.encoder(d, max(sum(nq), sum(nk)), len(nq), dtype)
    enc.diff_attention(q, k, v, T.offsets(nq), T.offsets(nk), lam, out, g)
    enc.sync_status()
    want, bound = T.diff_attention(q, k, v, nq, nk, heads, lam, g, dtype)
    worst = T.within(out, want, bound, f"{d} {nq} {nk}")
    off = (out.double() - want).square().mean().sqrt() / want.square().mean().sqrt()
    print(f"{dtype}, noise {noise}: off by {off.item():.2e} of the rows' size, {worst:.3f} of the bound", flush=True)
    enc.close()
