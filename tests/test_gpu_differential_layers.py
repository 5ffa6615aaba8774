"""The operators together: as a run of calls, captured and replayed, on another stream, and as the encoder's own layers in every one
of its passes, against the oracle."""
import numpy as np
import pytest

import differential_reference as T
from oracle import cfdetr_oracle as O
from oracle import differential_oracle as D
from paper_2505_23317_amd import synth

pytestmark = pytest.mark.gpu

BAR = {"bf16": 2e-2, "f32": 1e-4}   # the framework's bars of an encoder pass, relative to the largest value


@pytest.fixture(scope="module")
def K():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2505_23317_amd import cfdetr
    cfdetr.load_library()
    return cfdetr


def _weights(cfg, seed, parts):
    rng = np.random.default_rng(seed)
    w = {"lambda": rng.uniform(0.2, 0.9, (cfg.layers, cfg.heads // 2)).astype(np.float32)}
    for name, n in (("head_g", 2 * cfg.d_head), ("post1_g", cfg.d), ("post2_g", cfg.d), ("gate1", cfg.d), ("gate2", cfg.d)):
        if name.rstrip("_g") in parts or name in parts:
            w[name] = (0.5 + 0.1 * rng.standard_normal((cfg.layers, n))).astype(np.float32)
    return w


ALL = ("head_g", "post1_g", "post2_g", "gate1", "gate2")
CFGS = {
    64: synth.Config("diff64", 3, 64, 96, (16, 8), 64, 2, 2, 128, "bf16", box_rule="poisson", box_lambda=2.0, side_lo=8, side_hi=40),
    256: synth.Config("diff256", 2, 128, 96, (16, 8), 256, 8, 2, 512, "bf16", box_rule="poisson", box_lambda=2.0, side_lo=8, side_hi=60),
    384: synth.Config("diff384", 2, 96, 160, (32, 16, 8), 384, 6, 3, 768, "bf16", box_rule="tiered", box_lambda=3.0, side_lo=8, side_hi=60),
    768: synth.Config("diff768", 2, 64, 64, (16, 8), 768, 12, 1, 1536, "bf16", box_rule="poisson", box_lambda=1.0, side_lo=8, side_hi=40),
}


def _rel(got, want):
    return float(np.abs(got.cpu().numpy() - want).max() / np.abs(want).max())


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
@pytest.mark.parametrize("d,parts,interleaved,scale", [(64, ALL, False, 1.0), (256, ALL, True, 1.0), (384, ALL, False, 1.5), (768, ("head_g",), False, 1.0),
                                                       (256, (), False, 1.0)])
def test_every_pass_of_the_encoder(K, d, parts, interleaved, scale, dtype):
    import torch
    cfg = CFGS[d]
    wl = synth.make_workload(cfg, seed=3)
    w = synth.make_weights(cfg, 4, sharp=True)
    diff = _weights(cfg, 5, parts)
    rot = K.rotary_params(cfg.d_head, 2, interleaved, base=100.0)
    freq = D.rotary_frequencies(cfg.d_head, 2, base=100.0)
    enc = K.Encoder(cfg, w, act_dtype=dtype)
    enc.attach_differential(diff, rot, scale)
    img = enc.upload_images(wl["images"])
    boxes = enc.upload_boxes(wl["boxes"], wl["tier"], wl["box_offsets"])
    out = enc.alloc_outputs(cfg.B)
    enc.multilevel_batch(img, cfg.B, *boxes, out)
    enc.sync_status()
    rows, cols = cfg.grid(0)
    grid = np.asarray([(0, r, c) for r in range(rows) for c in range(cols)] * cfg.B)
    tok, cu, _ = O.select_fine(wl["boxes"], wl["tier"], wl["box_offsets"], cfg.B, cfg.H, cfg.W, cfg.patch)
    args = (cfg.patch, w, diff, cfg.heads, freq, interleaved, scale)
    coarse = D.fine_encode(wl["images"], grid, np.arange(cfg.B + 1) * rows * cols, *args)
    mixed = D.fine_encode(wl["images"], tok, cu, *args)
    n = int(cu[-1])
    e0, e1 = _rel(out["y_coarse"], coarse), _rel(out["y_mixed"][:n], mixed)
    print(f"{d} {dtype}: coarse {e0:.2e} mixed {e1:.2e}", flush=True)
    assert e0 <= BAR[dtype] and e1 <= BAR[dtype]
    assert not out["y_mixed"][n:].any()
    # the single calls, and the padded form: the sums of a query may be split otherwise, so the bar again
    one = enc.alloc_outputs(cfg.B)
    enc.coarse_encode(img, cfg.B, one["x0_cache"], one["y_coarse"])
    enc.select_fine(*boxes, cfg.B, one["tok_desc"], one["cu_seqlens"])
    enc.fine_encode(img, cfg.B, one["tok_desc"], one["cu_seqlens"], one["x0_cache"], one["y_mixed"])
    longest = max(int(np.diff(cu).max()), cfg.n_cells(0))
    padded = torch.zeros(cfg.B * longest, cfg.d, device="cuda")
    enc.fine_encode_padded(img, cfg.B, one["tok_desc"], one["cu_seqlens"], one["x0_cache"], longest, padded)
    enc.sync_status()
    assert _rel(one["y_coarse"], coarse) <= BAR[dtype] and _rel(one["y_mixed"][:n], mixed) <= BAR[dtype]
    for f in range(cfg.B):
        a, b = int(cu[f]), int(cu[f + 1])
        assert _rel(padded[f * longest:f * longest + b - a], mixed[a:b]) <= BAR[dtype]
    # the operators change the result: plain layers with the same matrices are elsewhere
    plain = K.Encoder(cfg, w, act_dtype=dtype)
    plain.coarse_encode(img, cfg.B, one["x0_cache"], one["y_coarse"])
    plain.sync_status()
    assert _rel(one["y_coarse"], coarse) > 2 * BAR[dtype]
    plain.close()
    enc.close()


def test_as_many_cameras_as_there_may_be(K):
    """The merged run then has 128 sequences."""
    cfg = synth.replace(CFGS[64], B=64, H=32, W=32, layers=1)
    wl = synth.make_workload(cfg, seed=8)
    w, diff = synth.make_weights(cfg, 4, sharp=True), _weights(cfg, 5, ALL)
    enc = K.Encoder(cfg, w)
    enc.attach_differential(diff, K.rotary_params(32))
    out = enc.alloc_outputs(64)
    enc.multilevel_batch(enc.upload_images(wl["images"]), 64, *enc.upload_boxes(wl["boxes"], wl["tier"], wl["box_offsets"]), out)
    enc.sync_status()
    tok, cu, _ = O.select_fine(wl["boxes"], wl["tier"], wl["box_offsets"], 64, 32, 32, cfg.patch)
    mixed = D.fine_encode(wl["images"], tok, cu, cfg.patch, w, diff, 2, D.rotary_frequencies(32, 2))
    assert _rel(out["y_mixed"][:int(cu[-1])], mixed) <= BAR["bf16"]
    enc.close()


def _chain(K, d, lengths, dtype):
    """Rotation in place, attention and the step behind it on a context, as a program strings them together."""
    import torch
    rows, heads = sum(lengths), T.MODELS[d]
    enc = T.encoder(d, rows, len(lengths), dtype)
    rot = K.rotary_params(d // heads)
    s = dict(enc=enc, heads=heads, lengths=lengths, rot=rot, cu=T.offsets(lengths),
             freq=torch.tensor(K.cfdetr_rotary_frequencies(rot), dtype=torch.float64, device="cuda"),
             pos=torch.rand(rows, 2, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * 100,
             qkv=T.normal(2, rows, 3 * d).to(T.act(dtype)), lam=torch.full((heads // 2,), 0.4, device="cuda"),
             g=torch.ones(2 * d // heads, device="cuda"), x=T.normal(3, rows, d), o=torch.empty(rows, d, device="cuda").to(T.act(dtype)),
             x_out=torch.empty(rows, d, device="cuda"), normed=torch.empty(rows, d, device="cuda").to(T.act(dtype)),
             turned=torch.empty(rows, 2 * d, device="cuda").to(T.act(dtype)))
    gain = torch.ones(d, device="cuda")
    s["norm"] = K.norm_residual_params("rms", "layer", post_g=gain, pre_g=gain, pre_b=gain, gate=0.5 * gain)
    return s


def _call(s):
    d = s["x"].shape[1]
    qkv, t, enc = s["qkv"], s["turned"], s["enc"]
    enc.rotary(s["rot"], s["freq"], s["pos"], qkv[:, :d], t[:, :d], qkv[:, d:2 * d], t[:, d:], q_scale=T.log2e_over(d // s["heads"]))
    enc.diff_attention(t[:, :d], t[:, d:], qkv[:, 2 * d:], s["cu"], s["cu"], s["lam"], s["o"], s["g"], s.get("mask"), softmax_scale=0.0)
    enc.norm_residual(s["norm"], s["x"], s["o"], s["x_out"], s["normed"])


def _expected(s, dtype):
    """The chain in 64 bits, from the rounded rotation on."""
    d = s["x"].shape[1]
    n = s["lengths"]
    o, bound = T.diff_attention(s["turned"][:, :d], s["turned"][:, d:], s["qkv"][:, 2 * d:], n, n, s["heads"], s["lam"], s["g"], dtype, np.log(2.0))
    T.within(s["o"], o, bound)
    o = s["o"].double()
    x = s["x"].double() + 0.5 * o / (o.square().mean(1, keepdim=True) + T.LN_EPS).sqrt()
    return x


@pytest.mark.parametrize("d,lengths,dtype", [(256, [400, 1, 33, 777], "bf16"), (384, [129, 64], "bf16"), (64, [50], "f32")])
def test_a_run_of_them(K, d, lengths, dtype):
    import torch
    s = _chain(K, d, lengths, dtype)
    _call(s)
    s["enc"].sync_status()
    want, size = T.turned(s["qkv"][:, :d], s["pos"], s["freq"], s["heads"], False)
    scale = T.log2e_over(d // s["heads"])
    T.within(s["turned"][:, :d], want * scale, (want.abs() * T.HALF_STEP[dtype] + size * 2.0 ** -20) * scale * 1.001)
    x = _expected(s, dtype)
    # 32-bit norm of at most 384 columns: 64 roundings
    T.within(s["x_out"], x, 64 * T.EPS32 * (s["x"].double().abs() + (x - s["x"].double()).abs() + 1e-3))
    s["enc"].close()


@pytest.mark.parametrize("d,lengths,masked", [(256, [400, 1, 33, 777], False), (384, [65, 2100], True)])
def test_captured_and_replayed(K, d, lengths, masked):
    """Every replay against the eager result, with new inputs, eager calls and waits between them."""
    import torch
    s = _chain(K, d, lengths, "bf16")
    if masked:
        s["mask"] = (torch.rand(sum(lengths), device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)) > 0.4).to(torch.uint8)
    _call(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _call(s)
    for i in range(4):
        s["qkv"].copy_(T.normal(20 + i, *s["qkv"].shape).bfloat16())
        if masked and i % 2:
            s["mask"].fill_(1)
        _call(s)
        torch.cuda.synchronize()
        want = [s[k].clone() for k in ("turned", "o", "x_out", "normed")]
        for k in ("turned", "o", "x_out", "normed"):
            s[k].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k, w in zip(("turned", "o", "x_out", "normed"), want):
            assert torch.equal(s[k], w), (i, k)
    s["enc"].sync_status()
    s["enc"].close()


def test_two_graphs_of_one_context(K):
    """They share its work space (partial results, key lists): replayed in turn, with another mask and other runs each."""
    import torch
    pool = T.encoder(256, 9000, 3)
    states, graphs, wants = [], [], []
    for nq, nk, share in (([3, 1, 2], [4000, 1500, 3500], 0.4), ([40, 0, 5], [600, 2100, 5000], 0.8)):
        g = torch.Generator(device="cuda").manual_seed(sum(nq))
        s = dict(q=T.normal(5, sum(nq), 256).bfloat16(), kv=T.normal(6, sum(nk), 512).bfloat16(), cu_q=T.offsets(nq), cu_k=T.offsets(nk),
                 lam=torch.full((4,), 0.4, device="cuda"), mask=(torch.rand(sum(nk), device="cuda", generator=g) > share).to(torch.uint8),
                 out=torch.empty(sum(nq), 256, device="cuda").bfloat16())

        def call(s=s):
            pool.diff_attention(s["q"], s["kv"][:, :256], s["kv"][:, 256:], s["cu_q"], s["cu_k"], s["lam"], s["out"], key_mask=s["mask"])

        call()
        torch.cuda.synchronize()
        wants.append(s["out"].clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        states.append(s)
        graphs.append(graph)
    for i in range(6):
        for j in (0, 1) if i % 2 else (1, 0):
            states[j]["out"].zero_()
            graphs[j].replay()
        torch.cuda.synchronize()
        for s, w in zip(states, wants):
            assert torch.equal(s["out"], w)
    pool.sync_status()
    pool.close()


def test_another_stream(K):
    """The calls go to the current stream, behind what it holds."""
    import torch
    s = _chain(K, 256, [900, 33], "bf16")
    _call(s)
    torch.cuda.synchronize()
    want, qkv = s["x_out"].clone(), s["qkv"].clone()
    s["qkv"].zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(4):
            big = big @ big * 1e-3
        s["qkv"].copy_(qkv)
        _call(s)
    side.synchronize()
    assert torch.equal(s["x_out"], want)
    s["enc"].close()


def test_operators_beside_the_encoder(K):
    """On one context the operators leave the passes' results as they are, and the other way round."""
    import torch
    cfg = CFGS[256]
    wl, w = synth.make_workload(cfg, seed=3), synth.make_weights(cfg, 4)
    enc = K.Encoder(cfg, w)
    img, boxes = enc.upload_images(wl["images"]), enc.upload_boxes(wl["boxes"], wl["tier"], wl["box_offsets"])
    first, second = enc.alloc_outputs(2), enc.alloc_outputs(2)
    enc.multilevel_batch(img, 2, *boxes, first)
    s = _chain(K, 256, [40, 50], "bf16")
    s["enc"].close()
    s["enc"] = enc
    s["mask"] = torch.ones(90, dtype=torch.uint8, device="cuda")
    _call(s)
    want = s["normed"].clone()
    enc.multilevel_batch(img, 2, *boxes, second)
    _call(s)
    enc.sync_status()
    for k in ("y_coarse", "y_mixed", "tok_desc", "cu_seqlens"):
        assert torch.equal(first[k], second[k])
    assert torch.equal(s["normed"], want)
    enc.close()


def test_tensors_of_another_gpu(K):
    """They are refused; the context's number is changed, so that one GPU is enough."""
    import torch
    s = _chain(K, 256, [40, 50], "bf16")
    s["enc"].gpu += 1
    with pytest.raises(ValueError):
        _call(s)
    p = K.norm_residual_params("rms", "none", post_g=torch.ones(256, device="cuda"))
    x = torch.zeros(3, 256, device="cuda")
    with pytest.raises(ValueError):
        s["enc"].norm_residual(p, x, x.bfloat16(), x)
    s["enc"].gpu -= 1
    _call(s)
    s["enc"].close()


def test_attach_refusals(K):
    import ctypes
    cfg = synth.replace(CFGS[64], B=1)
    enc = K.Encoder(cfg, synth.make_weights(cfg, 1))
    diff = _weights(cfg, 5, ALL)
    for bad, rot, scale in (({"lambda": None}, {}, 1.0), ({"post1_g": None}, {}, 1.0), ({"gate2": None}, {}, 1.0), ({}, dict(rot_dim=48), 1.0),
                            ({}, dict(n_axes=1), 1.0), ({}, dict(base=0.5), 1.0), ({}, {}, float("nan"))):
        kept = {k: v for k, v in dict(diff, **bad).items() if v is not None}
        with pytest.raises(K.CfdetrError) as e:
            enc.attach_differential(kept, K.rotary_params(**dict(dict(rot_dim=32), **rot)), scale)
        assert e.value.status == K.CFDETR_EINVAL
    for bad in ({"post1": diff["post1_g"]}, {"lambda": diff["lambda"][:1]}, {"gate1": diff["gate1"][:, :32]}, {"head_g": diff["head_g"][0]}):
        with pytest.raises(ValueError):
            enc.attach_differential(dict(diff, **bad), K.rotary_params(32))
    enc.attach_differential(diff, K.rotary_params(32))
    with pytest.raises(K.CfdetrError):
        enc.attach_differential(diff, K.rotary_params(32))
    enc.close()
    odd = T.encoder(192, 8, heads=3)
    with pytest.raises(K.CfdetrError) as e:
        K.cfdetr_differential_attach(odd.ctx, K.CfdetrDifferentialWeights())
    assert e.value.status == K.CFDETR_ESHAPE
    assert K.load_library().cfdetr_differential_attach(odd.ctx, None) == K.CFDETR_EINVAL
    assert K.load_library().cfdetr_differential_attach(None, ctypes.byref(K.CfdetrDifferentialWeights())) == K.CFDETR_EINVAL
    odd.close()
