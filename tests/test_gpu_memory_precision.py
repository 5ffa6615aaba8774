"""How exact the operators of a stream memory are, against the formulas in 64 bits: weights of shared key heads."""
import pytest

import differential_reference as T
import stream_memory_reference as R
from test_gpu_memory_attention import Case

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
