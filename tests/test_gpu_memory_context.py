"""What a context says of a memory of streams: its work space, and why it refuses rows."""
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


@pytest.mark.parametrize("d,streams", [(64, 1), (768, 4096)])
def test_work_space_counts_the_memory(K, d, streams):
    """A maximum and a sum, a row and a counter for every head of a stream's piece at least; what is refused adds nothing."""
    enc, heads = T.encoder(d, 8), T.MODELS[d]
    bare = K.cfdetr_workspace_bytes(enc.ctx)
    with pytest.raises(K.CfdetrError):
        enc.attach_memory(8, 10, 4, 5000)
    assert K.cfdetr_workspace_bytes(enc.ctx) == bare
    enc.attach_memory(8, 10, 4, streams)
    with_memory = K.cfdetr_workspace_bytes(enc.ctx)
    assert with_memory - bare >= streams * heads * (8 + 4 * (d // heads) + 4)
    with pytest.raises(K.CfdetrError):
        enc.attach_memory(8, 10, 4, streams)
    assert K.cfdetr_workspace_bytes(enc.ctx) == with_memory
    enc.close()


def test_work_space_counts_the_differential_layers(K):
    """Two positions of 4 bytes for every token."""
    import torch
    enc = T.encoder(64, 100)
    bare = K.cfdetr_workspace_bytes(enc.ctx)
    enc.attach_differential({"lambda": torch.zeros(1, 1).numpy()}, K.rotary_params(32))
    assert K.cfdetr_workspace_bytes(enc.ctx) - bare >= 100 * 8
    enc.close()


def test_rows_of_keys_are_refused_for_their_own_width(K):
    """The reason names no width that the rows need not have: a key row here is 32 wide, a query row 64."""
    import torch
    enc = T.encoder(64, 8)
    enc.attach_memory(8, 4, 4, 2, 1)
    x = torch.zeros(64, 64, device="cuda", dtype=torch.bfloat16)
    i = torch.zeros(64, dtype=torch.int32, device="cuda")
    p, n = x.data_ptr(), i.data_ptr()
    for call in (lambda: K.cfdetr_memory_attention(enc.ctx, p, 64, 2, p, 24, p, 32, n, n, None, 0.1, p, 64, enc._stream()),
                 lambda: K.cfdetr_memory_append(enc.ctx, None, None, None, None, 1, p, 24, p, 32, n, p, 32, p, 32, enc._stream())):
        with pytest.raises(K.CfdetrError) as e:
            call()
        assert e.value.status == K.CFDETR_EINVAL and "apart" in K.cfdetr_last_error(enc.ctx) and "d_model" not in K.cfdetr_last_error(enc.ctx)
    enc.sync_status()
    enc.close()
