"""What the binding passes on when a memory of streams is attached, without a GPU."""
import pytest

from paper_2505_23317_amd import cfdetr as K
from test_stream_memory_rules import _context


@pytest.mark.parametrize("given,passed", [(None, 2), (1, 1), (2, 2), (0, 0), (-1, -1)])
def test_number_of_key_heads(monkeypatch, given, passed):
    """None stands for the context's heads; every number goes to the library as it is, which refuses none and fewer."""
    calls = []
    enc = _context(monkeypatch, calls)
    enc.attach_memory(16, 10, 4, 5, given)
    assert calls[0][1].n_kv_heads == passed and enc.kv_dim == passed * enc.cfg.d_head
