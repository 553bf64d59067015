"""From which size on rows are shared when the caller leaves it to the library, over bf16 and over 8-bit caches."""
import pytest
import torch

from paper_2402_17764_b200 import binding as B
from test_gpu_attention import rows
from test_gpu_attention_shared import shared

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,span,shares", [(16, 256, False), (16, 384, True), (8, 384, False), (8, 448, False), (8, 576, True)])
def test_the_bound_of_each_kind_of_cache(bits, span, shares):
    """130 sequences at 8 heads of 128: 34, 51, 60 and 77 M elements of keys (the bounds: 42 M for bf16, 67 M for codes)."""
    s, of = shared([(span, [span + 1 + i % 5 for i in range(130)])], 8, 128, 64, bits, 1)
    q = rows(130, 16, 128, 2)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    apart, together = B.attend_decode(cache, batch, q), B.attend_decode_shared(cache, batch, of, q, share_from=0)
    assert not torch.equal(apart, together)
    assert torch.equal(B.attend_decode_shared(cache, batch, of, q), together if shares else apart)
    cache.check()
