"""Attention over shared rows is as exact as attention that shares nothing: its weights keep 16 bits."""
import math

import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_attention import check, decode_error, rows
from test_gpu_attention_shared import CASES, shared

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,head_dim,page,groups,alone", CASES)
@pytest.mark.parametrize("bits", [16, 8])
def test_shared_rows_within_the_bound_of_single_ones(heads, kv_heads, head_dim, page, groups, alone, bits):
    s, of = shared(groups, kv_heads, head_dim, page, bits, heads + 100, alone)
    n = len(s.lens)
    q = rows(n, heads, head_dim, 3)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    got = B.attend_decode_shared(cache, batch, of, q, share_from=0)
    cache.check()
    check(got, *R.attend(s, q, [1] * n, **decode_error(bits)))


@pytest.mark.parametrize("apart", [0.003, 0.0017, 0.3])
@pytest.mark.parametrize("kv_heads,head_dim,own", [(1, 64, [256, 256]), (2, 128, [300, 257, 256] * 30)])
@pytest.mark.parametrize("bits", [16, 8])
def test_weights_that_nearly_cancel(apart, kv_heads, head_dim, own, bits):
    """Half of the shared keys weigh e^-apart times what the others do, and their values are -1 instead of 1: one rounding of the weights
    to bf16 (2^-8) is as much as what is left, and 16 times the bound."""
    s, of = shared([(256, own)], kv_heads, head_dim, 16, bits, 5)
    heads = 2 * kv_heads
    for pool in s.pools:
        pool.zero_()
    if bits == 8:
        for z in s.scales:
            z.fill_(1.0)
    # element 0 of a key is 1 where the value is -1, of a query -apart sqrt(head_dim) (times its scale: -apart)
    i = torch.arange(max(own), device="cuda")
    longest = own.index(max(own))
    for b in [longest] + [b for b in range(len(own)) if b != longest]:
        row = s.table[b].long()[i[:own[b]] // 16]
        s.pools[0][row, :, i[:own[b]] % 16, 0] = (i[:own[b]] % 2).to(s.pools[0].dtype)[:, None]
        s.pools[1][row, :, i[:own[b]] % 16, :head_dim] = (1 - 2 * (i[:own[b]] % 2)).to(s.pools[1].dtype)[:, None, None]
    q = torch.zeros(len(own), heads, head_dim, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = -apart * math.sqrt(head_dim)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)
    got = B.attend_decode_shared(cache, batch, of, q, share_from=0)
    cache.check()
    want, bound = R.attend(s, q, [1] * len(own), **decode_error(bits))
    check(got, want, bound)
    check(B.attend_decode(cache, batch, q), want, bound)
