"""Attention over the paged cache where one key takes all (scores of any size) and where a value is infinite."""
import math

import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_attention import QUERY_FIXED, rows

# heads, kv_heads, head_dim, page, new, past: every width of a cache row and every page size, whole tiles and parts of them;
# the last two are split among several CTAs
SHAPES = [
    (8, 1, 128, 64, [129, 1, 64], [0, 1000, 63]),
    (4, 4, 64, 256, [257, 3], [0, 300]),
    (6, 3, 100, 16, [37, 200], [411, 0]),
    (2, 2, 20, 32, [300], [0]),
    (12, 2, 80, 128, [130], [7]),
    (5, 1, 112, 16, [90, 33, 2], [0, 15, 16]),
    (3, 3, 48, 64, [100], [300]),
    (16, 8, 64, 32, [20, 20], [2100, 1300]),
    (4, 4, 128, 16, [60], [2500]),
]


def winners(s, q, counts, query_rounding):
    """(value, decided): of every token and head the value of the key with the largest score, in 64 bits, and whether it
    wins by so much that all other weights count as zero.

    A score, in fp32, is off by at most (D + 4) 2^-24 scale sum_i |q_i k_i| (kv_reference.attend), and by scale query_rounding
    max_i |q_i| sum_i |k_i| where the queries are rounded.  2^x is zero below 2^-150, e^-104; with twice the error of
    two scores on top, 110 + 4 error is enough.
    """
    T, H, D = q.shape
    G, scale = H // s.kv_heads, 1.0 / math.sqrt(D)
    value = torch.zeros(T, H, D, dtype=torch.float64, device=q.device)
    decided = torch.zeros(T, H, dtype=torch.bool, device=q.device)
    at = 0
    for b, n in enumerate(counts):
        L = s.lens[b]
        x = q[at:at + n].double().reshape(n, s.kv_heads, G, D).permute(1, 2, 0, 3)
        k, v = s.rows(0, b, L), s.rows(1, b, L)
        score = scale * torch.einsum("hgnd,hld->hgnl", x, k)
        off = (D + 4) * 2.0 ** -24 * scale * torch.einsum("hgnd,hld->hgnl", x.abs(), k.abs())
        off = off + query_rounding * scale * x.abs().amax(-1)[..., None] * k.abs().sum(-1)[:, None, None]
        hidden = torch.arange(L, device=q.device)[None] > (L - n + torch.arange(n, device=q.device))[:, None]
        score, off = score.masked_fill(hidden, -math.inf), off.masked_fill(hidden, 0.0).amax(-1)
        best = score.argmax(-1)
        top = score.gather(-1, best[..., None])[..., 0]
        second = score.scatter(-1, best[..., None], -math.inf).amax(-1)
        y = v[:, None, None].expand(-1, G, n, -1, -1).gather(3, best[..., None, None].expand(-1, -1, -1, 1, D))[:, :, :, 0]
        value[at:at + n] = y.permute(2, 0, 1, 3).reshape(n, H, D)
        decided[at:at + n] = (top - second > 110.0 + 4.0 * off).permute(2, 0, 1).reshape(n, H)
        at += n
    return value, decided


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv_heads,head_dim,page,new,past", SHAPES)
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("prompt", [False, True])
def test_one_key_takes_all_at_scores_of_any_size(heads, kv_heads, head_dim, page, new, past, bits, prompt):
    """Queries and keys of 30 to 2^56 times the usual size: scores of a thousand to 10^34.  The winner's value is the result: its
    weight, rounded to bf16 (2^-8) by the prompt kernel, and the result's rounding (2^-8); exponentials, sums and the
    division are off by less than 2^-18 together."""
    lens = [n + p for n, p in zip(new, past)]
    counts = new if prompt else [1] * len(new)
    T = sum(counts)
    s = R.Setup(lens, kv_heads, head_dim, page, bits, seed=61)
    cu = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")
    attend = B.attend_prompt if prompt else B.attend_decode
    base_k = s.pools[0].clone() if bits == 16 else s.scales[0].clone()
    for size in (30.0, 1000.0, 12000.0, 1e5, 2.0 ** 30, 2.0 ** 56):
        if bits == 16:
            s.pools[0].copy_((base_k.float() * size).to(torch.bfloat16))
        else:
            s.scales[0].copy_(base_k * size)
        q = rows(T, heads, head_dim, 62, size=1.5 * size)
        cache = s.cache()
        got = attend(cache, B.KVBatch(s.table, s.kv_lens, cu if prompt else None), q).double()
        cache.check()
        want, decided = winners(s, q, counts, QUERY_FIXED if bits == 8 and not prompt else 0.0)
        assert decided.double().mean() > 0.4
        off = (got - want).abs()[decided] - (2.02 * 2.0 ** -8 * want.abs()[decided] + 2.0 ** -134)
        assert torch.all(off <= 0), f"size {size}: {int((~(off <= 0)).any(-1).sum())} of {off.shape[0]} rows are wrong"


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.inf, -math.inf])
@pytest.mark.parametrize("past", [50, 2850])
@pytest.mark.parametrize("size", [0.0, 1.5])
@pytest.mark.parametrize("prompt", [False, True])
def test_an_infinite_value_gives_the_infinity_to_the_tokens_that_see_it(value, past, size, prompt):
    """Every weight is positive, so the sum is infinite, whatever the weight is (size 0: 1 over the number of keys)."""
    n, at = past + 150, past + 49
    s = R.Setup([n, n], 1, 64, 16, 16, seed=63)
    s.pools[1][s.table[0, at // 16].item(), 0, at % 16, 5] = value
    counts = [150, 150] if prompt else [1, 1]
    q = rows(sum(counts), 2, 64, 64, size=size)
    cu = torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32, device="cuda")
    got = (B.attend_prompt if prompt else B.attend_decode)(s.cache(), B.KVBatch(s.table, s.kv_lens, cu if prompt else None), q)
    sees = torch.zeros(sum(counts), dtype=torch.bool, device="cuda")
    sees[49 if prompt else 0:counts[0]] = True
    assert torch.all(got[sees][..., 5] == value)
    assert torch.all(torch.isfinite(got[~sees]))
    other = [d for d in range(64) if d != 5]
    assert torch.all(torch.isfinite(got[..., other]))
