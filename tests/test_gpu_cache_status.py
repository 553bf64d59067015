"""What the cache's status word reports, when, and what a call does with pages, lengths and token rows that do not exist."""
import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_attention import WEIGHT_BF16, check, error_of, rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["append", "decode", "prompt"])
def test_check_waits_for_calls_on_every_stream(call):
    """The call that meets a bad page runs on a side stream, behind work that takes about 50 ms; check() is asked on the
    default stream at once, and leaves a status word that is clear for the next call."""
    s = R.Setup([40, 40], 2, 64, 16, 16, seed=71)
    s.table[1, 2] = s.n_pages
    cache = s.cache()
    cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    batch = B.KVBatch(s.table, s.kv_lens, cu if call == "prompt" else None)
    q, kv = rows(2, 4, 64, 72), rows(2, 2, 64, 73)
    out, ws = torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda"), B.alloc_attend_workspace(4, 2, 64, prompt=call == "prompt")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(2):
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        if call == "append":
            B.kv_append(cache, batch, kv, kv, stream=side)
        else:
            (B.attend_prompt if call == "prompt" else B.attend_decode)(cache, batch, q, out=out, workspace=ws, stream=side)
        with pytest.raises(B.BitLinearError) as e:
            cache.check()
        assert e.value.status == B.ERR_PAGE
        torch.cuda.synchronize()
        assert cache.status.item() == B.OK


@pytest.mark.parametrize("bits", [16, 8])
def test_a_new_cache_is_ready_for_every_stream(bits):
    """The current stream is busy when the cache is made: what fills its tensors and its status word there must not come after a
    call on another stream."""
    s = R.Setup([40, 40], 2, 64, 16, bits, seed=88)
    s.table[0, :3] = torch.tensor([0, 1, 2], dtype=torch.int32)
    s.table[1, 2] = -1
    kv, side = rows(2, 2, 64, 89), torch.cuda.Stream()
    B.kv_append(s.cache(), B.KVBatch(s.table[:1], s.kv_lens[:1]), kv[:1], kv[:1])  # (a kernel's first launch loads it and waits)
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    cache = B.KVCache(8, 2, 64, page_size=16, bits=bits)
    B.kv_append(cache, B.KVBatch(s.table[:1], s.kv_lens[:1]), kv[:1], kv[:1], stream=side)
    torch.cuda.synchronize()
    stored = kv[0] if bits == 16 else R.codes(kv[0].double())[0]
    assert torch.equal(cache.v[2, :, 7], stored)
    torch.cuda._sleep(100_000_000)
    cache = s.cache()
    B.kv_append(cache, B.KVBatch(s.table, s.kv_lens), kv, kv, stream=side)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE


@pytest.mark.parametrize("prompt", [False, True])
def test_a_new_workspace_is_ready_for_every_stream(prompt):
    """The same of a workspace: the memory it gets held ones before."""
    new = [1, 1] if not prompt else [100, 33]
    cu = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda")
    s = R.Setup([4000, 600], 2, 128, 16, 16, seed=90)
    cache, batch, q = s.cache(), B.KVBatch(s.table, s.kv_lens, cu if prompt else None), rows(sum(new), 8, 128, 91)
    out, side = torch.empty(sum(new), 8, 128, dtype=torch.bfloat16, device="cuda"), torch.cuda.Stream()
    attend = B.attend_prompt if prompt else B.attend_decode
    attend(cache, batch, q)  # (a kernel's first launch loads it and waits)
    out.fill_(0.5)
    stale = torch.full((B.attend_workspace_bytes(8, 2, 128, prompt),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    del stale
    torch.cuda._sleep(100_000_000)
    ws = B.alloc_attend_workspace(8, 2, 128, prompt=prompt)
    attend(cache, batch, q, out=out, workspace=ws, stream=side)
    cache.check()
    want, bound = R.attend(s, q, new, **error_of(prompt, 16))
    check(out, want, bound)


def test_a_bad_page_does_not_replace_an_expired_wait():
    """The word keeps its code until the owner clears it: a timeout, which leaves results unspecified, is not made to look like
    a page by the calls behind it."""
    s = R.Setup([200, 40], 1, 64, 16, 16, seed=74)
    q = rows(60, 2, 64, 75)
    cu = torch.tensor([0, 60, 60], dtype=torch.int32, device="cuda")
    cache = s.cache()
    ws = B.alloc_attend_workspace(2, 1, 64, prompt=True)
    B.attend_prompt(cache, B.KVBatch(s.table, s.kv_lens, cu), q, workspace=ws)
    cache.check()
    B.test_expire_next_wait(2000, True)
    B.attend_prompt(cache, B.KVBatch(s.table, s.kv_lens, cu), q, workspace=ws)
    s.table[1, 1] = -1
    one, kv = rows(2, 2, 64, 76), rows(2, 1, 64, 77)
    s.kv_lens[1] = 20
    B.attend_decode(cache, B.KVBatch(s.table, s.kv_lens), one)
    B.kv_append(cache, B.KVBatch(s.table, s.kv_lens), kv, kv)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_TIMEOUT
    B.attend_decode(cache, B.KVBatch(s.table, s.kv_lens), one)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE


# bounds of two sequences of a call with five token rows; the rows of each that attend_prompt and kv_append serve
ROWS = [
    ([0, 4, 9], [range(0, 4), []], [range(0, 4), range(4, 5)]),
    ([0, 4, 2 ** 31 - 1], [range(0, 4), []], [range(0, 4), range(4, 5)]),
    ([0, 7, 7], [[], []], [range(0, 5), []]),
    ([-3, 2, 5], [[], range(2, 5)], [range(0, 2), range(2, 5)]),
    ([0, 5, 6], [range(0, 5), []], [range(0, 5), []]),
    ([-2, 0, 5], [[], range(0, 5)], [[], range(0, 5)]),
]


@pytest.mark.parametrize("cu,attended,appended", ROWS)
@pytest.mark.parametrize("bits", [16, 8])
def test_sequences_whose_rows_were_not_all_handed_over_are_reported(cu, attended, appended, bits):
    """attend_prompt leaves such a sequence out, kv_append stores the rows that it was given; both say so."""
    s = R.Setup([30, 21], 2, 64, 16, bits, seed=78)
    bounds = torch.tensor(cu, dtype=torch.int32, device="cuda")
    batch, cache = B.KVBatch(s.table, s.kv_lens, bounds), s.cache()
    q, out = rows(5, 4, 64, 79), torch.full((5, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    B.attend_prompt(cache, batch, q, out=out)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE
    served = [t for b in (0, 1) for t in attended[b]]
    for b in (0, 1):
        if len(attended[b]):
            alone = [0, 0]
            alone[b] = len(attended[b])
            want, bound = R.attend(s, q[list(attended[b])], alone, weight_rounding=WEIGHT_BF16)
            check(out[list(attended[b])], want, bound)
    assert torch.all(out[[t for t in range(5) if t not in served]] == 3.0)

    kv = rows(5, 2, 64, 80)
    before = s.pools[1].clone()
    B.kv_append(cache, batch, kv, kv)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE
    expected = before.clone()
    for b in (0, 1):
        for t in appended[b]:
            pos = s.lens[b] - (cu[b + 1] - cu[b]) + t - cu[b]
            if pos >= 0:
                value = kv[t] if bits == 16 else R.codes(kv[t].double())[0]
                expected[s.table[b, pos // 16].item(), :, pos % 16] = value
    kind = torch.int16 if bits == 16 else torch.int8
    assert torch.equal(s.pools[1].view(kind), expected.view(kind))


@pytest.mark.parametrize("cu", [[0, 3, 3], [0, 0, 2], [1, 3, 5]])
def test_rows_behind_the_last_sequence_and_in_front_of_the_first_are_no_error(cu):
    s = R.Setup([30, 21], 2, 64, 16, 16, seed=81)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens, torch.tensor(cu, dtype=torch.int32, device="cuda"))
    out = torch.full((5, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    kv = rows(5, 2, 64, 82)
    B.kv_append(cache, batch, kv, kv)
    B.attend_prompt(cache, batch, rows(5, 4, 64, 83), out=out)
    cache.check()
    assert torch.all(out[:cu[0]] == 3.0) and torch.all(out[cu[2]:] == 3.0)


def attend_without(s, b, dropped, q, length, prompt, bits):
    """(out, bound) of the new tokens q of sequence b over its keys but those of the dropped pages, the last token at length - 1.
    The bound is that of kv_reference.attend, with the keys that are left as the only ones."""
    n, H, D = q.shape
    G = H // s.kv_heads
    k, v = s.rows(0, b, length), s.rows(1, b, length)
    gone = torch.zeros(length, dtype=torch.bool, device=q.device)
    for p in dropped:
        gone[p * s.page_size:(p + 1) * s.page_size] = True
    scale = D ** -0.5
    x = q.double().reshape(n, s.kv_heads, G, D).permute(1, 2, 0, 3)
    score, size = scale * torch.einsum("hgnd,hld->hgnl", x, k), scale * torch.einsum("hgnd,hld->hgnl", x.abs(), k.abs())
    hidden = gone[None] | (torch.arange(length, device=q.device)[None] > (length - n + torch.arange(n, device=q.device))[:, None])
    w = torch.softmax(score.masked_fill(hidden, -float("inf")), -1).nan_to_num(0.0)
    y, A = torch.einsum("hgnl,hld->hgnd", w, v), torch.einsum("hgnl,hld->hgnd", w, v.abs())
    e = error_of(prompt, bits)
    worst = size.masked_fill(hidden, 0.0).amax(-1, keepdim=True) * (D + 4) * 2.0 ** -24
    fixed = scale * x.abs().amax(-1)[..., None] * k.abs().sum(-1)[:, None, None]
    worst = worst + e.get("query_rounding", 0.0) * fixed.masked_fill(hidden, 0.0).amax(-1, keepdim=True)
    d = 2 * worst + 2.0 ** -21 + e["weight_rounding"] + (length + 64) * 2.0 ** -24
    bound = 1.01 * 2 * d * A + 2.0 ** -8 * y.abs() + 2.0 ** -134 + length * 2.0 ** -119 * max(1.0, v.abs().max().item())
    return y.permute(2, 0, 1, 3).reshape(n, H, D), bound.permute(2, 0, 1, 3).reshape(n, H, D)


@pytest.mark.parametrize("prompt", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("heads,kv_heads,head_dim,page,length,new,dropped", [
    (4, 2, 64, 16, 130, 30, [3]),
    (4, 2, 64, 16, 130, 30, [0, 7]),    # a page inside the new tokens: some of them do not see it
    (4, 1, 64, 16, 130, 130, [0]),      # the first 16 tokens are left with nothing
    (2, 2, 100, 32, 200, 40, [1, 2]),
    (8, 1, 128, 64, 300, 20, [4]),      # the last, partial page
    (2, 1, 128, 256, 700, 60, [1]),     # two whole blocks of keys
    (2, 2, 64, 16, 3000, 20, [5, 90, 187]),  # split among several CTAs
])
@pytest.mark.parametrize("size", [1.5, 30.0])
def test_keys_of_bad_pages_alone_are_missing(heads, kv_heads, head_dim, page, length, new, dropped, bits, prompt, size):
    """The keys of those pages are the largest ones: they would take over where they took part.  Also with a sharp softmax, which
    shows single keys that are lost."""
    s = R.Setup([50, length], kv_heads, head_dim, page, bits, seed=84)
    for p in dropped:
        (s.pools if bits == 16 else s.scales)[0][s.table[1, p].item()] *= 4.0
    n = new if prompt else 1
    q = rows(20 + n if prompt else 2, heads, head_dim, 85, size=size)
    counts = [20, n] if prompt else [1, 1]
    cu = torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32, device="cuda")
    table = s.table.clone()
    for p, bad in zip(dropped, (s.n_pages, -1, 2 ** 31 - 1)):
        table[1, p] = bad
    cache = s.cache()
    got = (B.attend_prompt if prompt else B.attend_decode)(cache, B.KVBatch(table, s.kv_lens, cu if prompt else None), q)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE
    want, bound = attend_without(s, 1, dropped, q[counts[0]:], length, prompt, bits)
    check(got[counts[0]:], want, bound)
    want, bound = attend_without(s, 0, [], q[:counts[0]], 50, prompt, bits)
    check(got[:counts[0]], want, bound)


@pytest.mark.parametrize("prompt", [False, True])
@pytest.mark.parametrize("bits", [16, 8])
def test_a_length_beyond_the_table_counts_as_far_as_the_table_goes(prompt, bits):
    """Every key that the table covers takes part; the tokens behind it see all of them, those inside it their own part."""
    s = R.Setup([128], 2, 64, 16, bits, seed=86, table_extra=0)
    n = 40 if prompt else 1
    over = 25
    q = rows(n, 4, 64, 87)
    s.kv_lens[0] = 128 + over
    cache, cu = s.cache(), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    got = (B.attend_prompt if prompt else B.attend_decode)(cache, B.KVBatch(s.table, s.kv_lens, cu if prompt else None), q)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE
    for i in range(n):  # the token at position 128 + over - n + i
        sees = min(128, 128 + over - n + i + 1)
        want, bound = attend_without(s, 0, [], q[i:i + 1], sees, prompt, bits)
        check(got[i:i + 1], want, bound)


@pytest.mark.parametrize("tokens", [3, 40, 130])
@pytest.mark.parametrize("bits", [16, 8])
def test_a_long_prompt_does_not_use_up_the_waits_of_the_matmul_behind_it(bits, tokens):
    """A tile over 2^24 keys takes several ms.  The matmul launched next, whose waits are allowed 1 ms here, may not be resident
    meanwhile: its quantiser lets it in early, but is itself let in by the prompt kernel only when that is at its end."""
    from paper_2402_17764_b200 import synthetic as S
    keys, N, K = 1 << 24, 512, 1536
    cache = B.KVCache(keys // 256, 1, 4, page_size=256, bits=bits)
    table = torch.arange(keys // 256, dtype=torch.int32, device="cuda")[None]
    batch = B.KVBatch(table, torch.tensor([keys], dtype=torch.int32, device="cuda"), torch.tensor([0, 256], dtype=torch.int32, device="cuda"))
    q, out, ws = rows(256, 1, 4, 92), rows(256, 1, 4, 93), B.alloc_attend_workspace(1, 1, 4, prompt=True)
    packed, gamma = B.quantize_weights(S.latent_weights(N, K, 1).cuda())
    X, Y, matmul_ws = S.activations(tokens, K, 2).cuda(), torch.empty(tokens, N, dtype=torch.bfloat16, device="cuda"), B.alloc_workspace(tokens, N, K)
    B.forward(packed, gamma, X, N, workspace=matmul_ws, Y=Y)
    want = Y.clone()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    B.attend_prompt(cache, batch, q, out=out, workspace=ws)
    start.record()
    B.attend_prompt(cache, batch, q, out=out, workspace=ws)
    end.record()
    cache.check()
    assert start.elapsed_time(end) > 3.0
    Y.zero_()
    B.attend_prompt(cache, batch, q, out=out, workspace=ws)
    B.test_expire_next_wait(1000, False)
    B.forward(packed, gamma, X, N, workspace=matmul_ws, Y=Y)
    assert B.poll_status(matmul_ws) == B.OK
    cache.check()
    assert torch.equal(Y, want)
