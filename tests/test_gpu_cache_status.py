"""What the cache's status word reports, and when."""
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
