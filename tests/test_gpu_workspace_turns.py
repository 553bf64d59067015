"""One attention workspace, zeroed once, for calls of every kind and width in turn."""
import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_attention import rows
from test_gpu_attention_shared import shared

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS = 64, 4


def shared_call(head_dim, page, groups, bits, seed):
    s, of = shared(groups, KV_HEADS, head_dim, page, bits, seed)
    q = rows(len(s.lens), HEADS, head_dim, seed + 1)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)

    def call(workspace):
        out = torch.full_like(q, 7.0)
        B.attend_decode_shared(cache, batch, of, q, out=out, workspace=workspace, share_from=0)
        cache.check()
        return [out]

    return call, B.attend_shared_workspace_bytes(HEADS, KV_HEADS, head_dim, len(s.lens))


def decode_call(head_dim, page, lens, bits, seed, weigh):
    s = R.Setup(lens, KV_HEADS, head_dim, page, bits, seed=seed)
    q = rows(len(lens), HEADS, head_dim, seed + 1)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens)

    def call(workspace):
        out = torch.full_like(q, 7.0)
        if not weigh:
            B.attend_decode(cache, batch, q, out=out, workspace=workspace)
            cache.check()
            return [out]
        marks = B.KVMarks(cache)
        B.attend_decode_weigh(cache, batch, marks, q, out=out, workspace=workspace)
        cache.check()
        return [out, marks.mass]

    if weigh:
        return call, B.attend_weigh_workspace_bytes(HEADS, KV_HEADS, head_dim, bits, len(lens), sum(lens))
    return call, B.attend_workspace_bytes(HEADS, KV_HEADS, head_dim, False)


def prompt_call(head_dim, page, lens, new, bits, seed):
    s = R.Setup(lens, KV_HEADS, head_dim, page, bits, seed=seed)
    cu = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    q = rows(sum(new), HEADS, head_dim, seed + 1)
    cache, batch = s.cache(), B.KVBatch(s.table, s.kv_lens, cu)

    def call(workspace):
        out = torch.full_like(q, 7.0)
        B.attend_prompt(cache, batch, q, out=out, workspace=workspace)
        cache.check()
        return [out]

    return call, B.attend_workspace_bytes(HEADS, KV_HEADS, head_dim, True)


@pytest.mark.parametrize("bits", [16, 8])
def test_calls_of_every_kind_and_width_take_turns(bits):
    """The widest call fills the workspace with partial results (16 sequences of 16 query heads fill a tile's 256 rows, 8192 shared rows
    are split among 32 CTAs for each of the four heads); the others split their sequences among CTAs, whose counters have to be
    zero all the same.  Every call gives the bits that it gives on a workspace of its own."""
    calls = [
        shared_call(128, 64, [(8192, [8300 + 60 * i for i in range(16)])], bits, 1),
        shared_call(64, 64, [(64, [3000, 2000, 70])], bits, 3),
        decode_call(64, 32, [5000, 3, 700], bits, 5, weigh=True),
        shared_call(20, 16, [(320, [4000, 330])] * 2, bits, 7),
        decode_call(128, 64, [9000, 40], bits, 9, weigh=True),
        decode_call(100, 16, [6000], bits, 11, weigh=False),
        prompt_call(64, 32, [3000, 500], [40, 30], bits, 13),
        decode_call(64, 32, [70, 4000], bits, 15, weigh=False),
    ]
    want = [call(torch.zeros(nbytes, dtype=torch.uint8, device="cuda")) for call, nbytes in calls]
    workspace = torch.zeros(max(nbytes for _, nbytes in calls), dtype=torch.uint8, device="cuda")
    for first in range(len(calls)):
        for i in [0] + [(first + j) % len(calls) for j in range(len(calls))]:
            got = calls[i][0](workspace)
            assert all(torch.equal(x, y) for x, y in zip(got, want[i])), f"call {i}, of the turn that begins with {first}"
