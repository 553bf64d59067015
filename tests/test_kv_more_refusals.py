"""CPU-only: what appending with norms, the weighing and the shared attention, and evicting refuse before anything is launched."""
import ctypes
import math

import pytest
import torch

from test_kv_refusals import BATCH_ERRORS, CACHE_ERRORS, FAKE, B, address, batch, cache  # noqa: F401 (B is a fixture)


def marks(B, **changes):
    d = dict(mass=FAKE, pos=FAKE)
    d.update(changes)
    return B.KVMarksDesc(*d.values())


def append(B, c, s, **changes):
    d = dict(k=FAKE, k_stride=128, v=FAKE, v_stride=128, q=FAKE, q_stride=256, T=3, heads=4, q_gain=FAKE, k_gain=FAKE, eps=1e-5, rope=FAKE,
             rope_positions=64, interleaved=0, positions=FAKE, marks=marks(B), q_out=FAKE, q_out_stride=256, stream=None)
    d.update(changes)
    held = d["marks"]  # (alive until the call returns)
    d["marks"] = address(held)
    return B.load_library().bitlinear_kv_append_rmsnorm(address(c), address(s), *d.values())


def attend(B, c, s, which, **changes):
    d = dict(other=marks(B) if which == "weigh" else batch(B, cu_tokens=FAKE), q=FAKE, q_stride=256, heads=4, scale=0.125, share_from=0, out=FAKE + 4096,
             out_stride=256, workspace=FAKE, bytes=1 << 40, stream=None)
    if which == "weigh":
        d.pop("share_from")
    d.update(changes)
    held = d["other"]  # (alive until the call returns)
    d["other"] = address(held)
    L = B.load_library()
    f = L.bitlinear_attend_decode_weigh if which == "weigh" else L.bitlinear_attend_decode_shared
    return f(address(c), address(s), *d.values())


def select(B, c, s, **changes):
    d = dict(marks=marks(B), keep=8, recent=2, source=FAKE, new_lens=FAKE + 64, stream=None)
    d.update(changes)
    held = d["marks"]  # (alive until the call returns)
    d["marks"] = address(held)
    return B.load_library().bitlinear_kv_select(address(c), address(s), *d.values())


def compact(B, c, s, **changes):
    d = dict(source=FAKE, keep=8, marks=marks(B), stream=None)
    d.update(changes)
    held = d["marks"]  # (alive until the call returns)
    d["marks"] = address(held)
    return B.load_library().bitlinear_kv_compact(address(c), address(s), *d.values())


CALLS = {"append": append, "weigh": lambda B, c, s: attend(B, c, s, "weigh"), "shared": lambda B, c, s: attend(B, c, s, "shared"),
         "select": select, "compact": compact}


@pytest.mark.parametrize("which", list(CALLS))
def test_caches_and_batches_that_are_refused(B, which):  # noqa: F811
    call, own = CALLS[which], {} if which == "append" else dict(cu_tokens=None)
    assert call(B, None, batch(B, **own)) == B.ERR_ARG
    assert call(B, cache(B), None) == B.ERR_ARG
    for changes, status in CACHE_ERRORS:
        assert call(B, cache(B, **changes), batch(B, **own)) == getattr(B, status), changes
    for changes, status in BATCH_ERRORS:
        if own and "cu_tokens" in changes:
            continue
        assert call(B, cache(B), batch(B, **{**own, **changes})) == getattr(B, status), changes


def test_arguments_of_append_that_are_refused(B):  # noqa: F811
    c, s = cache(B), batch(B)
    for changes, status in [
        (dict(k=None), "ERR_ARG"), (dict(v=None), "ERR_ARG"), (dict(q_out=None), "ERR_ARG"), (dict(interleaved=2), "ERR_ARG"),
        (dict(T=-1), "ERR_SHAPE"), (dict(k_stride=120), "ERR_SHAPE"), (dict(v_stride=132), "ERR_SHAPE"), (dict(q_stride=248), "ERR_SHAPE"),
        (dict(q_out_stride=260), "ERR_SHAPE"), (dict(k=FAKE + 8), "ERR_ALIGN"), (dict(rope=FAKE + 8), "ERR_ALIGN"),
        (dict(rope_positions=0), "ERR_SHAPE"), (dict(heads=0), "ERR_SHAPE"), (dict(q_out_stride=264), "ERR_ARG"),
        (dict(eps=-1e-9), "ERR_ARG"), (dict(eps=math.nan), "ERR_ARG"), (dict(eps=math.inf), "ERR_ARG"), (dict(q_gain=FAKE + 8), "ERR_ALIGN"),
        (dict(k_gain=FAKE + 4), "ERR_ALIGN"), (dict(positions=FAKE + 2), "ERR_ALIGN"), (dict(marks=marks(B, mass=None)), "ERR_ARG"),
        (dict(marks=marks(B, pos=None)), "ERR_ARG"), (dict(marks=marks(B, mass=FAKE + 2)), "ERR_ALIGN"),
    ]:
        assert append(B, c, s, **changes) == getattr(B, status), changes


@pytest.mark.parametrize("which", ["weigh", "shared"])
def test_arguments_of_attention_that_are_refused(B, which):  # noqa: F811
    c, s = cache(B), batch(B, cu_tokens=None)
    for changes, status in [
        (dict(q=None), "ERR_ARG"), (dict(out=None), "ERR_ARG"), (dict(out=FAKE), "ERR_ARG"), (dict(workspace=None), "ERR_ARG"),
        (dict(scale=0.0), "ERR_ARG"), (dict(scale=math.nan), "ERR_ARG"), (dict(heads=3), "ERR_SHAPE"), (dict(heads=0), "ERR_SHAPE"),
        (dict(q_stride=252), "ERR_SHAPE"), (dict(out_stride=248), "ERR_SHAPE"), (dict(q=FAKE + 8), "ERR_ALIGN"), (dict(out=FAKE + 8), "ERR_ALIGN"),
        (dict(workspace=FAKE + 16), "ERR_ALIGN"), (dict(bytes=16), "ERR_WORKSPACE"), (dict(other=None), "ERR_ARG"),
    ]:
        assert attend(B, c, s, which, **changes) == getattr(B, status), changes
    assert attend(B, c, batch(B), which) == B.ERR_ARG  # one token per sequence: no bounds
    if which == "weigh":
        assert attend(B, c, s, which, other=marks(B, pos=None)) == B.ERR_ARG
        assert attend(B, c, s, which, other=marks(B, mass=FAKE + 1)) == B.ERR_ALIGN
        need = B.attend_weigh_workspace_bytes(4, 2, 64, 16, 3, 0)
        assert attend(B, c, s, which, bytes=need - 1) == B.ERR_WORKSPACE
    else:
        for changes, status in BATCH_ERRORS + [(dict(cu_tokens=None), "ERR_ARG")]:
            assert attend(B, c, s, which, other=batch(B, **changes)) == getattr(B, status), changes
        assert attend(B, c, s, which, bytes=B.attend_shared_workspace_bytes(4, 2, 64, 3) - 1) == B.ERR_WORKSPACE


def test_arguments_of_evicting_that_are_refused(B):  # noqa: F811
    c, s = cache(B), batch(B, cu_tokens=None)
    for changes, status in [
        (dict(marks=None), "ERR_ARG"), (dict(marks=marks(B, mass=None)), "ERR_ARG"), (dict(marks=marks(B, pos=FAKE + 2)), "ERR_ALIGN"),
        (dict(keep=0), "ERR_SHAPE"), (dict(keep=(1 << 30) + 1), "ERR_SHAPE"), (dict(recent=-1), "ERR_SHAPE"), (dict(recent=9), "ERR_SHAPE"),
        (dict(source=None), "ERR_ARG"), (dict(new_lens=None), "ERR_ARG"), (dict(new_lens=FAKE), "ERR_ARG"),  # (kv_lens itself)
        (dict(new_lens=FAKE + 8), "ERR_ARG"), (dict(new_lens=FAKE - 8), "ERR_ARG"),
        (dict(source=FAKE + 2), "ERR_ALIGN"), (dict(new_lens=FAKE + 65), "ERR_ALIGN"),
    ]:
        assert select(B, c, s, **changes) == getattr(B, status), changes
    long = dict(cu_tokens=None, table_pages=(1 << 18) // 16 + 1, table_stride=1 << 20)
    assert select(B, c, batch(B, **long)) == B.ERR_SHAPE
    assert select(B, cache(B, kv_heads=256, n_pages=4), batch(B, cu_tokens=None, n_seqs=(1 << 19) + 1)) == B.ERR_SHAPE
    for changes, status in [
        (dict(source=None), "ERR_ARG"), (dict(source=FAKE + 2), "ERR_ALIGN"), (dict(keep=0), "ERR_SHAPE"), (dict(keep=(1 << 30) + 1), "ERR_SHAPE"),
        (dict(marks=marks(B, pos=None)), "ERR_ARG"), (dict(marks=marks(B, mass=FAKE + 2)), "ERR_ALIGN"),
    ]:
        assert compact(B, c, s, **changes) == getattr(B, status), changes


def test_sizes_of_workspaces(B):  # noqa: F811
    for heads, kv_heads, head_dim in ((64, 8, 128), (71, 1, 64), (4, 4, 4)):
        for bits in (16, 8):
            few, many = (B.attend_weigh_workspace_bytes(heads, kv_heads, head_dim, bits, 3, n) for n in (0, 100000))
            assert few % 256 == 0 and many >= few + 100000 * heads * 4 * 0.99 > 0
        assert B.attend_shared_workspace_bytes(heads, kv_heads, head_dim, 10) % 256 == 0
        assert B.attend_shared_workspace_bytes(heads, kv_heads, head_dim, 10) >= 10 * heads * (head_dim + 2) * 4
    for bad in ((63, 8, 128, 16, 1, 1), (64, 8, 130, 16, 1, 1), (64, 8, 128, 4, 1, 1), (64, 8, 128, 16, -1, 1), (64, 8, 128, 16, 1, -1)):
        assert B.attend_weigh_workspace_bytes(*bad) == 0
    for bad in ((63, 8, 128, 1), (64, 8, 130, 1), (64, 8, 128, -1), (64, 8, 128, (1 << 20) + 1)):
        assert B.attend_shared_workspace_bytes(*bad) == 0


def test_without_an_sm100_device_valid_calls_are_refused(B):  # noqa: F811
    if torch.cuda.is_available() and torch.cuda.get_device_capability()[0] == 10:
        pytest.skip("an sm_100 device is present")
    for which, call in CALLS.items():
        assert call(B, cache(B), batch(B) if which == "append" else batch(B, cu_tokens=None)) == B.ERR_ARCH
    assert append(B, cache(B), batch(B), q_gain=None, k_gain=None, positions=None, marks=None) == B.ERR_ARCH
    assert compact(B, cache(B), batch(B, cu_tokens=None), marks=None) == B.ERR_ARCH


def test_marks_have_the_shape_of_their_cache(B):  # noqa: F811
    c = B.KVCache.__new__(B.KVCache)
    c.k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    c.n_pages, c.kv_heads, c.page_size, c.device, c.index = 4, 2, 16, c.k.device, -1
    mass, pos = torch.zeros(4, 2, 16), torch.zeros(4, 2, 16, dtype=torch.int32)
    assert ctypes.sizeof(B.KVMarks.from_tensors(c, mass, pos)._desc) == 16
    for bad in ((mass.double(), pos), (mass, pos.long()), (mass[:3], pos), (mass, pos.transpose(0, 1).contiguous()), (mass.transpose(0, 1), pos)):
        with pytest.raises(B.BitLinearError):
            B.KVMarks.from_tensors(c, *bad)
