"""CPU-only: what the cache and attention entry points refuse before anything is launched, and the kernels' look-ups of
lengths, pages and sequences (compiled for the host) on tables that are wrong in every way."""
import ctypes
import math
import subprocess
from pathlib import Path

import pytest
import torch

ROOT = Path(__file__).resolve().parent.parent
FAKE = 0x1000  # non-null and aligned; never dereferenced


@pytest.fixture(scope="module")
def B():
    from paper_2402_17764_b200 import binding, build
    build.build()
    binding.load_library()
    return binding


def cache(B, **changes):
    d = dict(k=FAKE, v=FAKE, k_scale=None, v_scale=None, status=FAKE, n_pages=8, kv_heads=2, head_dim=64, page_size=16, bits=16)
    d.update(changes)
    return B.KVCacheDesc(*d.values())


def batch(B, **changes):
    d = dict(page_table=FAKE, kv_lens=FAKE, cu_tokens=FAKE, n_seqs=3, table_stride=4, table_pages=4)
    d.update(changes)
    return B.KVBatchDesc(*d.values())


def address(x):
    return None if x is None else ctypes.addressof(x)


def append(B, c, s, **changes):
    d = dict(k=FAKE, k_stride=128, v=FAKE, v_stride=128, q=FAKE, q_stride=256, T=3, heads=4, rope=FAKE, rope_positions=64,
             interleaved=0, q_out=FAKE, q_out_stride=256, stream=None)
    d.update(changes)
    return B.load_library().bitlinear_kv_append(address(c), address(s), *d.values())


def attend(B, c, s, prompt, **changes):
    d = dict(q=FAKE, q_stride=256, T=3, heads=4, scale=0.125, out=FAKE + 4096, out_stride=256, workspace=FAKE, bytes=1 << 40, stream=None)
    d.update(changes)
    if not prompt:
        d.pop("T")
    f = B.load_library().bitlinear_attend_prompt if prompt else B.load_library().bitlinear_attend_decode
    return f(address(c), address(s), *d.values())


CACHE_ERRORS = [
    (dict(k=None), "ERR_ARG"), (dict(v=None), "ERR_ARG"), (dict(status=None), "ERR_ARG"), (dict(bits=4), "ERR_ARG"),
    (dict(bits=8), "ERR_ARG"), (dict(bits=8, k_scale=FAKE), "ERR_ARG"), (dict(k_scale=FAKE, v_scale=FAKE), "ERR_ARG"),
    (dict(kv_heads=0), "ERR_SHAPE"), (dict(kv_heads=1025), "ERR_SHAPE"), (dict(head_dim=66), "ERR_SHAPE"),
    (dict(head_dim=0), "ERR_SHAPE"), (dict(head_dim=132), "ERR_SHAPE"), (dict(page_size=8), "ERR_SHAPE"),
    (dict(page_size=48), "ERR_SHAPE"), (dict(page_size=512), "ERR_SHAPE"), (dict(n_pages=0), "ERR_SHAPE"),
    (dict(n_pages=(1 << 31) // 32), "ERR_SHAPE"), (dict(k=FAKE + 8), "ERR_ALIGN"), (dict(v=FAKE + 2), "ERR_ALIGN"),
    (dict(bits=8, k_scale=FAKE + 4, v_scale=FAKE), "ERR_ALIGN"), (dict(status=FAKE + 2), "ERR_ALIGN"),
]
BATCH_ERRORS = [
    (dict(page_table=None), "ERR_ARG"), (dict(kv_lens=None), "ERR_ARG"), (dict(n_seqs=-1), "ERR_SHAPE"),
    (dict(n_seqs=(1 << 20) + 1), "ERR_SHAPE"), (dict(table_pages=0), "ERR_SHAPE"), (dict(table_pages=5), "ERR_SHAPE"),
    (dict(table_pages=1 << 27, table_stride=1 << 27), "ERR_SHAPE"), (dict(page_table=FAKE + 1), "ERR_ALIGN"),
    (dict(kv_lens=FAKE + 2), "ERR_ALIGN"), (dict(cu_tokens=FAKE + 2), "ERR_ALIGN"),
]


@pytest.mark.parametrize("which", ["append", "decode", "prompt"])
def test_caches_and_batches_that_are_refused(B, which):
    def call(c, s):
        if which == "append":
            return append(B, c, s)
        return attend(B, c, s, which == "prompt")

    own = {} if which != "decode" else dict(cu_tokens=None)
    assert call(None, batch(B, **own)) == B.ERR_ARG
    assert call(cache(B), None) == B.ERR_ARG
    for changes, status in CACHE_ERRORS:
        assert call(cache(B, **changes), batch(B, **own)) == getattr(B, status), changes
    for changes, status in BATCH_ERRORS:
        if which == "decode" and "cu_tokens" in changes:
            continue
        assert call(cache(B), batch(B, **{**own, **changes})) == getattr(B, status), changes


def test_arguments_of_append_that_are_refused(B):
    c, s = cache(B), batch(B)
    for changes, status in [
        (dict(k=None), "ERR_ARG"), (dict(v=None), "ERR_ARG"), (dict(q_out=None), "ERR_ARG"), (dict(interleaved=2), "ERR_ARG"),
        (dict(T=-1), "ERR_SHAPE"), (dict(T=(1 << 20) + 1), "ERR_SHAPE"), (dict(k_stride=120), "ERR_SHAPE"),
        (dict(v_stride=132), "ERR_SHAPE"), (dict(q_stride=248), "ERR_SHAPE"), (dict(q_out_stride=260), "ERR_SHAPE"),
        (dict(k=FAKE + 8), "ERR_ALIGN"), (dict(v=FAKE + 8), "ERR_ALIGN"), (dict(q=FAKE + 8), "ERR_ALIGN"),
        (dict(q_out=FAKE + 8), "ERR_ALIGN"), (dict(rope=FAKE + 8), "ERR_ALIGN"), (dict(rope_positions=0), "ERR_SHAPE"),
        (dict(heads=0), "ERR_SHAPE"), (dict(heads=4097, q_stride=1 << 20, q_out_stride=1 << 20), "ERR_SHAPE"),
        (dict(q_out_stride=264), "ERR_ARG"),  # in place, with another stride
    ]:
        assert append(B, c, s, **changes) == getattr(B, status), changes
    assert append(B, c, batch(B, cu_tokens=None), T=4) == B.ERR_SHAPE  # one token per sequence: T = n_seqs


def test_arguments_of_attention_that_are_refused(B):
    for prompt in (False, True):
        c, s = cache(B), batch(B, cu_tokens=FAKE if prompt else None)
        for changes, status in [
            (dict(q=None), "ERR_ARG"), (dict(out=None), "ERR_ARG"), (dict(out=FAKE), "ERR_ARG"), (dict(workspace=None), "ERR_ARG"),
            (dict(scale=0.0), "ERR_ARG"), (dict(scale=-1.0), "ERR_ARG"), (dict(scale=math.inf), "ERR_ARG"),
            (dict(scale=math.nan), "ERR_ARG"), (dict(scale=3e38), "ERR_ARG"), (dict(heads=3), "ERR_SHAPE"), (dict(heads=0), "ERR_SHAPE"),
            (dict(heads=4098, q_stride=1 << 20, out_stride=1 << 20), "ERR_SHAPE"), (dict(q_stride=252), "ERR_SHAPE"),
            (dict(out_stride=248), "ERR_SHAPE"), (dict(q=FAKE + 8), "ERR_ALIGN"), (dict(out=FAKE + 8), "ERR_ALIGN"),
            (dict(workspace=FAKE + 16), "ERR_ALIGN"), (dict(bytes=16), "ERR_WORKSPACE"),
        ]:
            assert attend(B, c, s, prompt, **changes) == getattr(B, status), changes
        assert attend(B, c, batch(B, cu_tokens=None if prompt else FAKE), prompt) == B.ERR_ARG
    assert attend(B, cache(B), batch(B), True, T=(1 << 20) + 1) == B.ERR_SHAPE


def test_sizes_and_the_rotary_table(B):
    assert B.kv_cache_bytes(3, 2, 100, 16, 16) == 3 * 2 * 16 * 112 * 2
    assert B.kv_cache_bytes(3, 2, 128, 256, 8) == 3 * 2 * 256 * 128
    assert B.kv_cache_bytes(3, 2, 4, 32, 8) == 3 * 2 * 32 * 16
    for bad in ((0, 2, 64, 16, 16), (3, 0, 64, 16, 16), (3, 2, 65, 16, 16), (3, 2, 64, 24, 16), (3, 2, 64, 16, 32)):
        assert B.kv_cache_bytes(*bad) == 0
    for prompt in (False, True):
        assert B.attend_workspace_bytes(64, 8, 128, prompt) % 256 == 0 and B.attend_workspace_bytes(64, 8, 128, prompt) > 0
        assert B.attend_workspace_bytes(63, 8, 128, prompt) == 0 and B.attend_workspace_bytes(64, 8, 130, prompt) == 0
    L = B.load_library()
    assert L.bitlinear_attend_workspace_bytes(64, 8, 128, 2) == 0
    assert L.bitlinear_rope_table(None, 8, 64, 1e4, None) == B.ERR_ARG
    assert L.bitlinear_rope_table(FAKE, 0, 64, 1e4, None) == B.ERR_SHAPE
    assert L.bitlinear_rope_table(FAKE, 8, 62, 1e4, None) == B.ERR_SHAPE
    assert L.bitlinear_rope_table(FAKE, 8, 64, 0.0, None) == B.ERR_ARG
    assert L.bitlinear_rope_table(FAKE, 8, 64, math.inf, None) == B.ERR_ARG
    assert L.bitlinear_rope_table(FAKE + 8, 8, 64, 1e4, None) == B.ERR_ALIGN
    assert "page" in B.status_string(B.ERR_PAGE)


def test_without_an_sm100_device_valid_calls_are_refused(B):
    if torch.cuda.is_available() and torch.cuda.get_device_capability()[0] == 10:
        pytest.skip("an sm_100 device is present")
    assert append(B, cache(B), batch(B)) == B.ERR_ARCH
    assert attend(B, cache(B), batch(B, cu_tokens=None), False) == B.ERR_ARCH
    assert attend(B, cache(B), batch(B), True) == B.ERR_ARCH
    assert B.load_library().bitlinear_rope_table(FAKE, 8, 64, 1e4, None) == B.ERR_ARCH


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu(B):
    with pytest.raises(B.BitLinearError):
        B.KVCache.from_tensors(torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), 64)
    with pytest.raises(B.BitLinearError):
        B.KVBatch(torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(B.BitLinearError):
        B.KVCache(4, 2, 64, page_size=24)


# ---- the kernels' look-ups, on the host ------------------------------------------------------------------

HOST = r"""
#include <cstring>
#include "kv.cuh"
using namespace bitlinear;
static KvBatch batch_of(const int *table, const int *lens, const int *cu, int n, int capacity, long long stride)
{
    KvBatch s{};
    s.page_table = table; s.kv_lens = lens; s.cu_tokens = cu; s.n_seqs = n; s.capacity = capacity; s.table_stride = stride;
    return s;
}
extern "C" int length_of(const int *lens, int b, int capacity, int *over)
{
    bool o;
    const int n = kv_length(batch_of(nullptr, lens, nullptr, b + 1, capacity, 0), b, o);
    *over = o;
    return n;
}
extern "C" int page_of(const int *table, long long stride, int b, int pos, int shift, int n_pages)
{
    KvCache c{};
    c.page_shift = shift; c.n_pages = n_pages;
    return kv_page(c, batch_of(table, nullptr, nullptr, b + 1, 0, stride), b, pos);
}
extern "C" int row_of(int page, int head, int pos, int shift, int kv_heads)
{
    KvCache c{};
    c.page_shift = shift; c.kv_heads = kv_heads;
    return kv_row(c, page, head, pos);
}
extern "C" int sequence_of(const int *cu, int n, int t, int *first, int *count)
{
    return kv_sequence_of(batch_of(nullptr, nullptr, cu, n, 0, 0), t, *first, *count);
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    from paper_2402_17764_b200 import build
    at = tmp_path_factory.mktemp("lookups")
    (at / "lookups.cu").write_text(HOST)
    subprocess.run([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O1", "-Xcompiler", "-fPIC", "-shared",
                    "--cudart", "static", "-I", str(build.CSRC), "-o", str(at / "lookups.so"), str(at / "lookups.cu")], check=True)
    return ctypes.CDLL(str(at / "lookups.so"))


def ints(*x):
    return (ctypes.c_int * len(x))(*x)


def test_lengths_are_cut_to_the_page_table(host):
    over = ctypes.c_int()
    for n, want, cut in ((0, 0, 0), (5, 5, 0), (64, 64, 0), (65, 64, 1), (2 ** 31 - 1, 64, 1), (-1, 0, 0), (-2 ** 31, 0, 0)):
        assert (host.length_of(ints(n), 0, 64, ctypes.byref(over)), over.value) == (want, cut)


def test_page_numbers_outside_the_cache_are_none(host):
    table = ints(3, 0, 7, 8, -1, 2 ** 31 - 1, -2 ** 31, 6)
    stride = ctypes.c_longlong(4)
    got = [host.page_of(table, stride, b, 16 * p + 5, 4, 8) for b in (0, 1) for p in range(4)]
    assert got == [3, 0, 7, -1, -1, -1, -1, 6]


def test_rows_of_the_largest_caches_fit_31_bits(host):
    for shift, heads in ((4, 1024), (8, 1), (6, 8)):
        pages = (1 << 31) // (heads << shift) - 1
        assert host.row_of(pages - 1, heads - 1, (1 << 30) - 1, shift, heads) == pages * (heads << shift) - 1 < 2 ** 31


def test_sequences_of_token_rows(host):
    def of(cu, t):
        first, count = ctypes.c_int(-9), ctypes.c_int(-9)
        b = host.sequence_of(ints(*cu), len(cu) - 1, t, ctypes.byref(first), ctypes.byref(count))
        return (b, first.value, count.value) if b >= 0 else None
    assert [of([0, 2, 2, 5], t) for t in range(6)] == [(0, 0, 2), (0, 0, 2), (2, 2, 3), (2, 2, 3), (2, 2, 3), None]
    assert of([0, 0, 0], 0) is None and of([3, 5], 2) is None and of([3, 5], 4) == (0, 3, 2)
    for cu in ([5, 1, 7, 0], [-3, 100, -100], [2 ** 31 - 1, -2 ** 31]):  # nonsense: any answer inside the batch, or none
        for t in range(12):
            got = of(cu, t)
            assert got is None or 0 <= got[0] < len(cu) - 1
