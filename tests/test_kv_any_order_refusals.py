"""CPU-only: selection of rows in any order refuses what the other form refuses, before anything is launched."""
import pytest

from test_kv_more_refusals import marks
from test_kv_refusals import BATCH_ERRORS, CACHE_ERRORS, FAKE, B, address, batch, cache  # noqa: F401 (B is a fixture)


def select(B, c, s, **changes):
    d = dict(marks=marks(B), keep=8, recent=2, source=FAKE, new_lens=FAKE + 64, stream=None)
    d.update(changes)
    held = d["marks"]  # (alive until the call returns)
    d["marks"] = address(held)
    return B.load_library().bitlinear_kv_select_any_order(address(c), address(s), *d.values())


def test_caches_and_batches_that_are_refused(B):  # noqa: F811
    s = batch(B, cu_tokens=None)
    for changes, status in CACHE_ERRORS:
        assert select(B, cache(B, **changes), s) == getattr(B, status), changes
    for changes, status in BATCH_ERRORS:
        assert select(B, cache(B), batch(B, **{"cu_tokens": None, **changes})) == getattr(B, status), changes


@pytest.mark.parametrize("changes,status", [
    (dict(marks=None), "ERR_ARG"), (dict(keep=0), "ERR_SHAPE"), (dict(keep=(1 << 30) + 1), "ERR_SHAPE"), (dict(recent=-1), "ERR_SHAPE"),
    (dict(recent=9), "ERR_SHAPE"), (dict(source=None), "ERR_ARG"), (dict(new_lens=None), "ERR_ARG"), (dict(new_lens=FAKE + 8), "ERR_ARG"),
    (dict(source=FAKE + 2), "ERR_ALIGN"), (dict(new_lens=FAKE + 65), "ERR_ALIGN"),
])
def test_arguments_that_are_refused(B, changes, status):  # noqa: F811
    assert select(B, cache(B), batch(B, cu_tokens=None), **changes) == getattr(B, status)
