"""More of what the marks receive and decide: every row of the results is looked at."""
import pytest
import torch

import kv_reference as R
from paper_2402_17764_b200 import binding as B
from test_gpu_attention import check, decode_error, rows
from test_gpu_attention_weigh import check_mass, marks_of, weights
from test_gpu_kv_evict import row_numbers

pytestmark = pytest.mark.gpu


def test_positions_at_both_ends_of_their_range():
    """One row is 2^32 - 1 positions younger than all others: it stays, and of the others, all equal, the first ones."""
    s = R.Setup([200], 1, 16, 16, 16, seed=4)
    cache = s.cache()
    marks, row = B.KVMarks(cache), row_numbers(s, 0, 0, 200).cuda()
    marks.mass.fill_(1.0)
    marks.pos.view(-1)[row], marks.pos.view(-1)[row[-1]] = -2 ** 31, 2 ** 31 - 1
    for recent in (1, 30):
        source, _ = B.kv_select(cache, B.KVBatch(s.table, s.kv_lens), marks, 30, recent)
        assert source[0, 0].tolist() == list(range(29)) + [199]
    cache.check()


@pytest.mark.parametrize("bits", [16, 8])
def test_rows_on_a_bad_page_get_no_weight_and_the_others_theirs(bits):
    s = R.Setup([200, 40, 100], 2, 64, 16, bits, seed=10)
    q = rows(3, 8, 64, 11)
    cache = s.cache()
    s.table[0, 3] = s.n_pages
    marks = marks_of(cache, 12)
    before = marks.mass.clone()
    B.attend_decode_weigh(cache, B.KVBatch(s.table, s.kv_lens), marks, q, workspace=B.alloc_attend_weigh_workspace(8, 2, 64, bits, 3, 340))
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE
    # the same sequence without that page: every row's weight, and nothing anywhere else
    without = R.Setup([1], 2, 64, 16, bits)
    without.__dict__.update(s.__dict__)
    without.table = s.table.clone()
    without.table[0, 3:-1] = s.table[0, 4:]
    without.lens = [184, 40, 100]
    check_mass(marks.mass, before, weights(without, q))


@pytest.mark.parametrize("bits", [16, 8])
def test_what_there_is_room_for_is_added(bits):
    """Scores are kept in the order of the sequences.  With room for those of the first and part of the second, the first gets all its
    weights, the second those of its first rows, and the third none."""
    lens = [700, 3000, 100]
    s = R.Setup(lens, 1, 64, 16, bits, seed=10)
    q = rows(3, 4, 64, 11)
    cache = s.cache()
    marks = marks_of(cache, 12)
    before = marks.mass.clone()
    room = B.alloc_attend_weigh_workspace(4, 1, 64, bits, 3, 1500)
    out = B.attend_decode_weigh(cache, B.KVBatch(s.table, s.kv_lens), marks, q, workspace=room)
    with pytest.raises(B.BitLinearError) as e:
        cache.check()
    assert e.value.status == B.ERR_PAGE
    check(out, *R.attend(s, q, [1] * 3, **decode_error(bits)))
    given = (marks.mass - before).flatten()
    all_of = weights(s, q)
    number, p, off = all_of[0]
    assert torch.all((given[number].double() - p).abs() <= off + 2.0 ** -23), "there is room for all of the first sequence"
    number, p, off = all_of[1]
    whole, none = (given[number].double() - p).abs() <= off + 2.0 ** -23, given[number] == 0
    assert torch.all(whole | none)
    # from the beginning of some block on (of 128 or 256 keys) nothing, in front of it everything
    end = int((~none).nonzero()[:, 1].max()) + 1
    assert torch.all(whole[:, :end]) and 256 <= end < 2500 and torch.all((p < 2.0 ** -20) | ~none | (torch.arange(3000, device="cuda") >= -(-end // 256) * 256))
    assert torch.all(given[all_of[2][0]] == 0)
    # with room for all of it, all of it
    marks.mass.copy_(before)
    B.attend_decode_weigh(cache, B.KVBatch(s.table, s.kv_lens), marks, q, workspace=B.alloc_attend_weigh_workspace(4, 1, 64, bits, 3, sum(lens)))
    cache.check()
    check_mass(marks.mass, before, all_of)
