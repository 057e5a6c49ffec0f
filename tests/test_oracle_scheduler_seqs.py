"""The scheduling oracle where a strategy's GPU store has room for a number of sequences only (CPU)."""
import pytest

from oracle import scheduler as sc

PROMPTS, OUTS = [5, 20, 7, 33, 4, 18, 9, 2], [3, 1, 4, 2, 6, 2, 3, 5]


def _run(**kw):
    return sc.simulate(PROMPTS, OUTS, 200, 50, 60, 8, **kw)


def test_room_for_all_changes_nothing():
    assert _run(prefill_seqs=8, decode_seqs=8) == _run()


@pytest.mark.parametrize("p,d", [(1, 1), (2, 3), (3, 8)])
def test_batches_and_admissions_stay_within_the_room(p, d):
    trace, stats = _run(prefill_seqs=p, decode_seqs=d)
    batches = [ids for code, ids in trace if code == sc.PREFILL]
    assert max(map(len, batches)) == min(p, 3) and [r for b in batches for r in b] == list(range(8))
    on_board, most = set(), 0
    for code, ids in trace:
        if code == sc.SWAP_IN:
            on_board |= set(ids)
        elif code == sc.FINISH:
            on_board -= set(ids)
        most = max(most, len(on_board))
    assert most <= d and stats["tokens"] == sum(OUTS)


def test_a_request_that_is_finished_by_its_prefill_takes_room_in_its_batch():
    trace, _ = sc.simulate([4, 4, 4, 4], [1, 2, 1, 2], 100, 50, 100, 8, prefill_seqs=2)
    assert [ids for code, ids in trace if code == sc.PREFILL] == [[0, 1], [2, 3]]
