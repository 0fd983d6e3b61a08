"""What adapted_step does with slots and offsets that do not fit, with every operator replaced by a
stand-in on the CPU: an index out of range that torch looks up itself ends the process on a GPU."""

from types import SimpleNamespace

import pytest
import torch

from paper_2607_27744_amd import ops, pipelines


@pytest.fixture
def step(monkeypatch):
    """Calls adapted_step over 4 slots of 5, 0, 9 and 2 rows; returns the candidates' positions."""
    seen = {}

    def rotate(x, freqs, *, positions):
        seen["positions"] = positions
        return x

    def request_ids(offsets, n):
        return torch.repeat_interleave(torch.arange(offsets.numel() - 1), offsets.diff()).int()

    def reserve(slots, offsets, m, *cache):
        seen["reserved"] = True
        return torch.full((m,), -1), torch.tensor([3, 0])

    for name, fn in dict(adapter_linear=lambda x, w, *a, **k: x @ w.T, cache_reserve=reserve,
                         cache_append=lambda k, v, *a, q, **kw: q, ikbo_linear=lambda x, w: x @ w.T,
                         paged_attention_fp4=lambda q, *a, **k: q, rotate=rotate,
                         request_ids=request_ids).items():
        monkeypatch.setattr(ops, name, fn)
    p = SimpleNamespace(h=2, hk=1, d=4, page=16, wqkv=torch.ones(16, 3), wq_c=torch.ones(8, 3), a=None, b=None,
                        scales=None, freqs=None, pool=[None], table=None, refs=None,
                        lens=torch.tensor([5, 0, 9, 2], dtype=torch.int32))

    def call(slots, counts):
        i32 = lambda v: torch.tensor(v, dtype=torch.int32)   # noqa: E731
        off = i32([0, *torch.tensor(counts).cumsum(0).tolist()])
        pipelines.adapted_step(p, i32(slots), i32([0] * len(slots)), torch.ones(len(slots), 3),
                               i32(list(range(len(slots) + 1))), torch.ones(sum(counts), 3), off)
        return seen["positions"].tolist()
    call.seen = seen
    return call


def test_candidates_stand_behind_the_history(step):
    assert step([2, 0, 1], [2, 1, 3]) == [9, 9, 5, 0, 0, 0]


@pytest.mark.parametrize("bad", [4, 99, 2 ** 31 - 1, -1, -4, -5, -2 ** 31])
def test_a_slot_out_of_range_is_clamped(step, bad):
    # cache_reserve reports it in its status; the rest of the step stays within the cache.
    got = step([2, bad], [1, 2])
    assert got[0] == 9 and got[1:] in ([5, 5], [2, 2])


@pytest.mark.parametrize("counts", [[2], [1, 1, 4]])
def test_candidates_of_other_requests_are_refused(step, counts):
    with pytest.raises(ValueError, match="cand_offsets"):
        step([2, 0], counts)
    assert "reserved" not in step.seen
