"""GPU: the history operators together, as a serving loop uses them: batches of new events are
appended to a paged cache, encoded over it, and candidates attend over the pages, while slots are
forked, freed and compacted in between. Every batch is compared with the oracle's attention over
the whole histories (bf16 at operator boundaries), and with the packed operators."""

import numpy as np
import pytest
import torch

from gpu_util import assert_close, dev_bf16, dev_i32, host
from oracle import history as oracle
from oracle import ikbo
from oracle.bf16 import round_bf16
from paper_2607_27744_amd import ops, pipelines
from paper_2607_27744_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _project(x, w, heads, d):
    return round_bf16(ikbo.linear(x, w)).reshape(x.shape[0], heads, d)


@pytest.mark.parametrize("head_dim, kv_heads, page", [(64, 2, 16), (128, 4, 64), (32, 1, 24)])
def test_ranking_over_cached_histories(gpu_lib, head_dim, kv_heads, page):
    counts = [33, 1, 0, 140, 7]
    events = [[70, 1, 40, 129, 0], [1, 1, 1, 1, 1], [9, 0, 3, 64, 2], [1, 1, 1, 1, 1]]
    w = wl.history_case(counts, events, heads=4, kv_heads=kv_heads, head_dim=head_dim, seed=3)
    p = pipelines.prepare_history_cache(w, pages=90, page_size=page, table_width=20, slots=8)
    hist = {s: np.zeros((0, 256)) for s in range(8)}          # the features behind every slot
    slot_of = np.array([6, 0, 3, 5, 1])
    for i, b in enumerate(w.batches):
        slots = dev_i32(slot_of)
        got = pipelines.history_step(p, slots, dev_bf16(b.s), dev_i32(b.offsets), dev_bf16(b.e_c),
                                     dev_i32(b.cand_offsets), max_kv_len=None if i % 2 else 400)
        ops.cache_check(got["status"])
        for r, s in enumerate(slot_of):
            hist[s] = np.concatenate([hist[s], b.s[b.offsets[r]:b.offsets[r + 1]]])
        seq = [hist[s] for s in slot_of]
        lens = [x.shape[0] for x in seq]
        kv = _project(np.concatenate(seq), w.wkv, 2 * kv_heads, head_dim)
        k, v = kv[:, :kv_heads], kv[:, kv_heads:]
        new = np.diff(b.offsets)
        q_s, q_c = _project(b.s, w.wq_s, 4, head_dim), _project(b.e_c, w.wq_c, 4, head_dim)
        want = oracle.attention(q_s, k, v, new, lens, slopes=w.slopes)[0]
        assert_close(host(got["events"]), round_bf16(want), f"batch {i} events")
        want = oracle.attention(q_c, k, v, counts, lens, causal=False)[0]
        assert_close(host(got["candidates"]), round_bf16(want), f"batch {i} candidates")
        # The packed operators on the same rows: DCA, and the whole histories at once.
        ko = dev_i32(np.concatenate([[0], np.cumsum(lens)]))
        if kv_heads == 4:
            dca = ops.dca_attention(dev_bf16(q_c)[:, None], dev_bf16(k), dev_bf16(v),
                                    dev_i32(b.cand_offsets), ko)
            assert_close(host(got["candidates"]), host(dca)[:, 0], f"batch {i} against DCA")
        q_all = _project(np.concatenate(seq), w.wq_s, 4, head_dim)
        whole = ops.history_attention(dev_bf16(q_all), dev_bf16(k), dev_bf16(v), ko, ko,
                                      slopes=p.slopes)
        last = np.concatenate([np.arange(e - n, e) for n, e in zip(new, np.cumsum(lens))])
        if last.size:
            assert_close(host(got["events"]), host(whole)[last.astype(int)], f"batch {i} whole")
        # Between batches: a history is forked (both go on apart), one is dropped, pages move.
        if i == 1:
            ops.cache_check(ops.cache_fork(dev_i32([5, 6]), dev_i32([2, 7]), p.table, p.lens,
                                           p.refs, p.pool))
            hist[2], hist[7] = hist[5], hist[6]
            slot_of = np.array([7, 0, 3, 2, 1])               # the forks go on, ..
        if i == 2:
            ops.cache_free(dev_i32([3, 6]), p.table, p.lens, p.refs, p.page)
            hist[3], hist[6] = hist[3][:0], hist[6][:0]
            live = ops.cache_check(ops.cache_compact(p.table, p.lens, p.refs, p.pool))
            assert int((p.refs > 0).sum()) == live and not p.refs[live:].any()
            slot_of = np.array([7, 0, 3, 5, 1])               # .. and so does a parent


def test_a_failed_append_leaves_the_cache(gpu_lib):
    w = wl.history_case([2, 2], [[20, 20], [100, 1]], seed=4)
    p = pipelines.prepare_history_cache(w, pages=4, page_size=16, table_width=8)
    slots = dev_i32([0, 1])
    for i, b in enumerate(w.batches):
        got = pipelines.history_step(p, slots, dev_bf16(b.s), dev_i32(b.offsets), dev_bf16(b.e_c),
                                     dev_i32(b.cand_offsets))
        if i == 0:
            ops.cache_check(got["status"])
            kept = [t.clone() for t in (p.pool, p.table, p.lens, p.refs)]
    with pytest.raises(ops.RocsError, match="6 pages"):
        ops.cache_check(got["status"])
    assert all(torch.equal(a, b) for a, b in zip(kept, (p.pool, p.table, p.lens, p.refs)))


@pytest.mark.parametrize("name", ["history_attention", "paged_step", "history_step"])
def test_the_variants_run(gpu_lib, name):
    from paper_2607_27744_amd import variants
    line = variants.run(name, steps=2, warmup=1)
    assert line["variant"] == name and line["ms"] > 0 and name in variants.NAMES
