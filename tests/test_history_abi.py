"""Checks of the history attention and the cache's page operators that need no GPU: the library
exports what include/rocs_history.h declares and refuses bad arguments before any HIP call, and
ops.py refuses what it documents."""

import ctypes
import os
import re

import pytest
import torch

from paper_2607_27744_amd import _lib, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p
FAKE = [P(0x1000000 * (i + 1)) for i in range(14)]     # never dereferenced
no_gpu = pytest.mark.skipif(torch.cuda.device_count() > 0,
                            reason="fake-pointer argument checks run on hosts without a GPU")


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def test_every_declared_symbol_is_exported_and_bound(lib):
    text = open(os.path.join(ROOT, "include", "rocs_history.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(rocs_[a-z0-9_]+)\s*\(", text)))
    assert sorted(_lib.HISTORY_SIGNATURES) == names and len(names) == 10
    for n in names:
        assert hasattr(lib, n)


def test_workspace_sizes(lib):
    size = lib.rocs_history_workspace_size
    assert size(0, 4, 8, 8, 64, 100, 1) == 0 and size(4, 0, 8, 8, 64, 100, 1) == 0
    assert size(1, 1, 8, 3, 64, 100, 1) == 0                 # no such heads
    assert size(1, 1, 8, 8, 64, 40, 1) == 0                  # too short to split
    assert size(1, 1, 8, 8, 64, 100000, 1) % 256 == 0 and size(1, 1, 8, 8, 64, 100000, 1) > 0
    assert size(4096, 4096 * 128, 8, 8, 64, 100000, 1) == 0  # tiles enough
    assert lib.rocs_cache_workspace_size(-1, 5) == 0 and lib.rocs_cache_workspace_size(0, 0) == 0
    assert lib.rocs_cache_workspace_size(10, 5000) >= 4 * 15000


def _packed(lib, **kw):
    a = dict(q=FAKE[0], qs=0, k=FAKE[1], v=FAKE[2], ks=0, qo=FAKE[3], ko=FAKE[4], prefix=None,
             qd=None, kd=None, slopes=None, R=2, N=8, L=64, H=4, Hk=2, D=64, scale=0.0, cap=0.0,
             causal=1, most=64, dtype=1, out=FAKE[5], ws=None, ws_bytes=0, stream=None)
    a.update(kw)
    return lib.rocs_history_attention(*a.values())


@no_gpu
@pytest.mark.parametrize("bad, status", [
    (dict(dtype=7), _lib.INVALID_ARGUMENT), (dict(Hk=3), _lib.INVALID_ARGUMENT),
    (dict(causal=2), _lib.INVALID_ARGUMENT), (dict(cap=-1.0), _lib.INVALID_ARGUMENT),
    (dict(cap=1e-38), _lib.INVALID_ARGUMENT),
    (dict(cap=float("nan")), _lib.INVALID_ARGUMENT), (dict(cap=float("inf")), _lib.INVALID_ARGUMENT),
    (dict(D=257), _lib.UNSUPPORTED), (dict(N=1 << 30), _lib.UNSUPPORTED),
    (dict(qs=64), _lib.INVALID_ARGUMENT), (dict(ks=64), _lib.INVALID_ARGUMENT),
    (dict(R=0), _lib.INVALID_ARGUMENT), (dict(q=None), _lib.INVALID_ARGUMENT),
    (dict(k=None), _lib.INVALID_ARGUMENT), (dict(qd=FAKE[6]), _lib.INVALID_ARGUMENT),
    (dict(out=FAKE[0]), _lib.INVALID_ARGUMENT), (dict(out=FAKE[2]), _lib.INVALID_ARGUMENT),
    (dict(out=FAKE[3]), _lib.INVALID_ARGUMENT), (dict(L=-1), _lib.INVALID_ARGUMENT),
    (dict(qd=FAKE[6], kd=FAKE[7], out=P(FAKE[7].value + 128)), _lib.INVALID_ARGUMENT),
    (dict(most=-1), _lib.INVALID_ARGUMENT),
    (dict(most=100000), _lib.WORKSPACE_TOO_SMALL),
    (dict(most=100000, ws=P(0x90000010), ws_bytes=1 << 30), _lib.INVALID_ARGUMENT),
    (dict(most=100000, ws=FAKE[1], ws_bytes=1 << 30), _lib.INVALID_ARGUMENT),
    (dict(N=0), _lib.OK)])
def test_history_refusals(lib, bad, status):
    assert _packed(lib, **bad) == status
    assert (lib.rocs_last_error_message() == b"") == (status == _lib.OK)


def _paged(lib, **kw):
    a = dict(q=FAKE[0], qs=0, k=FAKE[1], v=FAKE[2], ps=0, ks=0, table=FAKE[3], W=4, lens=FAKE[4],
             slots=None, S=2, qo=FAKE[5], prefix=None, slopes=None, R=2, N=2, P=8, page=16, H=4,
             Hk=2, D=64, scale=0.0, cap=0.0, causal=1, most=0, dtype=1, out=FAKE[6], ws=None,
             ws_bytes=0, stream=None)
    a.update(kw)
    return lib.rocs_paged_attention(*a.values())


@no_gpu
@pytest.mark.parametrize("bad, status", [
    (dict(W=0), _lib.INVALID_ARGUMENT), (dict(P=0), _lib.INVALID_ARGUMENT),
    (dict(page=0), _lib.INVALID_ARGUMENT), (dict(ps=100), _lib.INVALID_ARGUMENT),
    (dict(W=1 << 28), _lib.UNSUPPORTED), (dict(S=1), _lib.INVALID_ARGUMENT),
    (dict(S=0), _lib.INVALID_ARGUMENT), (dict(table=None), _lib.INVALID_ARGUMENT),
    (dict(out=FAKE[1]), _lib.INVALID_ARGUMENT), (dict(out=FAKE[3]), _lib.INVALID_ARGUMENT),
    (dict(N=0), _lib.OK)])
def test_paged_refusals(lib, bad, status):
    assert _paged(lib, **bad) == status


@no_gpu
def test_cache_refusals(lib):
    ws = dict(ws=FAKE[9], ws_bytes=1 << 20, stream=None)

    def reserve(**kw):
        a = dict(slots=FAKE[0], off=FAKE[1], n=2, m=4, table=FAKE[2], W=4, lens=FAKE[3], S=8,
                 refs=FAKE[4], P=8, page=16, rows=FAKE[5], status=FAKE[6], **ws)
        a.update(kw)
        return lib.rocs_cache_reserve(*a.values())

    def fork(**kw):
        a = dict(par=FAKE[0], kid=FAKE[1], n=2, table=FAKE[2], W=4, lens=FAKE[3], S=8, refs=FAKE[4],
                 P=8, page=16, pool=FAKE[7], layers=1, row=64, status=FAKE[6], **ws)
        a.update(kw)
        return lib.rocs_cache_fork(*a.values())

    def compact(**kw):
        a = dict(table=FAKE[2], W=4, S=8, refs=FAKE[4], P=8, page=16, pool=FAKE[7], layers=1, row=64,
                 status=FAKE[6], **ws)
        a.update(kw)
        return lib.rocs_cache_compact(*a.values())

    for call in (reserve, fork, compact):
        assert call(P=0) == call(W=0) == call(S=0) == call(page=0) == _lib.INVALID_ARGUMENT
        assert call(S=(1 << 18) + 1) == call(P=1 << 28) == call(W=1 << 28) == _lib.UNSUPPORTED
        assert call(table=None) == call(refs=None) == call(status=None) == _lib.INVALID_ARGUMENT
        assert call(ws=None) == call(ws_bytes=16) == _lib.WORKSPACE_TOO_SMALL
        assert call(ws=P(0xa0000010)) == _lib.INVALID_ARGUMENT
        assert call(refs=FAKE[2]) == call(status=FAKE[4]) == _lib.INVALID_ARGUMENT
    assert reserve(n=(1 << 30) + 1) == fork(n=(1 << 30) + 1) == _lib.UNSUPPORTED
    for out in (FAKE[0], FAKE[1], FAKE[2], FAKE[3], FAKE[4], FAKE[6], FAKE[9]):
        assert reserve(rows=out) == _lib.INVALID_ARGUMENT       # rows over another array
    assert reserve(slots=FAKE[3]) == reserve(off=FAKE[4]) == _lib.INVALID_ARGUMENT
    assert fork(par=FAKE[2]) == fork(kid=FAKE[6]) == fork(kid=FAKE[7]) == _lib.INVALID_ARGUMENT
    assert reserve(n=-1) == reserve(m=-1) == reserve(n=0) == reserve(rows=None) == _lib.INVALID_ARGUMENT
    assert fork(layers=0) == fork(row=0) == fork(pool=None) == fork(par=None) == _lib.INVALID_ARGUMENT
    assert compact(layers=0) == compact(pool=FAKE[4]) == _lib.INVALID_ARGUMENT
    free = lambda n=2, slots=FAKE[0], table=FAKE[2]: lib.rocs_cache_free(   # noqa: E731
        slots, n, table, 4, FAKE[3], 8, FAKE[4], 8, 16, None)
    assert free(n=-1) == free(slots=None) == free(table=None) == _lib.INVALID_ARGUMENT
    assert free(slots=FAKE[3]) == free(slots=FAKE[4]) == _lib.INVALID_ARGUMENT
    assert free(n=1 << 24) == _lib.UNSUPPORTED and free(n=0) == _lib.OK
    write = lambda x=FAKE[0], xs=64, m=4, n=8, row=64, pool=FAKE[2]: lib.rocs_cache_write(  # noqa: E731
        x, xs, FAKE[1], m, pool, n, row, None)
    assert write(xs=32) == write(n=0) == write(row=0) == write(x=None) == _lib.INVALID_ARGUMENT
    assert write(pool=FAKE[0]) == _lib.INVALID_ARGUMENT and write(m=0) == _lib.OK
    copy = lambda src=FAKE[2], sp=8, dst=FAKE[2], dp=8, n=2, by=64: lib.rocs_cache_copy(    # noqa: E731
        FAKE[0], FAKE[1], n, src, sp, dst, dp, 1, by, None)
    assert copy(sp=0) == copy(by=0) == copy(dst=None) == copy(dp=4) == _lib.INVALID_ARGUMENT
    assert copy(n=0) == _lib.OK


BF = torch.bfloat16
OFF = torch.tensor([0, 2, 4], dtype=torch.int32)


def _history_args(**kw):
    a = dict(q=torch.zeros(4, 4, 64, dtype=BF), k=torch.zeros(4, 2, 64, dtype=BF),
             v=torch.zeros(4, 2, 64, dtype=BF), q_offsets=OFF, kv_offsets=OFF)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad, match", [
    (dict(q=torch.zeros(4, 256, dtype=BF)), "q must be"),
    (dict(q=torch.zeros(4, 3, 64, dtype=BF)), "heads that divide"),
    (dict(v=torch.zeros(3, 2, 64, dtype=BF)), "k and v must be"),
    (dict(k=torch.zeros(4, 2, 64), v=torch.zeros(4, 2, 64)), "one dtype"),
    (dict(q_offsets=OFF.long()), "offsets"), (dict(kv_offsets=OFF[:2]), "offsets"),
    (dict(prefix_lens=OFF), "prefix_lens"), (dict(q_docs=OFF), "go together"),
    (dict(q_docs=torch.zeros(4, dtype=torch.int32), kv_docs=OFF), "kv_docs"),
    (dict(slopes=torch.zeros(4, dtype=BF)), "slopes"), (dict(cap=-1.0), "cap"),
    (dict(cap=float("nan")), "cap"), (dict(max_kv_len=-1), "max_kv_len"),
    (dict(out=torch.zeros(4, 4, 64)), "out must be"),
    (dict(q=torch.zeros(4, 64, 4, dtype=BF).transpose(1, 2)), "q rows must be dense"),
    (dict(k=torch.zeros(1, 2, 64, dtype=BF).expand(4, 2, 64)), "must not overlap"),
    (dict(v=torch.zeros(4, 4, 64, dtype=BF)[:, :2]), "row stride"),
    (dict(), "on the GPU")])
def test_history_attention_refuses(bad, match):
    with pytest.raises(ValueError, match=match):
        ops.history_attention(**_history_args(**bad))


@pytest.mark.parametrize("bad, match", [
    (dict(k_pages=torch.zeros(8, 2, 64, dtype=BF)), "k_pages and v_pages"),
    (dict(page_table=torch.zeros(2, 4)), "page_table"), (dict(kv_lens=OFF), "kv_lens"),
    (dict(slots=OFF), "slots"), (dict(q_offsets=torch.zeros(4, dtype=torch.int32)), "R <= slots"),
    (dict(v_pages=torch.zeros(8, 16, 4, 64, dtype=BF)[:, :, :2]), "share strides"),
    (dict(k_pages=torch.zeros(1, 16, 2, 64, dtype=BF).expand(8, 16, 2, 64)), "share|overlap"),
    (dict(), "on the GPU")])
def test_paged_attention_refuses(bad, match):
    a = dict(q=torch.zeros(4, 4, 64, dtype=BF), k_pages=torch.zeros(8, 16, 2, 64, dtype=BF),
             v_pages=torch.zeros(8, 16, 2, 64, dtype=BF),
             page_table=torch.zeros(2, 4, dtype=torch.int32),
             kv_lens=torch.zeros(2, dtype=torch.int32), q_offsets=OFF)
    a.update(bad)
    with pytest.raises(ValueError, match=match):
        ops.paged_attention(**a)


def test_cache_operators_refuse():
    pool, table, lens, refs = ops.cache_pool(2, 8, 16, 2, 4, slots=3, table_width=4, device="cpu")
    assert pool.shape == (2, 8, 16, 2, 2, 4) and int(table.max()) == -1
    slots, off = torch.tensor([0, 1], dtype=torch.int32), OFF
    for bad, match in ((dict(slots=slots.long()), "slots"), (dict(row_offsets=off[:2]), "offsets"),
                       (dict(num_rows=-1), "num_rows"), (dict(page_size=0), "page_size"),
                       (dict(lens=slots), "lens"), (dict(refs=refs.float()), "refs"),
                       (dict(page_table=table[:, :2]), "page_table"), (dict(), "on the GPU")):
        a = dict(slots=slots, row_offsets=off, num_rows=4, page_table=table, lens=lens, refs=refs,
                 page_size=16)
        a.update(bad)
        with pytest.raises(ValueError, match=match):
            ops.cache_reserve(**a)
    x, rows = torch.zeros(4, 16, dtype=BF), torch.zeros(4, dtype=torch.int32)
    for a, match in (((x.float(), rows, pool[0]), "one dtype"), ((x[:, :8], rows, pool[0]), "width"),
                     ((x, rows[:2], pool[0]), "rows"), ((x, rows, pool[0].transpose(0, 1)), "pool"),
                     ((x.t().contiguous().t(), rows, pool[0]), "dense"),
                     ((x, rows, pool[0]), "on the GPU")):
        with pytest.raises(ValueError, match=match):
            ops.cache_write(*a)
    for a, match in (((slots, off, table, lens, refs, pool), "children"),
                     ((slots, slots, table, lens, refs, pool[:, :4]), "pool"),
                     ((slots, slots, table, lens, refs, pool), "on the GPU")):
        with pytest.raises(ValueError, match=match):
            ops.cache_fork(*a)
    with pytest.raises(ValueError, match="page_size"):
        ops.cache_free(slots, table, lens, refs, 0)
    with pytest.raises(ValueError, match="on the GPU"):
        ops.cache_free(slots, table, lens, refs, 16)
    with pytest.raises(ValueError, match="pool"):
        ops.cache_compact(table, lens, refs, pool[0])
    with pytest.raises(ValueError, match="on the GPU"):
        ops.cache_compact(table, lens, refs, pool)
    with pytest.raises(ValueError, match="same layers"):
        ops.cache_copy(slots, slots, pool, pool[:1])
    with pytest.raises(ValueError, match="dst_pages"):
        ops.cache_copy(slots, off, pool)


def test_cache_check_reads_the_status():
    assert ops.cache_check(torch.tensor([0, 7])) == 7
    for status, match in (([1, 3], "3 pages"), ([2, 0], "table"), ([3, 0], "slot")):
        with pytest.raises(ops.RocsError, match=match):
            ops.cache_check(torch.tensor(status))
