"""Checks of the adapter linear, the rotated append and the attention over a cache in 4 bits that
need no GPU: the library exports what include/rocs_layer.h declares and refuses bad arguments before
any HIP call, and ops.py refuses what it documents."""

import ctypes
import os
import re

import pytest
import torch

from oracle import layer as oracle
from paper_2607_27744_amd import _lib, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p
FAKE = [P(0x10000000 * (i + 1)) for i in range(16)]     # never dereferenced
BAD, UNS = _lib.INVALID_ARGUMENT, _lib.UNSUPPORTED
no_gpu = pytest.mark.skipif(torch.cuda.device_count() > 0,
                            reason="fake-pointer argument checks run on hosts without a GPU")


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def test_every_declared_symbol_is_exported_and_bound(lib):
    text = open(os.path.join(ROOT, "include", "rocs_layer.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(rocs_[a-z0-9_]+)\s*\(", text)))
    assert sorted(_lib.LAYER_SIGNATURES) == names and len(names) == 8
    for n in names:
        assert hasattr(lib, n)


def test_sizes(lib):
    for hk, d in ((8, 128), (1, 32), (3, 96), (5, 256), (1, 64)):
        assert lib.rocs_fp4_row_bytes(hk, d) == oracle.row_bytes(hk, d)
    assert lib.rocs_fp4_row_bytes(1, 48) == 0 and lib.rocs_fp4_row_bytes(0, 64) == 0
    assert lib.rocs_fp4_row_bytes(1, 288) == 0
    assert lib.rocs_adapter_workspace_size(2, 0, 64, 64, 8, 1) == 0
    assert lib.rocs_adapter_workspace_size(2, 9, 64, 64, 257, 1) == 0
    assert lib.rocs_adapter_workspace_size(2, 9, 64, 64, 8, 1) % 256 == 0
    size = lib.rocs_paged_fp4_workspace_size
    assert size(0, 4, 8, 8, 64, 100, 1) == 0 and size(1, 1, 8, 3, 64, 100, 1) == 0
    assert size(1, 1, 8, 8, 64, 100000, 1) > 0 and size(1, 1, 8, 8, 64, 100000, 1) % 256 == 0


def _adapter(lib, **kw):
    a = dict(x=FAKE[0], xs=0, w=FAKE[1], a=FAKE[2], b=FAKE[3], scales=None, bias=None, off=FAKE[4],
             ids=FAKE[5], R=2, N=8, K=64, D=32, rank=8, count=3, dtype=1, act=0, out=FAKE[6],
             ws=FAKE[7], ws_bytes=1 << 20, stream=None)
    a.update(kw)
    return lib.rocs_adapter_linear(*a.values())


@no_gpu
@pytest.mark.parametrize("bad, status", [
    (dict(dtype=3), BAD), (dict(act=5), BAD), (dict(N=-1), BAD), (dict(K=0), BAD), (dict(rank=0), BAD),
    (dict(rank=257), UNS), (dict(K=1 << 22), UNS), (dict(N=1 << 31), UNS), (dict(N=1 << 28), UNS),
    (dict(R=1 << 23), UNS), (dict(N=1 << 22, D=1 << 20, ws_bytes=1 << 40), UNS), (dict(xs=63), BAD),
    (dict(R=0), BAD), (dict(x=None), BAD), (dict(w=None), BAD), (dict(a=None), BAD), (dict(b=None), BAD),
    (dict(off=None), BAD), (dict(ids=None), BAD), (dict(out=None), BAD), (dict(count=-1), BAD),
    (dict(ws=None), _lib.WORKSPACE_TOO_SMALL), (dict(ws_bytes=8), _lib.WORKSPACE_TOO_SMALL),
    (dict(ws=P(0x70000010)), BAD), (dict(out=FAKE[0]), BAD), (dict(out=FAKE[3]), BAD),
    (dict(ws=FAKE[1]), BAD), (dict(ws=FAKE[6]), BAD), (dict(out=FAKE[5]), BAD), (dict(N=0), _lib.OK),
    (dict(N=0, R=0), _lib.OK)])
def test_adapter_refusals(lib, bad, status):
    assert _adapter(lib, **bad) == status
    assert (lib.rocs_last_error_message() == b"") == (status == _lib.OK)


@no_gpu
@pytest.mark.parametrize("n, r, rank, k, d", [
    (80_000_000, 5_000_000, 136, 8, 4), (80_000_000, 5_000_000, 256, 8, 4), (88_000_000, 5_500_000, 200, 16, 8),
    (80_000_000, 5_000_000, 64, 8, 4), (80_000_000, 5_000_000, 32, 8, 4), (250_000_000, 1, 256, 8, 4),
    (1, (1 << 23) - 2, 256, 8, 4), ((1 << 28) - 64, 1, 16, 8, 4), (1 << 26, 64, 16, 8, 31 * 128), (8_000, 500, 16, 8, 4)])
def test_adapter_sizes_within_the_limits_are_launched(lib, n, r, rank, k, d):
    # Calls that the limits allow fit a launch's grid: they fail here for want of a GPU alone.
    far = [P((i + 1) << 44) for i in range(8)]
    need = lib.rocs_adapter_workspace_size(r, n, k, d, rank, 1)
    assert _adapter(lib, x=far[0], w=far[1], a=far[2], b=far[3], off=far[4], ids=far[5], out=far[6], ws=far[7],
                    R=r, N=n, K=k, D=d, rank=rank, ws_bytes=need) not in (_lib.OK, BAD, UNS)
    assert b"grid" not in lib.rocs_last_error_message()


@no_gpu
@pytest.mark.parametrize("sizes", [dict(N=(1 << 28) - 63), dict(N=(1 << 28) - 32, R=1), dict(N=33, R=(1 << 23) - 2),
                                   dict(N=1 << 26, D=32 * 128), dict(N=(1 << 26) - 127, D=31 * 128 + 1)])
def test_adapter_sizes_past_the_limits(lib, sizes):
    far = [P((i + 1) << 44) for i in range(8)]
    assert _adapter(lib, x=far[0], w=far[1], a=far[2], b=far[3], off=far[4], ids=far[5], out=far[6], ws=far[7],
                    ws_bytes=1 << 42, **sizes) == UNS
    assert b"batch too large" in lib.rocs_last_error_message()


def _append(lib, **kw):
    a = dict(q=FAKE[0], qs=0, k=FAKE[1], v=FAKE[2], ks=0, rows=FAKE[3], freqs=FAKE[4], rot=64, inter=0,
             pos=None, off=FAKE[5], slots=FAKE[6], lens=FAKE[7], R=2, S=4, M=8, H=4, Hk=2, D=64, dtype=1,
             pool=FAKE[8], pool_rows=64, form=0, qo=FAKE[9], stream=None)
    a.update(kw)
    return lib.rocs_cache_append(*a.values())


@no_gpu
@pytest.mark.parametrize("bad, status", [
    (dict(dtype=3), BAD), (dict(form=2), BAD), (dict(M=-1), BAD), (dict(D=257), UNS), (dict(rot=63), BAD),
    (dict(rot=66), BAD), (dict(rot=-2), BAD), (dict(inter=2), BAD), (dict(freqs=None), BAD),
    (dict(lens=None), BAD), (dict(off=None), BAD), (dict(R=0), BAD), (dict(S=0), BAD),
    (dict(slots=None, S=1), BAD), (dict(k=None), BAD), (dict(v=None), BAD), (dict(rows=None), BAD),
    (dict(pool=None), BAD), (dict(qo=None), BAD), (dict(H=0), BAD), (dict(Hk=0), BAD),
    (dict(ks=127), BAD), (dict(qs=255), BAD), (dict(pool_rows=-1), BAD), (dict(pool_rows=1 << 31), UNS),
    (dict(D=48, rot=48, form=1), UNS), (dict(form=1, pool=P(0x80000008)), BAD),
    (dict(pool=FAKE[1]), BAD), (dict(pool=FAKE[3]), BAD), (dict(qo=FAKE[0]), BAD), (dict(qo=FAKE[8]), BAD),
    (dict(qo=FAKE[7]), BAD), (dict(M=1 << 24), UNS), (dict(M=1 << 20, H=2048), UNS), (dict(M=0), _lib.OK)])
def test_append_refusals(lib, bad, status):
    assert _append(lib, **bad) == status
    assert (lib.rocs_last_error_message() == b"") == (status == _lib.OK)


@no_gpu
def test_rotate_and_read_refusals(lib):
    def rotate(**kw):
        a = dict(x=FAKE[0], xs=0, freqs=FAKE[1], rot=64, inter=0, pos=FAKE[2], off=None, slots=None,
                 lens=None, R=0, S=0, M=8, H=4, D=64, dtype=1, out=FAKE[3], stream=None)
        a.update(kw)
        return lib.rocs_rotate(*a.values())

    for bad in (dict(pos=None), dict(x=None), dict(out=None), dict(out=FAKE[0]), dict(H=0), dict(xs=255),
                dict(rot=128), dict(slots=FAKE[4]), dict(dtype=9), dict(out=FAKE[2])):
        assert rotate(**bad) == BAD, bad
    assert rotate(M=0) == _lib.OK

    def read(**kw):
        a = dict(rows=FAKE[0], M=4, pool=FAKE[1], pool_rows=64, Hk=2, D=64, dtype=1, out=FAKE[2],
                 stream=None)
        a.update(kw)
        return lib.rocs_cache_read_fp4(*a.values())

    for bad in (dict(rows=None), dict(pool=None), dict(out=None), dict(Hk=0), dict(dtype=9),
                dict(out=FAKE[1]), dict(out=FAKE[0]), dict(out=P(0x30000008)), dict(M=-1)):
        assert read(**bad) == BAD, bad
    assert read(D=48) == UNS and read(pool_rows=1 << 31) == UNS and read(M=0) == _lib.OK


def _paged(lib, **kw):
    a = dict(q=FAKE[0], qs=0, pages=FAKE[1], table=FAKE[2], W=4, lens=FAKE[3], slots=None, S=2,
             qo=FAKE[4], prefix=None, slopes=None, R=2, N=2, P=8, page=16, H=4, Hk=2, D=64, scale=0.0,
             cap=0.0, causal=1, most=0, dtype=1, out=FAKE[5], ws=None, ws_bytes=0, stream=None)
    a.update(kw)
    return lib.rocs_paged_attention_fp4(*a.values())


@no_gpu
@pytest.mark.parametrize("bad, status", [
    (dict(dtype=7), BAD), (dict(Hk=3), BAD), (dict(causal=2), BAD), (dict(cap=-1.0), BAD),
    (dict(cap=float("nan")), BAD), (dict(D=48), UNS), (dict(D=288), UNS), (dict(qs=64), BAD),
    (dict(W=0), BAD), (dict(P=0), BAD), (dict(page=0), BAD), (dict(W=1 << 28), UNS),
    (dict(P=1 << 28), UNS), (dict(S=1), BAD), (dict(S=0), BAD), (dict(table=None), BAD),
    (dict(q=None), BAD), (dict(pages=None), BAD), (dict(pages=P(0x20000008)), BAD), (dict(out=FAKE[1]), BAD),
    (dict(out=FAKE[2]), BAD), (dict(out=FAKE[0]), BAD), (dict(R=0), BAD), (dict(most=-1), BAD),
    (dict(W=10000), _lib.WORKSPACE_TOO_SMALL), (dict(W=10000, ws=P(0x90000010), ws_bytes=1 << 30), BAD),
    (dict(W=10000, ws=FAKE[1], ws_bytes=1 << 30), BAD), (dict(N=0), _lib.OK)])
def test_paged_refusals(lib, bad, status):
    assert _paged(lib, **bad) == status
    assert (lib.rocs_last_error_message() == b"") == (status == _lib.OK)


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def _i(n):
    return torch.zeros(n, dtype=torch.int32)


def test_ops_adapter_checks():
    ok = dict(x=_t(6, 16), w=_t(8, 16), a=_t(2, 4, 16), b=_t(2, 8, 4), offsets=_i(3), adapter_ids=_i(2))
    for bad, match in ((dict(w=_t(8, 15)), r"\[D, K\]"), (dict(a=_t(2, 4, 15)), "rank"),
                       (dict(b=_t(2, 8, 5)), "rank"), (dict(b=_t(3, 8, 4)), "rank"),
                       (dict(a=_t(2, 4, 16, dtype=torch.float32)), "one dtype"),
                       (dict(x=_t(6, 16, dtype=torch.float16)), "unsupported"),
                       (dict(w=_t(16, 8).t()), "contiguous"), (dict(x=_t(16, 6).t()), "dense"),
                       (dict(offsets=_i(3).long()), "int32"), (dict(adapter_ids=_i(3)), "adapter_ids"),
                       (dict(scales=_t(2)), "scales"), (dict(bias=_t(7, dtype=torch.float32)), "bias"),
                       (dict(activation="gelu"), "activation"), (dict(out=_t(6, 9)), "out must"),
                       (dict(), "on the GPU")):
        with pytest.raises((ValueError, TypeError), match=match):
            ops.adapter_linear(**{**ok, **bad})


def test_ops_append_checks():
    f = torch.zeros(16)
    ok = dict(k=_t(6, 2, 32), v=_t(6, 2, 32), rows=_i(6), pool=_t(3, 4, 2, 2, 32), freqs=f, offsets=_i(3),
              slots=_i(2), lens=_i(5))
    for bad, match in ((dict(v=_t(6, 2, 31)), "k and v"), (dict(rows=_i(5)), "rows"),
                       (dict(freqs=torch.zeros(17)), "rot_dim"), (dict(freqs=f.double()), "freqs"),
                       (dict(lens=None), "needs positions"), (dict(offsets=None), "need offsets"),
                       (dict(slots=_i(3)), "slots"), (dict(slots=None, lens=_i(1)), "R <= slots"),
                       (dict(pool=_t(3, 4, 2, 2, 31)), "pool must"), (dict(pool=_t(3, 4, 128)), "pool must"),
                       (dict(pool=_t(3, 4, 2, 2, 32, dtype=torch.float32)), "pool must"),
                       (dict(pool=_t(3, 4, 100, dtype=torch.uint8)), "4 bits"),
                       (dict(q=_t(5, 4, 32)), "q must"), (dict(q_out=_t(6, 4, 32)), "q_out needs"),
                       (dict(q=_t(6, 4, 32), q_out=_t(6, 4, 31)), "q_out must"),
                       (dict(interleaved=2), "interleaved"), (dict(positions=_i(4)), "positions"),
                       (dict(), "on the GPU")):
        with pytest.raises(ValueError, match=match):
            ops.cache_append(**{**ok, **bad})
    with pytest.raises(ValueError, match="multiple of 32"):
        ops.cache_append(_t(6, 2, 24), _t(6, 2, 24), _i(6), _t(3, 4, 64, dtype=torch.uint8))
    with pytest.raises(ValueError, match="needs positions"):
        ops.rotate(_t(6, 2, 32), f)
    with pytest.raises(ValueError, match="M, heads, d"):
        ops.rotate(_t(6, 32), f, positions=_i(6))
    with pytest.raises(ValueError, match="on the GPU"):
        ops.rotate(_t(6, 2, 32), f, positions=_i(6))
    with pytest.raises(ValueError, match="dtype"):
        ops.cache_read_fp4(_i(4), _t(3, 4, 80, dtype=torch.uint8), 1, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="4 bits"):
        ops.cache_read_fp4(_i(4), _t(3, 4, 81, dtype=torch.uint8), 1, 64)


def test_ops_paged_fp4_checks():
    ok = dict(q=_t(2, 4, 64), pages=_t(3, 16, 80, dtype=torch.uint8), page_table=_t(2, 5).int(),
              kv_lens=_i(2), q_offsets=_i(3), kv_heads=1)
    for bad, match in ((dict(q=_t(2, 4)), "heads, d"), (dict(kv_heads=3), "divide"), (dict(kv_heads=2), "4 bits"),
                       (dict(q=_t(2, 4, 48)), "multiple of 32"), (dict(pages=_t(3, 16, 80)), "4 bits"),
                       (dict(page_table=_i(5)), "page_table"), (dict(kv_lens=_i(3)), "kv_lens"),
                       (dict(slots=_i(1)), "slots"), (dict(q_offsets=_i(4)), "R <= slots"),
                       (dict(cap=-1.0), "cap"), (dict(slopes=torch.zeros(3)), "slopes"),
                       (dict(causal=2), "causal"), (dict(out=_t(2, 4, 32)), "out must"), (dict(), "on the GPU")):
        with pytest.raises(ValueError, match=match):
            ops.paged_attention_fp4(**{**ok, **bad})


def test_fp4_workspaces_have_a_bound(lib):
    # The header's bound for one workspace under calls of many sizes.
    size, tight = lib.rocs_paged_fp4_workspace_size, 0.0
    for dtype, d in ((1, 128), (1, 64), (1, 96), (1, 160), (0, 64)):
        c = 524288 if dtype == 1 and d <= 128 else 8192
        for h, hk in ((8, 8), (8, 2), (16, 1), (64, 8), (5, 5)):
            for n in (1, 3, 40, 500, 7000):
                for most in (1, 300, 5000, 70000, 3000000):
                    bound = 4 * (d + 2) * min(h * n * min(256, -(-most // 256)), c) + 512
                    for r in (1, 2, 7, 64, 129, 1000, 7000):
                        need = size(r, n, h, hk, d, most, dtype)
                        assert need <= bound, (dtype, d, h, hk, n, most, r)
                        tight = max(tight, need / bound)
    assert tight > 0.5
