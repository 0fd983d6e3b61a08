"""GPU: the history layer's operators through the native call path and through the Python one: the same
values, the same refusals, whatever one argument is replaced by. Trusted device data (offsets) keeps
its sizes, or the call is refused."""

from types import SimpleNamespace

import pytest
import torch

from paper_2607_27744_amd import ops
from test_gpu_binding import BF, _off, _outcome, _r, _same, _Spy, _spoiled

pytestmark = pytest.mark.gpu
F32 = torch.float32
PYTHON = SimpleNamespace(**{n: (lambda *a: None) for n in ("adapter", "append", "paged_fp4", "rotate", "read_fp4")})


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _append(**kw):
    """cache_append into a copy of the pool; its result and the pool."""
    if torch.is_tensor(kw["pool"]):
        kw["pool"] = kw["pool"].clone()
    return ops.cache_append(**kw), kw["pool"]


def _calls():
    g = torch.Generator(device="cuda").manual_seed(0)
    qkv = _r(7, 8 * 64)
    q, k, v = (x.unflatten(1, (-1, 64)) for x in qkv.split([4 * 64, 2 * 64, 2 * 64], 1))
    off, slots, lens, rows = _off(3, 0, 4), _i32(2, 0, 3), _i32(9, 0, 30, 4, 1), _i32(5, 1, -1, 40, 33, 7, 99)
    freqs = 10.0 ** -torch.arange(32, dtype=F32, device="cuda").div(32)
    pool = torch.randint(0, 256, (4, 16, ops.fp4_row_bytes(2, 64)), dtype=torch.uint8, device="cuda", generator=g)
    pool[..., 128:136] = 120
    table = _i32(0, 3, 1, 2, 2, 1, 3, -1, 9, 0).view(5, 2)
    adapter = dict(x=_r(7, 64), w=_r(36, 64), a=_r(2, 8, 64), b=_r(2, 36, 8), offsets=off, adapter_ids=_i32(1, 0, -1))
    append = dict(k=k, v=v, rows=rows, pool=pool, freqs=freqs, q=q, offsets=off, slots=slots, lens=lens)
    paged = dict(q=q, pages=pool, page_table=table, kv_lens=lens, q_offsets=off, kv_heads=2, slots=slots)
    return {
        "adapter": (ops.adapter_linear, dict(adapter, scales=_r(2, dtype=F32), bias=_r(36, dtype=F32), activation="relu")),
        "adapter plain": (ops.adapter_linear, adapter),
        "adapter none": (ops.adapter_linear, dict(adapter, a=adapter["a"][:0], b=adapter["b"][:0])),
        "adapter odd": (ops.adapter_linear, dict(x=_r(7, 5, dtype=F32), w=_r(3, 5, dtype=F32), a=_r(2, 3, 5, dtype=F32),
                                                 b=_r(2, 3, 3, dtype=F32), offsets=off, adapter_ids=_i32(1, 0, -1))),
        "adapter empty": (ops.adapter_linear, dict(adapter, x=_r(0, 64), offsets=_off(0, 0, 0))),
        "append": (_append, append),
        "append keys": (_append, dict(append, q=None, interleaved=True)),
        "append positions": (_append, dict(k=k, v=v, rows=rows, pool=_r(4, 16, 2, 2, 64), freqs=freqs[:9],
                                           positions=_i32(0, 1, -4, 1 << 30, 7, 7, 8))),
        "append as they are": (_append, dict(k=k, v=v, rows=rows, pool=_r(4, 16, 2, 2, 64))),
        "append empty": (_append, dict(k=k[:0], v=v[:0], rows=rows[:0], pool=pool, freqs=freqs, positions=rows[:0])),
        "rotate": (ops.rotate, dict(x=q, freqs=freqs, offsets=off, slots=slots, lens=lens)),
        "rotate positions": (ops.rotate, dict(x=q, freqs=freqs, positions=rows, interleaved=True)),
        "rotate nothing": (ops.rotate, dict(x=q, freqs=None)),
        "read": (ops.cache_read_fp4, dict(rows=rows, pool=pool, kv_heads=2, head_dim=64)),
        "read f32": (ops.cache_read_fp4, dict(rows=rows, pool=pool, kv_heads=2, head_dim=64, dtype=F32)),
        "paged": (ops.paged_attention_fp4, paged),
        "paged rules": (ops.paged_attention_fp4, dict(paged, prefix_lens=_i32(1, 0, 2), slopes=_r(4, dtype=F32).abs(),
                                                      cap=20.0, max_kv_len=40, scale=0.1)),
        "paged candidates": (ops.paged_attention_fp4, dict(paged, q=q[..., :].float().contiguous(), causal=False)),
        "paged empty": (ops.paged_attention_fp4, dict(paged, q=q[:0], q_offsets=_off(0, 0, 0))),
    }


@pytest.mark.parametrize("name", sorted(_calls() if torch.cuda.is_available() else ["none"]))
def test_same_as_the_python_path(gpu_lib, name, monkeypatch):
    torch.manual_seed(0)
    fn, kw = _calls()[name]
    native = _Spy(ops._native())
    cases = [("", kw)]
    for key, value in kw.items():
        # Another number of rows would leave some of the output as it was.
        cases += [(key, dict(kw, **{key: v})) for v in _spoiled(value, "x" if key in ("k", "v", "x", "q") else key)]
    cases.append(("stream", dict(kw, stream=torch.cuda.current_stream())))
    for key, ws in (("adapter", "workspace"), ("paged", "workspace")):
        if name.startswith(key):
            for size in (1 << 20, 0):
                cases.append((ws, dict(kw, workspace=torch.empty(size, dtype=torch.uint8, device="cuda"))))
    valid = 0
    for key, case in cases:
        monkeypatch.setattr(ops, "_binding", native)
        native.taken = None
        a = _outcome(fn, case)
        taken = native.taken
        monkeypatch.setattr(ops, "_binding", PYTHON)
        b = _outcome(fn, case)
        what = {k: (tuple(v.shape), v.dtype, str(v.device)) if torch.is_tensor(v) else v for k, v in case.items()}
        assert _same(a, b), (name, key, what, a, b)
        if isinstance(a, tuple):                # an error, the same on both paths
            assert key, (name, a)
            continue
        valid += 1
        if not key:
            assert taken, name
    assert valid > 1
