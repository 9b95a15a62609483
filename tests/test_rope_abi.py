"""Rotary positions on the host: what pa_rope refuses before any HIP call (with
placeholder addresses, so only where no GPU is visible), and pa_rope_frequencies against
its formulas."""
import ctypes
import math

import pytest
import torch

from paper_2504_09345_amd import binding as pb

host_only = pytest.mark.skipif(torch.cuda.is_available(), reason="placeholder addresses: host-only check")

P = 0x10000  # a 16-byte aligned placeholder
S = 0x1      # a stream that no refused call reaches


def dims(**kw):
    base = dict(num_seqs=8, num_q_heads=32, num_kv_heads=8, head_dim=128, page_size=16, max_context_len=1024, dtype=pb.PA_BF16)
    base.update(kw)
    return pb.PaDims(**base)


def call(d=None, q=P, k=2 * P, positions=None, cl=P, qsl=None, q_out=3 * P, k_out=4 * P, rope=None, **fields):
    r = dict(inv_freq=P, factor=1.0, rot_dim=128, interleaved=0)
    r.update(fields)
    r = pb.PaRope(**r)
    return pb.load().pa_rope(q, k, positions, cl, qsl, q_out, k_out, ctypes.byref(r), ctypes.byref(d or dims()), S)


@host_only
@pytest.mark.parametrize("kw,code", [
    (dict(head_dim=96), "PA_ENOTSUP"), (dict(head_dim=256), "PA_ENOTSUP"), (dict(dtype=2), "PA_ENOTSUP"), (dict(dtype=-1), "PA_ENOTSUP"),
    (dict(num_seqs=-1), "PA_EINVAL"), (dict(num_q_heads=0), "PA_EINVAL"), (dict(num_kv_heads=0), "PA_EINVAL"), (dict(num_kv_heads=-8), "PA_EINVAL"),
    (dict(max_context_len=-1), "PA_EINVAL"), (dict(num_q_rows=7), "PA_EINVAL"), (dict(num_q_rows=-1), "PA_EINVAL"),
    (dict(num_q_heads=1 << 30), "PA_ENOTSUP"),
])
def test_refused_dims(kw, code):
    assert call(dims(**kw)) == getattr(pb, code)


@host_only
@pytest.mark.parametrize("fields", [
    dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=130), dict(rot_dim=-2), dict(interleaved=2), dict(interleaved=-1),
    dict(factor=float("nan")), dict(factor=float("inf")), dict(inv_freq=None), dict(inv_freq=P + 4),
    dict(q_stride=32 * 128 - 8), dict(k_stride=8 * 128 - 8), dict(q_out_stride=8), dict(k_out_stride=-1024),
    dict(q_stride=32 * 128 + 4), dict(k_out_stride=8 * 128 + 1),
])
def test_refused_fields(fields):
    assert call(**fields) == pb.PA_EINVAL


@host_only
def test_refused_addresses():
    for name in ("q", "k", "q_out", "k_out", "cl"):
        assert call(**{name: None}) == pb.PA_EINVAL, name
        if name != "cl":
            assert call(**{name: P + 8}) == pb.PA_EINVAL, name
    assert call(q=None, k=None, q_out=None, k_out=None) == pb.PA_EINVAL
    assert call(q_out=P, q_stride=8192) == pb.PA_EINVAL                    # in place, at another stride
    assert call(k_out=2 * P, k_stride=1024, k_out_stride=2048) == pb.PA_EINVAL
    assert call(dims(num_q_rows=4, num_seqs=0), qsl=P) == pb.PA_EINVAL
    lib = pb.load()
    r, d = pb.PaRope(P, 1.0, 128), dims()
    assert lib.pa_rope(P, P, None, P, None, P, P, None, ctypes.byref(d), S) == pb.PA_EINVAL
    assert lib.pa_rope(P, P, None, P, None, P, P, ctypes.byref(r), None, S) == pb.PA_EINVAL


@host_only
def test_calls_without_rows_touch_nothing():
    none = dict(q=None, k=None, cl=None, q_out=None, k_out=None)
    assert call(dims(num_seqs=0), **none) == pb.PA_OK
    assert call(dims(num_q_rows=0), qsl=P, **none) == pb.PA_OK


@host_only
def test_binding(monkeypatch):
    with pytest.raises(pb.PagedAttnError):
        pb.pa_rope(P, P, P, P, P, P, dims(head_dim=96), rot_dim=64, stream=S)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    d, w = dims(num_seqs=2, num_q_heads=2, num_kv_heads=1), torch.ones(64, dtype=torch.float64)
    q = torch.zeros(2, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):
        pb.pa_rope(q, None, P, P, P, None, d, rot_dim=64, stream=S)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    for bad in (q[:1], q[:, :1], q[..., :64], torch.zeros(2, 2, 256, dtype=torch.bfloat16)[..., ::2], torch.zeros(2, 3, 256, dtype=torch.bfloat16)[:, :2, :128],
                torch.zeros(2, 2, 128, 1, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            pb.pa_rope(bad, None, P, w, P, None, d, stream=S)
    with pytest.raises(TypeError):
        pb.pa_rope(q.float(), None, P, w, P, None, d, stream=S)
    with pytest.raises(TypeError):
        pb.pa_rope(q, None, P, w.float(), P, None, d, stream=S)
    with pytest.raises(ValueError):  # fewer frequencies than rot_dim asks for
        pb.pa_rope(q, None, P, w, P, None, d, rot_dim=130, stream=S)


@host_only
def test_binding_refuses_rows_that_share_memory(monkeypatch):
    """Rows 0 elements apart (a broadcast tensor), which the library would take as packed
    ones, or fewer than a row's: 50 rows of 256 elements and fewer stored ones.  A lone row
    lies on no other, whatever its tensor's stride."""
    taken = []

    class Lib:
        def pa_rope(self, q, k, positions, cl, qsl, q_out, k_out, rope, d, stream):
            taken.append((rope._obj.q_stride, rope._obj.k_stride, rope._obj.q_out_stride, rope._obj.k_out_stride))
            return pb.PA_OK

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(pb, "load", lambda: Lib())
    w = torch.ones(64, dtype=torch.float64)

    def call(x, out, key, rows=50):
        d = dims(num_seqs=rows, num_q_heads=2, num_kv_heads=2)
        q, k, q_out, k_out = (None, x, None, out) if key else (x, None, out, None)
        for positions, cl in ((torch.zeros(rows, dtype=torch.int32), None), (None, torch.zeros(rows, dtype=torch.int32))):
            pb.pa_rope(q, k, cl, w, q_out, k_out, d, positions=positions, stream=S)

    rows = torch.zeros(50, 2, 128, dtype=torch.bfloat16)
    joint = torch.zeros(50, 3, 128, dtype=torch.bfloat16)[:, :2]
    flat = torch.zeros(50 * 256, dtype=torch.bfloat16)
    for key in (False, True):
        call(rows, joint, key)
        assert taken[-2:] == [(0, 0, 0, 384) if key else (0, 0, 384, 0)] * 2
        for bad in (rows[:1].expand(50, 2, 128), flat.as_strided((50, 2, 128), (128, 128, 1)), flat.as_strided((50, 2, 128), (248, 128, 1))):
            with pytest.raises(ValueError, match="rows"):
                call(bad, rows, key)
            with pytest.raises(ValueError, match="rows"):
                call(rows, bad, key)
        call(rows[:1].expand(50, 2, 128), rows, key, rows=1)  # (the first of them alone)
        assert taken[-1] == (0, 0, 0, 0)


@host_only
def test_rows_with_positions(monkeypatch):
    """With positions and no number of rows the rows are num_seqs, though
    query_start_loc is given too: arrays of fewer are refused."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    d, w, i32 = dims(num_seqs=2, num_q_heads=2, num_kv_heads=1, num_q_rows=0), torch.ones(32, dtype=torch.float64), torch.int32
    q, two, qsl = torch.zeros(2, 2, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=i32), torch.zeros(3, dtype=i32)
    for x, positions in ((q[:1], two), (q, two[:1]), (q[:0], two[:0])):
        for loc in (None, qsl):
            with pytest.raises(ValueError):
                pb.pa_rope(x, None, None, w, x, None, d, positions=positions, query_start_loc=loc, stream=S)


def test_dims_from_shapes():
    d = pb.make_dims_rope(torch.empty(3, 4, 64), torch.empty(3, 2, 64), 100)
    assert (d.num_seqs, d.num_q_heads, d.num_kv_heads, d.head_dim, d.max_context_len, d.dtype, d.num_q_rows) == (3, 4, 2, 64, 100, pb.PA_FP32, 0)
    d = pb.make_dims_rope(None, torch.empty(9, 2, 128, dtype=torch.bfloat16), 100, num_q_rows=9, num_seqs=2)
    assert (d.num_seqs, d.num_q_heads, d.num_kv_heads, d.num_q_rows, d.dtype) == (2, 0, 2, 9, pb.PA_BF16)


# --- frequencies -----------------------------------------------------------------

@pytest.mark.parametrize("rot_dim", [2, 6, 64, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_plain_and_linear(rot_dim, base):
    w, f = pb.pa_rope_frequencies(rot_dim, base)
    ref = [base ** (-2 * i / rot_dim) for i in range(rot_dim // 2)]
    assert f == 1.0 and w.dtype == torch.float64 and w.tolist() == pytest.approx(ref, rel=1e-15)
    w, f = pb.pa_rope_frequencies(rot_dim, base, "linear", 8)
    assert f == 1.0 and w.tolist() == pytest.approx([x / 8 for x in ref], rel=1e-15)


def test_larger_base():
    w, f = pb.pa_rope_frequencies(128, 10000, "base", 16)
    plain = pb.pa_rope_frequencies(128)[0]
    assert f == 1.0 and w[0] == 1.0 and float(w[-1] / plain[-1]) == pytest.approx(1 / 16, rel=1e-12)
    assert (w[1:] < plain[1:]).all()
    assert pb.pa_rope_frequencies(2, 10000, "base", 16)[0].tolist() == [1.0]


def test_ramp_over_turns():
    w, f = pb.pa_rope_frequencies(128, 10000, "turns", 32, 4096, 1, 32)
    for got, x in zip(w.tolist(), pb.pa_rope_frequencies(128)[0].tolist()):
        turns = 4096 * x / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1) / 31))
        assert got == pytest.approx(x * (keep + (1 - keep) / 32), rel=1e-14)
    assert f == 1.0 and w[0] == 1.0


def test_ramp_over_pairs():
    w, f = pb.pa_rope_frequencies(128, 10000, "pairs", 32, 4096, 1, 32)
    plain = pb.pa_rope_frequencies(128)[0].tolist()
    assert f == pytest.approx(0.1 * math.log(32) + 1, rel=1e-7)
    # by hand: pair i turns 4096 10000^(-i/64) / 2 pi times: 32 at i = 20.95, 1 at i = 45.03
    for i, (got, x) in enumerate(zip(w.tolist(), plain)):
        slow = min(1.0, max(0.0, (i - 20) / (46 - 20)))
        assert got == pytest.approx(x * (1 - slow) + x / 32 * slow, rel=1e-14), i


@pytest.mark.parametrize("kw", [
    dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=-2), dict(rot_dim=65538), dict(base=1.0), dict(base=float("inf")), dict(base=float("nan")),
    dict(kind="linear", stretch=0.5), dict(kind="linear", stretch=float("nan")), dict(kind="turns", trained_context=0),
    dict(kind="turns", low_turns=0), dict(kind="pairs", low_turns=32), dict(kind="pairs", high_turns=float("inf")),
])
def test_refused_frequencies(kw):
    with pytest.raises(pb.PagedAttnError):
        pb.pa_rope_frequencies(**{"rot_dim": 64, **kw})


def test_refused_results():
    with pytest.raises(ValueError):
        pb.pa_rope_frequencies(64, kind="other")
    lib, c, f = pb.load(), pb.PaRopeScaling(0, 4, 10000.0), ctypes.c_float()
    out = (ctypes.c_double * 2)()
    assert lib.pa_rope_frequencies(None, out, ctypes.byref(f)) == pb.PA_EINVAL
    assert lib.pa_rope_frequencies(ctypes.byref(c), None, ctypes.byref(f)) == pb.PA_EINVAL
    assert lib.pa_rope_frequencies(ctypes.byref(c), out, None) == pb.PA_EINVAL
    for kind in (-1, 5):
        c.kind = kind
        assert lib.pa_rope_frequencies(ctypes.byref(c), out, ctypes.byref(f)) == pb.PA_EINVAL
