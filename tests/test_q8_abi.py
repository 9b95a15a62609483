"""The 8-bit cache's C ABI and binding on the host: what the entry points refuse,
before any HIP call, and the sizes that they plan.  Refused calls enqueue nothing;
they use placeholder addresses and therefore run only where no GPU is visible."""
import ctypes

import pytest
import torch

from paper_2504_09345_amd import binding as pb

host_only = pytest.mark.skipif(torch.cuda.is_available(), reason="placeholder addresses: host-only check")

P = 0x10000  # a 16-byte aligned placeholder
S = 0x1      # a stream that no refused call reaches


def dims(**kw):
    base = dict(num_seqs=8, num_q_heads=32, num_kv_heads=8, head_dim=128, page_size=16, num_pages=600,
                max_pages_per_seq=64, max_context_len=1024, pages_per_split=0, dtype=pb.PA_BF16, num_q_rows=0, max_q_len=0)
    base.update(kw)
    return pb.PaDims(**base)


def rows_call(name, d, ptrs=(P,) * 4, qsl=None, pools=(P, P, P)):
    """pa_kv_append_q8 or pa_kv_read_q8: the dense pair first, table and lengths last; pools
    and scales."""
    (k, v, bt, cl), (kp, vp, sc) = ptrs, pools
    if name == "pa_kv_append_q8":
        return pb.pa_kv_append_q8(k, v, bt, cl, kp, vp, sc, d, query_start_loc=qsl, stream=S, check=False)
    return pb.pa_kv_read_q8(kp, vp, sc, bt, cl, k, v, d, query_start_loc=qsl, stream=S, check=False)


def decode(d, q=P, k=P, v=P, sc=P, bt=P, cl=P, scale=0.1, out=P, ws=P, ws_bytes=1 << 40):
    return pb.load().paged_attn_q8(q, k, v, sc, bt, cl, scale, out, ctypes.byref(d), ws, ws_bytes, S, None)


def varlen(d, q=P, k=P, v=P, sc=P, bt=P, cl=P, qsl=P, scale=0.1, out=P, ws=P, ws_bytes=1 << 40):
    return pb.load().paged_attn_varlen_q8(q, k, v, sc, bt, cl, qsl, scale, out, ctypes.byref(d), ws, ws_bytes, S, None)


def test_null_result_addresses():
    lib = pb.load()
    n = ctypes.c_size_t()
    assert lib.pa_workspace_size_q8(None, ctypes.byref(n)) == pb.PA_EINVAL
    assert lib.pa_workspace_size_q8(ctypes.byref(dims()), None) == pb.PA_EINVAL


# dims that no entry point takes, and the code
BAD_CACHE = [
    (dict(head_dim=96), "PA_ENOTSUP"), (dict(head_dim=256), "PA_ENOTSUP"), (dict(page_size=32), "PA_ENOTSUP"),
    (dict(dtype=2), "PA_ENOTSUP"), (dict(dtype=-1), "PA_ENOTSUP"),
    (dict(max_context_len=(1 << 30) + 1, max_pages_per_seq=1 << 27), "PA_ENOTSUP"),
    (dict(num_seqs=-1), "PA_EINVAL"), (dict(num_kv_heads=0), "PA_EINVAL"), (dict(num_pages=-1), "PA_EINVAL"),
    (dict(max_pages_per_seq=-1), "PA_EINVAL"), (dict(max_context_len=-1), "PA_EINVAL"),
    (dict(pages_per_split=4), "PA_EINVAL"), (dict(max_context_len=1025), "PA_EINVAL"),
    (dict(num_q_rows=7), "PA_EINVAL"),  # (a decode call's rows are its sequences)
]


@host_only
@pytest.mark.parametrize("kw,code", BAD_CACHE)
@pytest.mark.parametrize("name", ["pa_kv_append_q8", "pa_kv_read_q8", "decode"])
def test_refused_dims(name, kw, code):
    call = decode if name == "decode" else lambda d: rows_call(name, d)
    assert call(dims(**kw)) == getattr(pb, code)


@host_only
@pytest.mark.parametrize("kw,code", [
    (dict(num_q_heads=40), "PA_ENOTSUP"), (dict(num_q_heads=24), "PA_ENOTSUP"), (dict(num_q_heads=128), "PA_ENOTSUP"),
    (dict(num_q_heads=33), "PA_EINVAL"), (dict(num_q_heads=0), "PA_EINVAL"), (dict(max_q_len=2), "PA_EINVAL"),
])
def test_refused_heads(kw, code):
    assert decode(dims(**kw)) == getattr(pb, code)


@host_only
@pytest.mark.parametrize("kw,code", [
    (dict(num_q_rows=-1, max_q_len=1), "PA_EINVAL"), (dict(num_q_rows=16, max_q_len=0), "PA_EINVAL"),
    (dict(num_q_rows=16, max_q_len=-1), "PA_EINVAL"), (dict(num_q_rows=16, max_q_len=2000), "PA_EINVAL"),
    (dict(num_q_rows=16, max_q_len=2, num_seqs=0), "PA_EINVAL"),
    (dict(num_q_rows=1 << 26, max_q_len=2), "PA_ENOTSUP"),  # (32-bit row and head numbers)
])
def test_refused_rows(kw, code):
    assert varlen(dims(**kw)) == getattr(pb, code)


@host_only
@pytest.mark.parametrize("name", ["pa_kv_append_q8", "pa_kv_read_q8"])
@pytest.mark.parametrize("at", range(7))
def test_refused_row_addresses(name, at):
    p = [P] * 7
    p[at] = None
    assert rows_call(name, dims(), p[:4], pools=p[4:]) == pb.PA_EINVAL
    if at not in (2, 3):
        p[at] = P + (8 if at < 6 else 1)  # (scales are pairs of bytes)
        assert rows_call(name, dims(), p[:4], pools=p[4:]) == pb.PA_EINVAL
    d = dims(num_q_rows=-2)
    assert rows_call(name, d, qsl=P) == pb.PA_EINVAL
    assert rows_call(name, dims(num_q_rows=3, num_seqs=0), qsl=P) == pb.PA_EINVAL
    assert rows_call(name, dims(num_q_rows=3, num_seqs=1 << 30), qsl=P) == pb.PA_ENOTSUP


@host_only
def test_refused_attention_addresses():
    for name in ("q", "k", "v", "sc", "bt", "cl", "out"):
        assert decode(dims(), **{name: None}) == pb.PA_EINVAL, name
        assert varlen(dims(num_q_rows=20, max_q_len=13), **{name: None}) == pb.PA_EINVAL, name
    assert varlen(dims(num_q_rows=20, max_q_len=13), qsl=None) == pb.PA_EINVAL
    for name in ("q", "k", "v", "out", "ws"):
        assert decode(dims(), **{name: P + 4}) == pb.PA_EINVAL, name
    assert decode(dims(), sc=P + 1) == pb.PA_EINVAL and varlen(dims(num_q_rows=20, max_q_len=13), sc=P + 1) == pb.PA_EINVAL
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert decode(dims(), scale=scale) == pb.PA_EINVAL


@host_only
def test_workspaces_too_small():
    for d, call in ((dims(), decode), (dims(num_q_rows=20, max_q_len=13), varlen)):
        need = pb.pa_workspace_size_q8(d)
        assert need > 0
        for ws, n in ((P, need - 1), (P, 0), (None, need)):
            assert call(d, ws=ws, ws_bytes=n) == pb.PA_ENOSPC


@host_only
def test_binding_raises():
    """The same refusals through the binding, as errors that name the code."""
    with pytest.raises(pb.PagedAttnError):
        pb.paged_attn_q8(P, P, P, P, P, P, 0.1, P, dims(head_dim=96), workspace=P, stream=S)
    with pytest.raises(pb.PagedAttnError):
        pb.paged_attn_varlen_q8(P, P, P, P, P, P, P, 0.1, P, dims(num_q_rows=16, max_q_len=0), workspace=P, stream=S)
    with pytest.raises(pb.PagedAttnError):
        pb.pa_kv_append_q8(P, P + 8, P, P, P, P, P, dims(), stream=S)
    with pytest.raises(ValueError):  # a temporary workspace for a raw stream cannot be tracked
        pb.paged_attn_q8(P, P, P, P, P, P, 0.1, P, dims(), stream=S)


@host_only
@pytest.mark.parametrize("name,group", [("pa_kv_append_q8", 16), ("pa_kv_read_q8", 4)])
@pytest.mark.parametrize("seqs", [1, 1000])
def test_most_rows_of_a_call(name, group, seqs):
    """The header's bound: 2^26 - 4 groups of rows, 16 rows of chunks that are appended and
    4 that are read, single rows one by one, and two more for each sequence of a call with
    chunks.  (Without arrays: PA_EINVAL where the size is not refused.)"""
    none, most = dict(ptrs=(None,) * 4, pools=(None,) * 3), (1 << 26) - 4
    rows = (most - 2 * seqs) * group
    for n, code in ((rows, pb.PA_ENOTSUP), (rows - 1, pb.PA_EINVAL), (1 << 30, pb.PA_ENOTSUP), (rows // 2, pb.PA_EINVAL)):
        assert rows_call(name, dims(num_seqs=seqs, num_q_rows=n), qsl=P, **none) == code, n
    assert rows_call(name, dims(num_seqs=most), **none) == pb.PA_ENOTSUP
    assert rows_call(name, dims(num_seqs=most - 1), **none) == pb.PA_EINVAL


def test_calls_without_rows_touch_nothing():
    assert pb.pa_workspace_size_q8(dims(num_seqs=0)) == 0
    if not torch.cuda.is_available():
        for name in ("pa_kv_append_q8", "pa_kv_read_q8"):
            assert rows_call(name, dims(num_seqs=0), (None,) * 4, pools=(None, None, None)) == pb.PA_OK
            assert rows_call(name, dims(num_q_rows=0, num_seqs=3), (None,) * 4, qsl=P, pools=(None, None, None)) == pb.PA_OK
        assert decode(dims(num_seqs=0), None, None, None, None, None, None, 0.1, None, None, 0) == pb.PA_OK


def test_workspace_sizes():
    """What a call needs: decode rows 512 workgroups' two records and counters, chunks
    the records of their parts, both the larger."""
    def align(x):
        return (x + 255) // 256 * 256

    def stream(s, D):
        return align(1024 * s * D * 4) + align(1024 * s * 8) + align(512 * 128)

    for H_q, H_kv, D in ((32, 8, 128), (8, 1, 64), (6, 1, 128), (64, 64, 64)):
        d = dims(num_q_heads=H_q, num_kv_heads=H_kv, head_dim=D)
        assert pb.pa_workspace_size_q8(d) == stream(H_q // H_kv, D)
    # one chunk of 8 rows a sequence and no other row: no decode kernel, parts of the long context
    d = dims(num_seqs=2, num_q_rows=16, max_q_len=8, max_context_len=32768, max_pages_per_seq=2048)
    n = pb.pa_workspace_size_q8(d)
    parts = n // (16 * 32 * (128 * 4 + 8))
    assert 2 <= parts <= 64 and n == align(16 * 32 * parts * 128 * 4) + align(16 * 32 * parts * 8)
    # enough rows that nothing is cut
    assert pb.pa_workspace_size_q8(dims(num_seqs=4, num_q_rows=4096, max_q_len=1024)) == 0


@host_only
def test_binding_refuses_tensors(monkeypatch):
    """Of other shapes, types and places than dims and the format say."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: getattr(t, "place", 0))
    d = dims(num_seqs=2, num_q_heads=4, num_kv_heads=2, num_pages=5, max_pages_per_seq=3, max_context_len=48)
    good = dict(q=torch.zeros(2, 4, 128, dtype=torch.bfloat16), k=torch.zeros(5, 2, 2048, dtype=torch.uint8), v=torch.zeros(5, 2, 2048, dtype=torch.uint8),
                sc=torch.zeros(5, 2, 2, dtype=torch.uint8), bt=torch.zeros(2, 3, dtype=torch.int32), cl=torch.zeros(2, dtype=torch.int32),
                out=torch.zeros(2, 4, 128, dtype=torch.bfloat16))

    class Took(Exception):
        pass

    class Lib:
        def __getattr__(self, name):
            raise Took

    monkeypatch.setattr(pb, "load", lambda: Lib())

    def call(**kw):
        t = {**good, **kw}
        pb.paged_attn_q8(t["q"], t["k"], t["v"], t["sc"], t["bt"], t["cl"], 0.1, t["out"], d, workspace=P, stream=S)

    with pytest.raises(Took):
        call()
    for name, t in good.items():
        far = t.clone()
        far.place = 1
        with pytest.raises(ValueError, match="current device"):
            call(**{name: far})
        with pytest.raises(TypeError):
            call(**{name: t.to(torch.float16)})
        with pytest.raises(ValueError):
            call(**{name: t[:1].clone()})
        wide = torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype)[..., ::2]
        with pytest.raises(ValueError):
            call(**{name: wide})
    for name, shape in (("k", (5, 1, 4096)), ("v", (10, 2, 1024)), ("sc", (5, 4, 1)), ("sc", (5, 1, 4)), ("bt", (3, 2)), ("q", (2, 2, 256))):
        with pytest.raises(ValueError):
            call(**{name: good[name].view(shape)})


@host_only
def test_binding_refuses_host_tensors(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    d = dims(num_seqs=2)
    q = torch.zeros(2, 32, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):
        pb.paged_attn_q8(q, P, P, P, P, P, 0.1, P, d, workspace=P, stream=S)
    with pytest.raises(ValueError, match="current device"):
        pb.paged_attn_q8(P, P, P, torch.zeros(600, 8, 2, dtype=torch.uint8), P, P, 0.1, P, d, workspace=P, stream=S)
    with pytest.raises(ValueError, match="current device"):
        pb.pa_kv_append_q8(P, P, P, torch.zeros(2, dtype=torch.int32), P, P, P, d, stream=S)
    with pytest.raises(ValueError, match="current device"):
        pb.paged_attn_q8(P, P, P, P, P, P, 0.1, P, d, workspace=torch.zeros(1 << 22, dtype=torch.uint8), stream=S)


def test_dims_from_shapes():
    k = torch.empty(5, 2, 1024, dtype=torch.uint8)
    bt = torch.empty(3, 7, dtype=torch.int32)
    d = pb.make_dims_q8(torch.empty(3, 4, 64), k, bt, 100)
    assert (d.num_seqs, d.num_q_heads, d.num_kv_heads, d.head_dim, d.num_pages, d.max_pages_per_seq, d.dtype) == \
        (3, 4, 2, 64, 5, 7, pb.PA_FP32)
    with pytest.raises(ValueError):  # tiles of another head dim
        pb.make_dims_q8(torch.empty(3, 4, 128), k, bt, 100)


@pytest.mark.parametrize("seqs,rows,most", [(10, 2, 2), (1000, 2, 2), (5, 8, 8), (4096, 40, 39), (3, 3, 2)])
def test_more_sequences_than_rows(seqs, rows, most):
    """Batches padded with sequences of no rows are planned as what they can hold."""
    n = pb.pa_workspace_size_q8(dims(num_seqs=seqs, num_q_rows=rows, max_q_len=most))
    assert 0 < n < 1 << 28
