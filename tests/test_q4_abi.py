"""The 4-bit cache's C ABI and binding on the host: what the entry points refuse,
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


def rows_call(name, d, ptrs=(P,) * 4, qsl=None, pools=(P, P)):
    """pa_kv_append_q4 or pa_kv_read_q4: the dense pair first, table and lengths last."""
    dense, (bt, cl) = ptrs[:2], ptrs[2:]
    a, b = (dense, pools) if name == "pa_kv_append_q4" else (pools, dense)
    return getattr(pb, name)(*a, bt, cl, *b, d, query_start_loc=qsl, stream=S, check=False)


def decode(d, q=P, k=P, v=P, bt=P, cl=P, scale=0.1, out=P, ws=P, ws_bytes=1 << 40):
    return pb.load().paged_attn_q4(q, k, v, bt, cl, scale, out, ctypes.byref(d), ws, ws_bytes, S, None)


def varlen(d, q=P, k=P, v=P, bt=P, cl=P, qsl=P, scale=0.1, out=P, ws=P, ws_bytes=1 << 40):
    return pb.load().paged_attn_varlen_q4(q, k, v, bt, cl, qsl, scale, out, ctypes.byref(d), ws, ws_bytes, S, None)


@pytest.mark.parametrize("D", [64, 128])
def test_tile_bytes(D):
    assert pb.pa_q4_tile_bytes(D) == 8 * D + D // 2 == pb._Q4_TILE[D]


@pytest.mark.parametrize("D", [0, 32, 96, 256, -64])
def test_no_other_tile(D):
    with pytest.raises(pb.PagedAttnError):
        pb.pa_q4_tile_bytes(D)


def test_null_result_addresses():
    lib = pb.load()
    assert lib.pa_q4_tile_bytes(64, None) == pb.PA_EINVAL
    n = ctypes.c_size_t()
    assert lib.pa_workspace_size_q4(None, ctypes.byref(n)) == pb.PA_EINVAL
    assert lib.pa_workspace_size_q4(ctypes.byref(dims()), None) == pb.PA_EINVAL


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
@pytest.mark.parametrize("name", ["pa_kv_append_q4", "pa_kv_read_q4", "decode"])
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
@pytest.mark.parametrize("name", ["pa_kv_append_q4", "pa_kv_read_q4"])
@pytest.mark.parametrize("at", range(6))
def test_refused_row_addresses(name, at):
    p = [P] * 6
    p[at] = None
    assert rows_call(name, dims(), p[:4], pools=p[4:]) == pb.PA_EINVAL
    if at not in (2, 3):
        p[at] = P + 8
        assert rows_call(name, dims(), p[:4], pools=p[4:]) == pb.PA_EINVAL
    d = dims(num_q_rows=-2)
    assert rows_call(name, d, qsl=P) == pb.PA_EINVAL
    assert rows_call(name, dims(num_q_rows=3, num_seqs=0), qsl=P) == pb.PA_EINVAL
    assert rows_call(name, dims(num_q_rows=3, num_seqs=1 << 30), qsl=P) == pb.PA_ENOTSUP


@host_only
def test_refused_attention_addresses():
    for name in ("q", "k", "v", "bt", "cl", "out"):
        assert decode(dims(), **{name: None}) == pb.PA_EINVAL, name
        assert varlen(dims(num_q_rows=20, max_q_len=13), **{name: None}) == pb.PA_EINVAL, name
    assert varlen(dims(num_q_rows=20, max_q_len=13), qsl=None) == pb.PA_EINVAL
    for name in ("q", "k", "v", "out", "ws"):
        assert decode(dims(), **{name: P + 4}) == pb.PA_EINVAL, name
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert decode(dims(), scale=scale) == pb.PA_EINVAL


@host_only
def test_workspaces_too_small():
    for d, call in ((dims(), decode), (dims(num_q_rows=20, max_q_len=13), varlen)):
        need = pb.pa_workspace_size_q4(d)
        assert need > 0
        for ws, n in ((P, need - 1), (P, 0), (None, need)):
            assert call(d, ws=ws, ws_bytes=n) == pb.PA_ENOSPC


@host_only
def test_binding_raises():
    """The same refusals through the binding, as errors that name the code."""
    with pytest.raises(pb.PagedAttnError):
        pb.paged_attn_q4(P, P, P, P, P, 0.1, P, dims(head_dim=96), workspace=P, stream=S)
    with pytest.raises(pb.PagedAttnError):
        pb.paged_attn_varlen_q4(P, P, P, P, P, P, 0.1, P, dims(num_q_rows=16, max_q_len=0), workspace=P, stream=S)
    with pytest.raises(pb.PagedAttnError):
        pb.pa_kv_append_q4(P, P + 8, P, P, P, P, dims(), stream=S)
    with pytest.raises(ValueError):  # a temporary workspace for a raw stream cannot be tracked
        pb.paged_attn_q4(P, P, P, P, P, 0.1, P, dims(), stream=S)


def test_calls_without_rows_touch_nothing():
    assert pb.pa_workspace_size_q4(dims(num_seqs=0)) == 0
    if not torch.cuda.is_available():
        for name in ("pa_kv_append_q4", "pa_kv_read_q4"):
            assert rows_call(name, dims(num_seqs=0), (None,) * 4, pools=(None, None)) == pb.PA_OK
            assert rows_call(name, dims(num_q_rows=0, num_seqs=3), (None,) * 4, qsl=P, pools=(None, None)) == pb.PA_OK
        assert decode(dims(num_seqs=0), None, None, None, None, None, 0.1, None, None, 0) == pb.PA_OK


def test_workspace_sizes():
    """What a call needs: decode rows 512 workgroups' two records and counters, chunks
    the records of their parts, both the larger."""
    def align(x):
        return (x + 255) // 256 * 256

    def stream(s, D):
        return align(1024 * s * D * 4) + align(1024 * s * 8) + align(512 * 128)

    for H_q, H_kv, D in ((32, 8, 128), (8, 1, 64), (6, 1, 128), (64, 64, 64)):
        d = dims(num_q_heads=H_q, num_kv_heads=H_kv, head_dim=D)
        assert pb.pa_workspace_size_q4(d) == stream(H_q // H_kv, D)
    # one chunk of 8 rows a sequence and no other row: no decode kernel, parts of the long context
    d = dims(num_seqs=2, num_q_rows=16, max_q_len=8, max_context_len=32768, max_pages_per_seq=2048)
    n = pb.pa_workspace_size_q4(d)
    parts = n // (16 * 32 * (128 * 4 + 8))
    assert 2 <= parts <= 64 and n == align(16 * 32 * parts * 128 * 4) + align(16 * 32 * parts * 8)
    # enough rows that nothing is cut
    assert pb.pa_workspace_size_q4(dims(num_seqs=4, num_q_rows=4096, max_q_len=1024)) == 0


class Wrong:
    """A tensor's face on the host, of a given type, size and place."""

    def __init__(self, dtype, n, device=0, contiguous=True):
        self.dtype, self.device, self._n, self._c, self._d = dtype, f"cuda:{device}", n, contiguous, device

    def get_device(self):
        return self._d

    def numel(self):
        return self._n

    def is_contiguous(self):
        return self._c

    def data_ptr(self):
        return P


@host_only
def test_binding_refuses_tensors(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    d = dims()
    n = 8 * 32 * 128
    tiles = 600 * 8 * 1088

    def call(**kw):
        t = dict(q=Wrong(torch.bfloat16, n), out=Wrong(torch.bfloat16, n), k=Wrong(torch.uint8, tiles),
                 v=Wrong(torch.uint8, tiles), bt=Wrong(torch.int32, 8 * 64), cl=Wrong(torch.int32, 8))
        t.update(kw)
        return pb._take_q4(d, 32, False, t["q"], t["out"], t["k"], t["v"], t["bt"], t["cl"], None)

    assert call() == (P,) * 6 + (None,)
    for name, good, size in (("q", torch.bfloat16, n), ("out", torch.bfloat16, n), ("k", torch.uint8, tiles),
                             ("v", torch.uint8, tiles), ("bt", torch.int32, 512), ("cl", torch.int32, 8)):
        with pytest.raises(TypeError):
            call(**{name: Wrong(torch.float16, size)})
        with pytest.raises(ValueError, match="current device"):
            call(**{name: Wrong(good, size, device=1)})
        with pytest.raises(ValueError, match="needed"):
            call(**{name: Wrong(good, size - 1)})
        with pytest.raises(ValueError, match="contiguous"):
            call(**{name: Wrong(good, size, contiguous=False)})
    with pytest.raises(ValueError, match="needed"):
        pb._take_q4(dims(num_q_rows=9, max_q_len=2), 32, True, *(Wrong(torch.bfloat16, 9 * 32 * 128),) * 2,
                    *(Wrong(torch.uint8, tiles),) * 2, Wrong(torch.int32, 512), Wrong(torch.int32, 8), Wrong(torch.int32, 8))


@host_only
def test_binding_refuses_host_tensors(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    d = dims(num_seqs=2)
    q = torch.zeros(2, 32, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):
        pb.paged_attn_q4(q, P, P, P, P, 0.1, P, d, workspace=P, stream=S)
    with pytest.raises(ValueError, match="current device"):
        pb.pa_kv_append_q4(P, P, P, torch.zeros(2, dtype=torch.int32), P, P, d, stream=S)


def test_dims_from_shapes():
    k = torch.empty(5, 2, 544, dtype=torch.uint8)
    bt = torch.empty(3, 7, dtype=torch.int32)
    d = pb.make_dims_q4(torch.empty(3, 4, 64), k, bt, 100)
    assert (d.num_seqs, d.num_q_heads, d.num_kv_heads, d.head_dim, d.num_pages, d.max_pages_per_seq, d.dtype) == \
        (3, 4, 2, 64, 5, 7, pb.PA_FP32)
    with pytest.raises(ValueError):  # tiles of another head dim
        pb.make_dims_q4(torch.empty(3, 4, 128), k, bt, 100)
    with pytest.raises(pb.PagedAttnError):
        pb.make_dims_q4(torch.empty(3, 4, 80), k, bt, 100)


@pytest.mark.parametrize("seqs,rows,most", [(10, 2, 2), (1000, 2, 2), (5, 8, 8), (4096, 40, 39), (3, 3, 2)])
def test_more_sequences_than_rows(seqs, rows, most):
    """Batches padded with sequences of no rows are planned as what they can hold."""
    n = pb.pa_workspace_size_q4(dims(num_seqs=seqs, num_q_rows=rows, max_q_len=most))
    assert 0 < n < 1 << 28
