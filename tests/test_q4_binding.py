"""What the binding of the 4-bit cache takes and refuses, on the host.  Refused calls
enqueue nothing; they use placeholder addresses and therefore run only where no GPU is
visible."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2504_09345_amd import binding as pb
from test_q4_abi import P, S, dims, host_only

VARLEN = dict(num_q_rows=20, max_q_len=13)


def attend(name, d, q=P, workspace=None, stream=S):
    if name == "paged_attn_q4":
        return pb.paged_attn_q4(q, P, P, P, P, 0.1, P, d, workspace=workspace, stream=stream)
    return pb.paged_attn_varlen_q4(q, P, P, P, P, P, 0.1, P, d, workspace=workspace, stream=stream)


CALLS = [("paged_attn_q4", dims()), ("paged_attn_varlen_q4", dims(**VARLEN))]


class Never:
    """A library that no refused call reaches."""

    def __init__(self, lib):
        self.pa_workspace_size_q4 = lib.pa_workspace_size_q4


@pytest.fixture
def unreached(monkeypatch):
    lib = pb.load()
    monkeypatch.setattr(pb, "load", lambda: Never(lib))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)


@host_only
@pytest.mark.parametrize("name,d", CALLS)
def test_workspaces_on_the_host_are_refused(name, d, unreached):
    with pytest.raises(ValueError, match="current device"):
        attend(name, d, workspace=torch.zeros(pb.pa_workspace_size_q4(d), dtype=torch.uint8))


@host_only
@pytest.mark.parametrize("name,d", CALLS)
@pytest.mark.parametrize("device,wide,match", [(1, 1, "current device"), (0, 4, "contiguous")])
def test_workspaces_that_are_refused(name, d, device, wide, match, unreached, monkeypatch):
    """Of another device; an expanded view, whose elements are more than its storage."""
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: device)
    n = pb.pa_workspace_size_q4(d)
    with pytest.raises(ValueError, match=match):
        attend(name, d, workspace=torch.zeros(n // wide, dtype=torch.uint8).expand(wide, n // wide) if wide > 1
               else torch.zeros(n, dtype=torch.uint8))


@host_only
@pytest.mark.parametrize("name,d", CALLS)
def test_temporary_workspaces_are_on_the_gpu(name, d, unreached, monkeypatch):
    """Also of calls whose arrays are addresses, which have no device."""
    class Made(Exception):
        pass

    def empty(*shape, dtype, device):
        raise Made(device)

    monkeypatch.setattr(torch, "empty", empty)
    with pytest.raises(Made, match="cuda"):
        attend(name, d, stream=None)


def arrays(name, d):
    """Arrays of the call that dims describe, of meta tensors: shapes without memory."""
    rows = d.num_q_rows or d.num_seqs
    heads = d.num_kv_heads if name.startswith("pa_kv") else d.num_q_heads
    dense = [torch.empty(rows, heads, d.head_dim, dtype=torch.bfloat16, device="meta") for _ in range(2)]
    pools = [torch.empty(d.num_pages, d.num_kv_heads, 1088, dtype=torch.uint8, device="meta") for _ in range(2)]
    return dense + pools + [torch.empty(d.num_seqs, d.max_pages_per_seq, dtype=torch.int32, device="meta")]


def call(name, d, t):
    qsl = torch.empty(d.num_seqs + 1, dtype=torch.int32, device="meta") if d.num_q_rows else None
    x, y, k, v, bt = t
    cl = torch.empty(d.num_seqs, dtype=torch.int32, device="meta")
    if name == "pa_kv_append_q4":
        return pb.pa_kv_append_q4(x, y, bt, cl, k, v, d, query_start_loc=qsl, stream=S)
    if name == "pa_kv_read_q4":
        return pb.pa_kv_read_q4(k, v, bt, cl, x, y, d, query_start_loc=qsl, stream=S)
    if name == "paged_attn_q4":
        return pb.paged_attn_q4(x, k, v, bt, cl, 0.1, y, d, workspace=P, stream=S)
    return pb.paged_attn_varlen_q4(x, k, v, bt, cl, qsl, 0.1, y, d, workspace=P, stream=S)


class Reached(Exception):
    pass


@host_only
@pytest.mark.parametrize("name", ["pa_kv_append_q4", "pa_kv_read_q4", "paged_attn_q4", "paged_attn_varlen_q4"])
def test_rows_of_other_shapes_are_refused(name, monkeypatch):
    """Arrays with more heads, dims or pages a sequence than dims say hold enough
    elements, and would be read with the strides of others."""
    d = dims(**(VARLEN if name == "paged_attn_varlen_q4" else {}))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(torch.Tensor, "data_ptr", lambda t: P)

    class Lib:
        def __getattr__(self, what):
            def entry(*a):
                raise Reached
            return entry

    n = pb.pa_workspace_size_q4(d)
    monkeypatch.setattr(pb, "pa_workspace_size_q4", lambda dims: n)
    monkeypatch.setattr(pb, "load", lambda: Lib())
    good = arrays(name, d)
    with pytest.raises(Reached):
        call(name, d, good)
    flat = list(good)
    flat[0] = good[0].reshape(-1)  # (an array of another rank is taken by its elements)
    with pytest.raises(Reached):
        call(name, d, flat)
    for i, t in enumerate(good):
        wider = [(t.shape[0], 2 * t.shape[1], *t.shape[2:])]
        if i < 2:
            wider.append((t.shape[0], t.shape[1], 2 * t.shape[2]))
            wider.append((2 * t.shape[0], t.shape[1], t.shape[2] // 2))
        for shape in wider:
            bad = list(good)
            bad[i] = torch.empty(shape, dtype=t.dtype, device="meta")
            with pytest.raises(ValueError, match="rows of"):
                call(name, d, bad)


@host_only
@pytest.mark.parametrize("name", ["pa_kv_append_q4", "pa_kv_read_q4", "paged_attn_q4", "paged_attn_varlen_q4"])
def test_head_dims_are_the_librarys_to_refuse(name, monkeypatch):
    d = dims(head_dim=96, **(VARLEN if name == "paged_attn_varlen_q4" else {}))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    with pytest.raises(pb.PagedAttnError, match="not compiled|ENOTSUP|-2"):
        call(name, d, arrays(name, d))


@host_only
@pytest.mark.parametrize("name", ["pa_kv_append_q4", "paged_attn_q4"])
def test_arrays_that_are_no_tensors(name, monkeypatch):
    d = dims()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    good = arrays(name, d)
    for i in range(len(good)):
        bad = list(good)
        bad[i] = np.zeros(1, np.int8)
        with pytest.raises(TypeError):
            call(name, d, bad)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [pb.PA_BF16, pb.PA_FP32])
@pytest.mark.parametrize("seqs", [2, 33, 257, 513, 1024, 4096, 100000])
@pytest.mark.parametrize("ctx", [1000, 32768, 65536, 131072, 1 << 20])
def test_workspaces_of_chunks_beside_decode_rows(D, dtype, seqs, ctx):
    """One chunk of two rows (or 60) among decode rows: records of parts take 64 MiB at
    most, whatever the other rows are."""
    for most in (2, 60):
        n = pb.pa_workspace_size_q4(dims(num_seqs=seqs, num_q_rows=seqs - 1 + most, max_q_len=most, max_context_len=ctx,
                                         max_pages_per_seq=1 << 16, head_dim=D, dtype=dtype))
        assert 0 < n <= (64 << 20) + 512, (n, most)


@host_only
@pytest.mark.parametrize("name", ["pa_kv_append_q4", "pa_kv_read_q4"])
def test_more_rows_than_a_launch_has_threads(name):
    """A wave of 64 threads a row, or four rows of a sequence, and fewer than 2^32 in all."""
    for kw, qsl in ((dict(num_seqs=1 << 26), None), (dict(num_seqs=3, num_q_rows=1 << 28), P), (dict(num_seqs=1 << 25, num_q_rows=1 << 25), P)):
        assert getattr(pb, name)(P, P, P, P, P, P, dims(**kw), query_start_loc=qsl, stream=S, check=False) == pb.PA_ENOTSUP, kw


@host_only
@pytest.mark.parametrize("dtype", [pb.PA_BF16, pb.PA_FP32])
def test_more_chunk_rows_than_a_launch_has_threads(dtype):
    """(Contexts of 16 tokens; one head, whose 16 rows are a wave's.)"""
    for rows, fits in ((1 << 28, True), (1 << 29, False)):
        d = dims(num_seqs=rows // 16, num_q_rows=rows, max_q_len=16, num_q_heads=1, num_kv_heads=1, max_context_len=16, dtype=dtype)
        n = ctypes.c_size_t()
        assert pb.load().pa_workspace_size_q4(ctypes.byref(d), ctypes.byref(n)) == (pb.PA_OK if fits else pb.PA_ENOTSUP)


@pytest.mark.parametrize("has", [True, False])
def test_current_stream(has, monkeypatch):
    """The current stream's handle, also from a torch without the shorter way to it."""
    class Stream:
        cuda_stream = 0x50

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: Stream)
    if has:
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x40 + device, raising=False)
    else:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert pb._stream(None) == (0x43 if has else 0x50)
    assert pb._stream(0) is None and pb._stream(7) == 7 and pb._stream(Stream) == 0x50
