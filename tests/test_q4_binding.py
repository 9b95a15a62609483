"""What the binding of the 4-bit cache takes and refuses, on the host.  Refused calls
enqueue nothing; they use placeholder addresses and therefore run only where no GPU is
visible."""
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
