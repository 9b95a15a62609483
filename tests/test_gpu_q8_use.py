"""The 8-bit cache as a program uses it on the GPU: a serving step with its rotary
positions, pools past 4 GiB, other streams, captured steps that share a workspace, calls
side by side, and appends and reads of every split."""
import numpy as np
import pytest
import torch

from oracle import q8
from paper_2504_09345_amd import binding as pb
from q4_util import check
from q8_util import Batch, same_bytes
from test_gpu_rope import check as check_rope

from parity_util import announce

pytestmark = pytest.mark.gpu


def test_a_serving_step():
    """Prompts and then single tokens: a joint projection's rows are rotated at their
    positions, written, attend and are read back, on a stream of its own."""
    announce("q8 serving steps")
    H_q, H_kv, D = 8, 2, 128
    b = Batch([(70, 70), (33, 33), (5, 5)], H_q, H_kv, D, seed=8)
    d = b.upload()
    stream = torch.cuda.Stream()
    bt = np.concatenate([b.bt, np.zeros((3, 8 - b.bt.shape[1]), np.int32)], 1)
    free = [p for p in range(b.num_pages) if p not in set(b.bt[0, :5]) | set(b.bt[1, :3]) | set(b.bt[2, :1])]
    bt[0, 5], bt[1, 3], bt[2, 1] = free[:3]
    b.bt = bt
    w, factor = pb.pa_rope_frequencies(64, kind="turns", stretch=4)
    inv_freq = w.cuda()
    g = torch.Generator(device="cuda").manual_seed(3)
    for step in range(14):  # (the third sequence crosses a page, its fifth token on)
        if step > 0:
            b.ctx, b.n_rows, b.qsl, b.T = b.ctx + 1, [1] * 3, np.arange(4, dtype=np.int32), 3
        pos = np.concatenate([np.arange(c - n, c) for c, n in zip(b.ctx, b.n_rows)])
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            joint = torch.randn(b.T, H_q + 2 * H_kv, D, device="cuda", generator=g) * (1 + step)
            joint = joint.bfloat16()
            dbt, dcl, dqsl = b.cuda(bt), b.cuda(b.ctx), b.cuda(b.qsl)
            q, k, v = torch.empty(b.T, H_q, D, dtype=torch.bfloat16, device="cuda"), *torch.empty(2, b.T, H_kv, D, dtype=torch.bfloat16, device="cuda")
            v.copy_(joint[:, H_q + H_kv:])
            pb.pa_rope(joint[:, :H_q], joint[:, H_q:H_q + H_kv], dcl, inv_freq, q, k,
                       pb.make_dims_rope(q, k, 128, num_q_rows=b.T, num_seqs=3), factor=factor, query_start_loc=dqsl)
            dims = pb.make_dims_q8(k, d["k"], dbt, 128, num_q_rows=b.T, max_q_len=max(b.n_rows))
            pb.pa_kv_append_q8(k, v, dbt, dcl, d["k"], d["v"], d["scales"], dims, query_start_loc=dqsl)
            dims.num_q_heads = H_q
            out, back = torch.empty_like(q), torch.empty((2,) + k.shape, dtype=torch.bfloat16, device="cuda")
            pb.paged_attn_varlen_q8(q, d["k"], d["v"], d["scales"], dbt, dcl, dqsl, b.scale, out, dims)
            pb.pa_kv_read_q8(d["k"], d["v"], d["scales"], dbt, dcl, back[0], back[1], dims, query_start_loc=dqsl)
        stream.synchronize()
        check_rope(q, joint[:, :H_q], pos, w, np.float32(factor), False, f"step {step}")
        check_rope(k, joint[:, H_q:H_q + H_kv], pos, w, np.float32(factor), False, f"step {step}")
        kn, vn, b.q = (x.float().cpu().numpy() for x in (k, v, q))
        b.k, b.v, b.scales = ref = b.written(kn, vn)
        assert same_bytes(d, ref) == "", f"step {step}"
        check(out.float().cpu(), b.expected(), 90, "bf16", f"step {step}")
        assert np.array_equal(back.float().cpu().numpy(), q8.read(*ref, b.bt, b.ctx, D, b.qsl))


# --- how rows are split ----------------------------------------------------------

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_from_any_slot(D, dtype):
    """Appends of 0 .. 17 rows that begin at every slot of a page: the bytes of the slots
    after them stay."""
    announce(f"q8 append from any slot D={D} {dtype}")
    lens = [(p + n, n) for p in range(17) for n in (0, 1, 2, 3, 5, 15, 16, 17) if p + n]
    b = Batch(lens, 2, 2, D, dtype, seed=D)
    kn, vn = b.new_rows(5), b.new_rows(6)
    d = b.upload()
    b.append(d, kn, vn)
    ref = b.written(kn, vn)
    assert same_bytes(d, ref) == ""
    assert np.array_equal(b.read(d).astype(np.float64), q8.read(*ref, b.bt, b.ctx, D, b.qsl))


@pytest.mark.parametrize("dtype,D,H_kv", [("bf16", 128, 64), ("fp32", 64, 70)])
def test_long_reads_are_the_short_ones(dtype, D, H_kv):
    """A read whose output the caches do not hold, against reads of one sequence."""
    announce(f"q8 long read {dtype} D={D} H_kv={H_kv}")
    rng = np.random.default_rng(D)
    lens = [1, 3, 2000, 17, 0, 2016, 4097, 250]
    prior = [0, 5, 7, 30, 0, 0, 2, 6]
    pages = [-(-(n + p) // 16) for n, p in zip(lens, prior)]
    num = sum(pages) + 2
    perm = rng.permutation(num).astype(np.int32)
    bt = np.full((len(lens), 5000 // 16), -1, np.int32)
    at = 0
    for i, n in enumerate(pages):
        bt[i, :n] = perm[at:at + n]
        at += n
    bt[5, 3] = num  # a page outside the pool: 16 rows of NaN
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randint(0, 256, (num, H_kv, 16 * D), dtype=torch.uint8, device="cuda", generator=g) for _ in range(2))
    scales = torch.randint(100, 140, (num, H_kv, 2), dtype=torch.uint8, device="cuda", generator=g)
    qsl = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    cl = torch.from_numpy((np.array(lens) + prior).astype(np.int32)).cuda()
    bt = torch.from_numpy(bt).cuda()
    rows = sum(lens) + 5  # (the last five are of no sequence)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    assert 2 * rows * H_kv * D * kind.itemsize > 256 << 20

    def read(n, bt, cl, qsl):
        out = torch.full((2, n, H_kv, D), -3.0, dtype=kind, device="cuda")
        pb.pa_kv_read_q8(k, v, scales, bt, cl, out[0], out[1], pb.make_dims_q8(out[0], k, bt, 5000 // 16 * 16, num_q_rows=n), query_start_loc=qsl)
        return out

    got = read(rows, bt, cl, qsl)
    for i, n in enumerate(lens):
        if n:
            one = read(n, bt[i:i + 1].contiguous(), cl[i:i + 1].contiguous(), torch.tensor([0, n], dtype=torch.int32, device="cuda"))
            part = got[:, int(qsl[i]):int(qsl[i]) + n]
            assert torch.equal(part.nan_to_num(7.0), one.nan_to_num(7.0)) and torch.equal(part.isnan(), one.isnan()), i
    a = int(qsl[5]) + 48
    assert got[:, a:a + 16].isnan().all()
    assert (got[:, sum(lens):] == -3).all()


# --- pools past 4 GiB ----------------------------------------------------------

def test_pools_past_32_bits():
    """Pages behind the first 4 GiB of the pools: the same bits as near ones."""
    announce("q8 pools past 4 GiB")
    H_q, H_kv, D = 32, 8, 128
    page = H_kv * 16 * D
    num = (1 << 32) // page + 200
    lens = [(200, 1), (90, 33), (300, 150), (16, 16)]
    b = Batch(lens, H_q, H_kv, D, seed=8)
    d = b.upload()
    far = dict(d)
    for w in ("k", "v"):
        far[w] = torch.empty(num, H_kv, 16 * D, dtype=torch.uint8, device="cuda")
        far[w][num - b.num_pages:] = d[w]
    far["scales"] = torch.empty(num, H_kv, 2, dtype=torch.uint8, device="cuda")
    far["scales"][num - b.num_pages:] = d["scales"]
    far["bt"] = d["bt"] + (num - b.num_pages)
    g = torch.Generator(device="cuda").manual_seed(2)
    rows = torch.randn(2, b.T, H_kv, D, device="cuda", generator=g).bfloat16()
    res = []
    for x in (d, far):
        dims = b.dims(x, rows[0])
        pb.pa_kv_append_q8(rows[0], rows[1], x["bt"], x["cl"], x["k"], x["v"], x["scales"], dims, query_start_loc=x["qsl"])
        back = torch.empty_like(rows)
        pb.pa_kv_read_q8(x["k"], x["v"], x["scales"], x["bt"], x["cl"], back[0], back[1], dims, query_start_loc=x["qsl"])
        wide = dict(x, bt=torch.cat([x["bt"], x["bt"][:, :1].expand(-1, (1 << 16) - x["bt"].shape[1])], 1).contiguous())
        last = [int(b.qsl[i + 1]) - 1 for i in range(len(lens))]
        q1, cl = x["q"][last].contiguous(), x["cl"]
        one = torch.empty_like(q1)
        pb.paged_attn_q8(q1, x["k"], x["v"], x["scales"], x["bt"], cl, b.scale, one, pb.make_dims_q8(q1, x["k"], x["bt"], 300))
        res.append((back, b.attend(x), b.attend(wide, b.dims(wide, max_context_len=1 << 20)), one))
    for a, c in zip(*res):
        assert torch.equal(a, c)
    del far
    torch.cuda.empty_cache()


# --- streams and graphs ----------------------------------------------------------

def _step(b, d, out, ws, rows, back, stream=None):
    dims = b.dims(d, rows[0])
    adims = b.dims(d)
    pb.pa_kv_append_q8(rows[0], rows[1], d["bt"], d["cl"], d["k"], d["v"], d["scales"], dims, query_start_loc=d["qsl"], stream=stream)
    b.attend(d, adims, out, workspace=ws, stream=stream)
    pb.pa_kv_read_q8(d["k"], d["v"], d["scales"], d["bt"], d["cl"], back[0], back[1], dims, query_start_loc=d["qsl"], stream=stream)


def _made(lens, seed, H_q=16, H_kv=2, D=128):
    b = Batch(lens, H_q, H_kv, D, seed=seed)
    d = b.upload()
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = torch.randn(2, b.T, H_kv, D, device="cuda", generator=g).bfloat16()
    return b, d, rows, torch.empty_like(d["q"]), torch.empty_like(rows)


@pytest.mark.parametrize("own", [True, False], ids=["workspace", "temporary"])
def test_other_streams(own):
    """A step on another stream than the current one: as a torch stream, as the current
    stream of a context, with the caller's workspace and with a temporary one."""
    announce(f"q8 step on another stream own={own}")
    b, d, rows, out, back = _made([(3000, 1), (70, 20), (500, 1), (64, 64)], 3)
    size = pb.pa_workspace_size_q8(b.dims(d))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda") if own else None
    _step(b, d, out, ws, rows, back)
    torch.cuda.synchronize()
    want = out.clone(), back.clone()
    side = torch.cuda.Stream()
    for how in ("argument", "context"):
        out.fill_(0)
        back.fill_(0)
        side.wait_stream(torch.cuda.current_stream())
        if how == "argument":
            _step(b, d, out, ws, rows, back, stream=side)
        else:
            with torch.cuda.stream(side):
                _step(b, d, out, ws, rows, back)
        side.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(back, want[1]), how


def test_calls_side_by_side():
    """Two streams, each with its own workspace, and the same pools read by both."""
    announce("q8 calls on two streams")
    b, d, rows, out, _ = _made([(6000, 1), (900, 40), (2000, 1)] * 3, 4)
    size = pb.pa_workspace_size_q8(b.dims(d))
    want = b.attend(d)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in streams]
    outs = [[torch.zeros_like(out) for _ in range(6)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(6):
        for s, ws, o in zip(streams, spaces, outs):
            b.attend(d, b.dims(d), o[i], workspace=ws, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        for x in o:
            assert torch.equal(x, want)


def test_two_graphs_share_a_workspace():
    """Two captured steps and eager ones use one workspace in turn, which holds anything
    in between; every replay is the eager result."""
    announce("q8 two graphs, one workspace")
    made = [_made([(3000, 1), (70, 20), (500, 1)], 5), _made([(40, 40), (9000, 1), (9000, 1), (300, 2)], 6)]
    size = max(pb.pa_workspace_size_q8(b.dims(d)) for b, d, *_ in made)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    want, graphs = [], []
    for b, d, rows, out, back in made:
        _step(b, d, out, ws, rows, back)
        torch.cuda.synchronize()
        want.append((out.clone(), back.clone()))
    for b, d, rows, out, back in made:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _step(b, d, out, ws, rows, back)
        graphs.append(graph)
    for turn in range(5):
        ws.fill_(37 * turn + 1)
        for i in ((0, 1), (1, 0), (0, 0), (1, 1), (0, 1))[turn]:
            b, d, rows, out, back = made[i]
            out.zero_()
            back.zero_()
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[i][0]) and torch.equal(back, want[i][1]), (turn, i)
        b, d, rows, out, back = made[turn & 1]
        _step(b, d, out, ws, rows, back)
        torch.cuda.synchronize()
        assert torch.equal(out, want[turn & 1][0])


def test_results_do_not_depend_on_order():
    """Items joined by whichever workgroup is last: the same bits every time."""
    announce("q8 decode, the same bits again")
    b = Batch([(20000, 1)] * 2 + [(700, 1)] * 5, 16, 4, 128, seed=11, varlen=False)
    d = b.upload()
    first = b.attend(d)
    for _ in range(20):
        assert torch.equal(b.attend(d), first)


def test_events_of_a_call():
    announce("q8 timing events")
    b, d, rows, out, back = _made([(3000, 1), (70, 20), (500, 1)], 7)
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    for e in ev:
        e.record()  # (creates the handle)
    torch.cuda.synchronize()
    timing = pb.PaTiming(*(e.cuda_event for e in ev))
    b.attend(d, b.dims(d), out, timing=timing)
    torch.cuda.synchronize()
    assert ev[0].elapsed_time(ev[1]) > 0 and ev[1].elapsed_time(ev[2]) >= 0
