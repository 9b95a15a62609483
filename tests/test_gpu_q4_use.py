"""The 4-bit cache as a program uses it on the GPU: pools past 4 GiB, other streams,
captured steps that share a workspace, calls side by side, and the sizes at which the
kernels split their work differently."""
import numpy as np
import pytest
import torch

from oracle import q4
from paper_2504_09345_amd import binding as pb
from q4_util import Batch, check

from parity_util import announce

pytestmark = pytest.mark.gpu


# --- how chunks and reads are split ------------------------------------------

@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,H_q,H_kv,lens", [
    ("fp32", 32, 8, [(600, 600)]),                      # two waves share an item
    ("fp32", 32, 8, [(1500, 1500)]),                    # each its own
    ("fp32", 8, 8, [(31, 31), (32, 32), (33, 33)]),     # one unit and two, four waves for them
    ("bf16", 16, 2, [(100, 1), (64, 3), (7000, 40)]),   # parts in the workspace too
    ("bf16", 6, 1, [(97, 5), (65, 64)]),                # columns left over
], ids=["two", "one", "short", "parts", "six"])
def test_waves_that_share_an_item(D, dtype, H_q, H_kv, lens):
    announce(f"q4 chunks {dtype} D={D} heads={H_q}/{H_kv} {lens}")
    b = Batch(lens, H_q, H_kv, D, dtype=dtype, seed=len(lens))
    check(b.attend(b.upload()).float().cpu(), b.expected_gpu(), max(c for c, _ in lens), dtype)


def test_parts_without_a_key_and_nan_blocks():
    """The last rows' units are the last wave's alone, and a NaN block in one wave's part
    reaches exactly the rows and dims that see it."""
    announce("q4 chunks, a NaN block in a shared item")
    b = Batch([(130, 9)], 8, 2, 128, seed=6)
    b.v[b.bt[0, 7], 1, q4.scale_byte_of(128, 11, 2)] = 255  # token 123: rows from 2 on
    b.v[b.bt[0, 1], 0, q4.scale_byte_of(128, 0, 3)] = 255   # token 16: every row
    ref = b.expected()
    assert np.isnan(ref[0]).any() and not np.isnan(ref[0]).all()
    check(b.attend(b.upload()).float().cpu(), ref, 130, "bf16")


@pytest.mark.parametrize("dtype,D,H_kv", [("bf16", 128, 64), ("fp32", 64, 70)])
def test_long_reads_are_the_short_ones(dtype, D, H_kv):
    """A read whose output the caches do not hold, against reads of one sequence."""
    announce(f"q4 long read {dtype} D={D} H_kv={H_kv}")
    rng = np.random.default_rng(D)
    lens = [1, 3, 2000, 17, 0, 2016, 4097, 250]
    prior = [0, 5, 7, 30, 0, 0, 2, 6]
    pages = [-(-(n + p) // 16) for n, p in zip(lens, prior)]
    num = sum(pages) + 2
    perm = rng.permutation(num).astype(np.int32)
    bt = np.full((len(lens), max(pages)), -1, np.int32)
    at = 0
    for i, n in enumerate(pages):
        bt[i, :n] = perm[at:at + n]
        at += n
    bt[5, 3] = num  # a page outside the pool: 16 rows of NaN
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randint(0, 256, (num, H_kv, q4.tile_bytes(D)), dtype=torch.uint8, device="cuda", generator=g) for _ in range(2))
    qsl = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    cl = torch.from_numpy((np.array(lens) + prior).astype(np.int32)).cuda()
    bt = torch.from_numpy(bt).cuda()
    rows = sum(lens) + 5  # (the last five are of no sequence)
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    assert 2 * rows * H_kv * D * kind.itemsize > 256 << 20

    def read(n, bt, cl, qsl):
        out = torch.full((2, n, H_kv, D), -3.0, dtype=kind, device="cuda")
        pb.pa_kv_read_q4(k, v, bt, cl, out[0], out[1], pb.make_dims_q4(out[0], k, bt, 5000 // 16 * 16, num_q_rows=n), query_start_loc=qsl)
        return out

    bt = torch.cat([bt, torch.full((len(lens), 5000 // 16 - bt.shape[1]), -1, dtype=torch.int32, device="cuda")], 1)
    got = read(rows, bt, cl, qsl)
    for i, n in enumerate(lens):
        if n:
            one = read(n, bt[i:i + 1].contiguous(), cl[i:i + 1].contiguous(), torch.tensor([0, n], dtype=torch.int32, device="cuda"))
            part = got[:, int(qsl[i]):int(qsl[i]) + n]
            assert torch.equal(part.nan_to_num(7.0), one.nan_to_num(7.0)) and torch.equal(part.isnan(), one.isnan()), i
    a = int(qsl[5]) + 48
    assert got[:, a:a + 16].isnan().all()
    assert (got[:, sum(lens):] == -3).all()


@pytest.mark.parametrize("D", [64, 128])
def test_rows_from_any_slot(D):
    """Appends of 0 .. 9 rows that begin at every slot of a group of four: the bytes of
    the slots beside them stay."""
    announce(f"q4 append from any slot D={D}")
    lens = [(p + n, n) for p in range(8) for n in range(10) if p + n]
    b = Batch(lens, 2, 2, D, seed=D)
    rng = np.random.default_rng(5)
    kn, vn = (b.round(rng.standard_normal((b.T, 2, D))) for _ in range(2))
    ek, ev = q4.append(kn, vn, b.bt, b.ctx, b.k, b.v, b.qsl)
    d = b.upload()
    rows = b.cuda(kn).to(torch.bfloat16)
    pb.pa_kv_append_q4(rows, b.cuda(vn).to(torch.bfloat16), d["bt"], d["cl"], d["k"], d["v"], b.dims(d, rows), query_start_loc=d["qsl"])
    assert np.array_equal(d["k"].cpu().numpy(), ek) and np.array_equal(d["v"].cpu().numpy(), ev)


@pytest.mark.parametrize("H_kv,n,ctx", [(8, 3, 2048), (1, 1, 512), (3, 5, 7), (64, 2, 33), (8, 40, 64), (5, 300, 100)])
def test_decode_items_and_workgroups(H_kv, n, ctx):
    """Items within a wave, a workgroup, and over several of them."""
    announce(f"q4 decode ranges {n} x {ctx} H_kv={H_kv}")
    rng = np.random.default_rng(n)
    b = Batch([(int(c), 1) for c in rng.integers(max(1, ctx // 2), ctx + 1, n)], 2 * H_kv, H_kv, 64, seed=n, varlen=False)
    check(b.attend(b.upload()).float().cpu(), b.expected_gpu(), ctx, "bf16")


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "fp32")])
@pytest.mark.parametrize("lens", [[(0, 0)] * 40 + [(70, 2)] + [(9, 0)] * 30, [(300, 39)] + [(0, 0)] * 200 + [(33, 1)]],
                         ids=["two rows", "a chunk and a row"])
def test_more_sequences_than_rows(D, dtype, lens):
    announce(f"q4 chunks among empty sequences D={D} {dtype}")
    b = Batch(lens, 8, 2, D, dtype=dtype, seed=2)
    check(b.attend(b.upload()).float().cpu(), b.expected_gpu(), 300, dtype)


@pytest.mark.parametrize("ctx", [4000, 20000, 70000, 300000, 1100000])
@pytest.mark.parametrize("H_q", [1, 8])
def test_items_over_many_workgroups(H_q, ctx):
    """One item over 16 to 512 workgroups, each size of the joins' groups.  Queries of
    zeros weigh every key alike, and all sums are exact: the output is the mean of V,
    1 / l and one product from exact (2^-22 of it)."""
    announce(f"q4 one item of {ctx} tokens H_q={H_q}")
    D, pool = 64, 97
    rng = np.random.default_rng(ctx)
    k, v = (rng.integers(0, 256, (pool, 1, q4.tile_bytes(D)), dtype=np.uint8) for _ in range(2))
    k[..., 8 * D:] = rng.integers(120, 130, k[..., 8 * D:].shape)
    v[..., 8 * D:] = 127
    pages = -(-ctx // 16)
    bt = rng.integers(0, pool, (1, pages)).astype(np.int32)
    count = np.bincount(bt[0, :ctx // 16], minlength=pool)
    x = q4.unpack("v", v[:, 0], D)  # [page][token][dim]
    total = np.einsum("p,ptd->d", count.astype(np.float64), x)
    if ctx % 16:
        total += x[bt[0, -1], :ctx % 16].sum(0)
    t = [torch.from_numpy(a).cuda() for a in (k, v, bt, np.array([ctx], np.int32))]
    q = torch.zeros(1, H_q, D, device="cuda")
    for dtype, step in ((torch.float32, 2.0 ** -24), (torch.bfloat16, 2.0 ** -8)):
        out = torch.empty(1, H_q, D, dtype=dtype, device="cuda")
        pb.paged_attn_q4(q.to(dtype), t[0], t[1], t[2], t[3], 1.0, out, pb.make_dims_q4(out, t[0], t[2], ctx))
        off = np.abs(out[0].double().cpu().numpy() - total / ctx)
        assert (off <= (step + 2.0 ** -22) * np.abs(total / ctx)).all()


@pytest.mark.parametrize("varlen", [False, True])
def test_shortest(varlen):
    """Contexts of one token (its value) and of none."""
    announce(f"q4 shortest contexts varlen={varlen}")
    b = Batch([(1, 1), (0, 0) if varlen else (0, 1), (1, 1), (2, 2) if varlen else (2, 1)], 4, 1, 128, seed=3, varlen=varlen)
    got = b.attend(b.upload()).float().cpu()
    ref = b.expected()
    check(got, ref, 2, "bf16")
    assert np.array_equal(got[0].numpy(), ref[0][0].astype(np.float32))  # (one weight of 1: V itself)


# --- pools past 4 GiB ----------------------------------------------------------

def test_pools_past_32_bits():
    """Pages behind the first 4 GiB of the pools: the same bits as near ones."""
    announce("q4 pools past 4 GiB")
    H_q, H_kv, D = 32, 8, 128
    page = H_kv * q4.tile_bytes(D)
    num = (1 << 32) // page + 200
    lens = [(200, 1), (90, 33), (300, 150), (16, 16)]
    b = Batch(lens, H_q, H_kv, D, seed=8)
    d = b.upload()
    far = dict(d)
    for w in ("k", "v"):
        far[w] = torch.empty(num, H_kv, q4.tile_bytes(D), dtype=torch.uint8, device="cuda")
        far[w][num - b.num_pages:] = d[w]
    far["bt"] = d["bt"] + (num - b.num_pages)
    g = torch.Generator(device="cuda").manual_seed(2)
    rows = torch.randn(2, b.T, H_kv, D, device="cuda", generator=g).bfloat16()
    res = []
    for x in (d, far):
        dims = b.dims(x, rows[0])
        pb.pa_kv_append_q4(rows[0], rows[1], x["bt"], x["cl"], x["k"], x["v"], dims, query_start_loc=x["qsl"])
        back = torch.empty_like(rows)
        pb.pa_kv_read_q4(x["k"], x["v"], x["bt"], x["cl"], back[0], back[1], dims, query_start_loc=x["qsl"])
        wide = dict(x, bt=torch.cat([x["bt"], x["bt"][:, :1].expand(-1, (1 << 16) - x["bt"].shape[1])], 1).contiguous())
        last = [int(b.qsl[i + 1]) - 1 for i in range(len(lens))]
        q1, cl = x["q"][last].contiguous(), x["cl"]
        one = torch.empty_like(q1)
        pb.paged_attn_q4(q1, x["k"], x["v"], x["bt"], cl, b.scale, one, pb.make_dims_q4(q1, x["k"], x["bt"], 300))
        res.append((back, b.attend(x), b.attend(wide, b.dims(wide, max_context_len=1 << 20)), one))
    for a, c in zip(*res):
        assert torch.equal(a, c)
    del far
    torch.cuda.empty_cache()


# --- streams and graphs ----------------------------------------------------------

def _step(b, d, out, ws, rows, back, stream=None):
    dims = b.dims(d, rows[0])
    adims = b.dims(d)
    pb.pa_kv_append_q4(rows[0], rows[1], d["bt"], d["cl"], d["k"], d["v"], dims, query_start_loc=d["qsl"], stream=stream)
    b.attend(d, adims, out, workspace=ws, stream=stream)
    pb.pa_kv_read_q4(d["k"], d["v"], d["bt"], d["cl"], back[0], back[1], dims, query_start_loc=d["qsl"], stream=stream)


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
    announce(f"q4 step on another stream own={own}")
    b, d, rows, out, back = _made([(3000, 1), (70, 20), (500, 1), (64, 64)], 3)
    size = pb.pa_workspace_size_q4(b.dims(d))
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
    announce("q4 calls on two streams")
    b, d, rows, out, _ = _made([(6000, 1), (900, 40), (2000, 1)] * 3, 4)
    size = pb.pa_workspace_size_q4(b.dims(d))
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
    announce("q4 two graphs, one workspace")
    made = [_made([(3000, 1), (70, 20), (500, 1)], 5), _made([(40, 40), (9000, 1), (9000, 1), (300, 2)], 6)]
    size = max(pb.pa_workspace_size_q4(b.dims(d)) for b, d, *_ in made)
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
    announce("q4 decode, the same bits again")
    b = Batch([(20000, 1)] * 2 + [(700, 1)] * 5, 16, 4, 128, seed=11, varlen=False)
    d = b.upload()
    first = b.attend(d)
    for _ in range(20):
        assert torch.equal(b.attend(d), first)


def test_events_of_a_call():
    announce("q4 timing events")
    b, d, rows, out, back = _made([(3000, 1), (70, 20), (500, 1)], 7)
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    for e in ev:
        e.record()  # (creates the handle)
    torch.cuda.synchronize()
    timing = pb.PaTiming(*(e.cuda_event for e in ev))
    b.attend(d, b.dims(d), out, timing=timing)
    torch.cuda.synchronize()
    assert ev[0].elapsed_time(ev[1]) > 0 and ev[1].elapsed_time(ev[2]) >= 0
