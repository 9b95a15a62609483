"""The 4-bit paged KV cache on the GPU against its plain form in float64: the
append's bytes and the read's values exactly, attention within its arithmetic's
bound, and a serving step made of all of them."""
import numpy as np
import pytest
import torch

from oracle import q4
from paper_2504_09345_amd import binding as pb
from q4_util import Batch, check

from parity_util import announce

pytestmark = pytest.mark.gpu


# --- the cache write and read ------------------------------------------------

def _rows(b, seed, odd=False):
    """New rows of widely different sizes, as the call's type holds them."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((b.T, b.H_kv, b.D)) * np.exp(2 * rng.standard_normal((b.T, b.H_kv, 1)))
    if odd:
        flat = x.reshape(-1, 32)
        for i, y in enumerate([0.0, -0.0, 1e-38, 2.0 ** -133, 3e38, np.inf, -np.inf, np.nan]):
            flat[i::37, (5 * i) % 32] = y
        flat[3::41] = 0.0
        flat[4::43] *= 2.0 ** -126
        flat[5::47] = 1.75 * 2.0 ** 5 * np.tanh(rng.standard_normal(flat[5::47].shape))
        flat[5::47, 3] = 1.75 * 2.0 ** 5
    return b.round(x)


def _append(b, d, kn, vn, **kw):
    dt = b.torch_dtype
    rows = b.cuda(kn).to(dt)
    pb.pa_kv_append_q4(rows, b.cuda(vn).to(dt), d["bt"], d["cl"], d["k"], d["v"], b.dims(d, rows, **kw), query_start_loc=d["qsl"])


def _read(b, d, out=None, **kw):
    out = torch.full((2, b.T, b.H_kv, b.D), -3.0, dtype=b.torch_dtype, device="cuda") if out is None else out
    pb.pa_kv_read_q4(d["k"], d["v"], d["bt"], d["cl"], out[0], out[1], b.dims(d, out[0], **kw), query_start_loc=d["qsl"])
    return out.float().cpu().numpy()


LENS = [(1, 1), (16, 16), (17, 3), (40, 40), (33, 1), (70, 6), (0, 0), (5, 5), (129, 30)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_kv", [1, 3, 8])
def test_append_and_read_varlen(dtype, D, H_kv):
    announce(f"q4 append varlen {dtype} D={D} H_kv={H_kv}")
    b = Batch(LENS, H_q=H_kv, H_kv=H_kv, D=D, dtype=dtype, seed=H_kv)
    kn, vn = _rows(b, 1, odd=True), _rows(b, 2, odd=True)
    ek, ev = q4.append(kn, vn, b.bt, b.ctx, b.k, b.v, b.qsl)
    d = b.upload()
    _append(b, d, kn, vn)
    assert np.array_equal(d["k"].cpu().numpy(), ek)
    assert np.array_equal(d["v"].cpu().numpy(), ev)
    got = _read(b, d)
    for x, new in ((got[0], kn), (got[1], vn)):
        assert np.array_equal(x.astype(np.float64), q4.values(*q4.quantise(new)), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_append_and_read_decode(dtype, D):
    announce(f"q4 append decode {dtype} D={D}")
    b = Batch([(c, 1) for c in (1, 0, 16, 17, 300, 0, 31)], H_q=4, H_kv=4, D=D, dtype=dtype, varlen=False)
    kn, vn = _rows(b, 1), _rows(b, 2)
    ek, ev = q4.append(kn, vn, b.bt, b.ctx, b.k, b.v)
    d = b.upload()
    _append(b, d, kn, vn)
    assert np.array_equal(d["k"].cpu().numpy(), ek)
    assert np.array_equal(d["v"].cpu().numpy(), ev)
    got = _read(b, d)
    live = b.ctx > 0
    assert np.array_equal(got[0][live], q4.values(*q4.quantise(kn))[live])
    assert np.array_equal(got[1][live], q4.values(*q4.quantise(vn))[live])
    assert (got[:, ~live] == -3.0).all()  # no row: left as it was


def test_read_whole_contexts():
    announce("q4 read whole contexts")
    b = Batch([(c, c) for c in (1, 47, 16, 0, 130, 64)], H_q=2, H_kv=2, D=128, spare=1)
    got = _read(b, b.upload())
    for i, (r0, r1) in enumerate(zip(b.qsl[:-1], b.qsl[1:])):
        for which, pool, x in (("k", b.k, got[0]), ("v", b.v, got[1])):
            ref = q4.dense(which, pool, b.bt, i, int(b.ctx[i]), b.D)
            assert np.array_equal(x[r0:r1].transpose(1, 0, 2).astype(np.float64), ref)


def test_rows_outside_the_contract():
    announce("q4 append and read, rows outside the contract")
    b = Batch([(20, 4), (40, 2), (33, 33), (18, 18), (9, 2)], H_q=2, H_kv=2, D=64)
    kn, vn = _rows(b, 1), _rows(b, 2)
    d = b.upload()
    ctx = b.ctx.copy()
    ctx[0] = 3        # a chunk longer than its context
    ctx[1] = 1000     # a context above max_context_len
    d["cl"] = b.cuda(ctx)
    bt = b.bt.copy()
    bt[2, 1], bt[3, 1] = -1, b.num_pages  # pages outside the pool: tokens 16 .. 31, 16, 17
    d["bt"] = b.cuda(bt)
    _append(b, d, kn, vn, max_context_len=48)
    keep = np.ones(b.T, bool)
    keep[:6] = False
    keep[6 + 16:6 + 32] = False
    keep[6 + 33 + 16:6 + 33 + 18] = False
    ek, ev = b.k.copy(), b.v.copy()
    for r, seq, pos in q4.rows_of(b.ctx, b.qsl):
        if keep[r]:
            for g in range(2):
                q4.put("k", ek, b.bt[seq, pos // 16], g, pos % 16, kn[r, g])
                q4.put("v", ev, b.bt[seq, pos // 16], g, pos % 16, vn[r, g])
    assert np.array_equal(d["k"].cpu().numpy(), ek) and np.array_equal(d["v"].cpu().numpy(), ev)
    got = _read(b, d, max_context_len=48)
    assert np.isnan(got[:, ~keep]).all()
    assert np.array_equal(got[0][keep], q4.values(*q4.quantise(kn))[keep])
    assert np.array_equal(got[1][keep], q4.values(*q4.quantise(vn))[keep])


def test_rows_behind_the_last_sequence():
    announce("q4 read and attention, rows behind the last sequence")
    b = Batch([(20, 4), (40, 1)], H_q=4, H_kv=2, D=64)
    d = b.upload()
    d["q"] = torch.cat([d["q"], d["q"][:3]])
    out = b.attend(d, b.dims(d, num_q_rows=b.T + 3), torch.full_like(d["q"], 7.0))
    assert (out[b.T:] == 7.0).all()
    check(out[:b.T].float().cpu(), b.expected(), 40, "bf16")
    rows = torch.full((2, b.T + 3, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    _read(b, d, rows, num_q_rows=b.T + 3)
    assert (rows[:, b.T:] == 7.0).all() and not (rows[:, :b.T] == 7.0).all(-1).any()


# --- attention ---------------------------------------------------------------

DECODE = [1, 15, 16, 17, 31, 32, 33, 0, 64, 200, 333, 48]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_q,H_kv", [(8, 8), (4, 2), (4, 1), (18, 3), (64, 8)])
def test_decode(dtype, D, H_q, H_kv):
    announce(f"q4 decode {dtype} D={D} heads={H_q}/{H_kv}")
    b = Batch([(c, 1) for c in DECODE], H_q, H_kv, D, dtype, seed=H_q, varlen=False)
    out = b.attend(b.upload())
    check(out.float().cpu(), b.expected(), max(DECODE), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_q,H_kv", [(2, 2), (4, 2), (4, 1), (6, 1), (16, 2)])
@pytest.mark.parametrize("lens", [
    [(1, 1), (40, 2), (33, 1), (0, 0), (18, 3)],                    # few rows each
    [(100, 7), (64, 64), (16, 1), (90, 33), (1, 1), (200, 5)],       # chunks beside decode rows
    [(130, 130), (150, 65)],                                         # chunks alone
], ids=["few", "mixed", "chunks"])
def test_varlen(dtype, D, H_q, H_kv, lens):
    announce(f"q4 varlen {dtype} D={D} heads={H_q}/{H_kv} {lens}")
    b = Batch(lens, H_q, H_kv, D, dtype, seed=len(lens))
    out = b.attend(b.upload())
    check(out.float().cpu(), b.expected(), max(c for c, _ in lens), dtype)


@pytest.mark.parametrize("n,ctx", [(1, 5000), (3, 2500)])
def test_long_contexts_are_cut_and_joined(n, ctx):
    announce(f"q4 decode {n} x {ctx}")
    b = Batch([(ctx - 100 * i, 1) for i in range(n)], 8, 2, 128, varlen=False, seed=n)
    d = b.upload()
    check(b.attend(d).float().cpu(), b.expected(), ctx, "bf16")
    # a declared bound far above the contexts changes the parts, not the result
    d["bt"] = torch.cat([d["bt"], d["bt"][:, :1].expand(-1, 4000 - d["bt"].shape[1])], 1).contiguous()
    check(b.attend(d, b.dims(d, max_context_len=64000)).float().cpu(), b.expected(), ctx, "bf16")


def test_chunk_of_few_rows_on_a_long_context():
    announce("q4 varlen 3 rows on 4000")
    b = Batch([(4000, 3), (50, 2), (3000, 1)], 8, 2, 64, "fp32", seed=5)
    check(b.attend(b.upload()).float().cpu(), b.expected(), 4000, "fp32")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_scores(D, dtype):
    announce(f"q4 decode, scores of hundreds D={D} {dtype}")
    b = Batch([(c, 1) for c in (300, 40, 700)], 8, 2, D, dtype, varlen=False, k_size=60.0)
    check(b.attend(b.upload()).float().cpu(), b.expected(), 700, dtype)


def test_nan_blocks_reach_the_rows_that_see_them():
    announce("q4 varlen, NaN blocks")
    b = Batch([(70, 40), (64, 1), (33, 33)], 4, 2, 128, seed=3)
    # V of sequence 0, token 45, head 1, block 2: rows from 45 - 30 = 15 on
    b.v[b.bt[0, 2], 1, q4.scale_byte_of(128, 13, 2)] = 255
    # K of sequence 2, token 20, head 0: rows from 20 on
    b.k[b.bt[2, 1], 0, q4.scale_byte_of(128, 4, 1)] = 255
    # V of sequence 1 (a decode row)
    b.v[b.bt[1, 0], 0, q4.scale_byte_of(128, 0, 3)] = 255
    ref = b.expected()
    assert np.isnan(ref[0]).any() and not np.isnan(ref[0][:15]).any()
    check(b.attend(b.upload()).float().cpu(), ref, 70, "bf16")


@pytest.mark.parametrize("varlen", [False, True])
def test_attention_rows_outside_the_contract(varlen):
    announce(f"q4 attention, rows outside the contract varlen={varlen}")
    b = Batch([(50, 1), (40, 1), (33, 1), (64, 1), (20, 1)] if not varlen else [(50, 5), (40, 3), (33, 20), (64, 1), (20, 2)],
              4, 2, 64, varlen=varlen)
    ref = b.expected()
    d = b.upload()
    ctx, bt = b.ctx.copy(), b.bt.copy()
    ctx[0] = 5000                 # above max_context_len
    bt[2, 1] = b.num_pages + 7    # outside the pool
    bt[3, 0] = -5
    d["cl"], d["bt"] = b.cuda(ctx), b.cuda(bt)
    out = b.attend(d, b.dims(d, max_context_len=64)).float().cpu().numpy()
    q0 = [0, 1, 2, 3, 4, 5] if not varlen else b.qsl
    ref[0][q0[0]:q0[1]] = np.nan
    for r in range(q0[2], q0[3]):
        if int(b.ctx[2]) - (q0[3] - r) >= 16:  # sees page 1
            ref[0][r] = np.nan
    ref[0][q0[3]:q0[4]] = np.nan
    check(out, ref, 64, "bf16")
    if varlen:  # a chunk longer than its context
        ctx[1] = 2
        d["cl"] = b.cuda(ctx)
        out = b.attend(d, b.dims(d, max_context_len=64)).float().cpu().numpy()
        ref[0][q0[1]:q0[2]] = np.nan
        check(out, ref, 64, "bf16")


def test_infinite_query():
    announce("q4 decode, a query that is not finite")
    b = Batch([(50, 1), (40, 1), (7, 1)], 4, 2, 64, varlen=False)
    b.q[1, 2, 5] = np.nan
    ref = b.expected()
    check(b.attend(b.upload()).float().cpu(), ref, 50, "bf16")


def test_a_serving_step():
    """Prompts are written and attend in chunks, then the same sequences decode:
    append, attention and the read back over the same pages, on a stream of its
    own, against the plain form."""
    announce("q4 serving steps")
    H_q, H_kv, D = 8, 2, 128
    rng = np.random.default_rng(8)
    b = Batch([(70, 70), (33, 33), (5, 5)], H_q, H_kv, D, seed=8)
    k, v, d = b.k, b.v, b.upload()
    stream = torch.cuda.Stream()
    width = 8
    bt = np.concatenate([b.bt, np.zeros((3, width - b.bt.shape[1]), np.int32)], 1)
    free = [p for p in range(b.num_pages) if p not in set(b.bt[0, :5]) | set(b.bt[1, :3]) | set(b.bt[2, :1])]
    bt[0, 5], bt[1, 3], bt[2, 1] = free[:3]
    ctx = b.ctx.copy()
    for step in range(3):
        qsl = b.qsl if step == 0 else np.arange(4, dtype=np.int32)
        T = int(qsl[-1])
        kn, vn, q = (b.round(rng.standard_normal((T, h, D))) for h in (H_kv, H_kv, H_q))
        k, v = q4.append(kn, vn, bt, ctx, k, v, qsl)
        ref = q4.attention(q, k, v, bt, ctx, b.scale, qsl)
        with torch.cuda.stream(stream):
            dk, dv, dq = (b.cuda(x).to(torch.bfloat16) for x in (kn, vn, q))
            dbt, dcl, dqsl = b.cuda(bt), b.cuda(ctx), b.cuda(qsl)
            out, back = torch.empty_like(dq), torch.empty((2,) + dk.shape, dtype=torch.bfloat16, device="cuda")
            dims = pb.make_dims_q4(dk, d["k"], dbt, 128, num_q_rows=T, max_q_len=int(np.diff(qsl).max()))
            pb.pa_kv_append_q4(dk, dv, dbt, dcl, d["k"], d["v"], dims, query_start_loc=dqsl)
            dims.num_q_heads = H_q
            pb.paged_attn_varlen_q4(dq, d["k"], d["v"], dbt, dcl, dqsl, b.scale, out, dims)
            pb.pa_kv_read_q4(d["k"], d["v"], dbt, dcl, back[0], back[1], dims, query_start_loc=dqsl)
        stream.synchronize()
        check(out.float().cpu(), ref, 80, "bf16", f"step {step}")
        assert np.array_equal(back[0].float().cpu().numpy(), q4.values(*q4.quantise(kn)))
        assert np.array_equal(back[1].float().cpu().numpy(), q4.values(*q4.quantise(vn)))
        ctx = ctx + 1
    assert np.array_equal(d["k"].cpu().numpy(), k) and np.array_equal(d["v"].cpu().numpy(), v)


# --- the decode kernel's division of work ------------------------------------

@pytest.mark.parametrize("H_kv", [1, 2, 4, 8])
@pytest.mark.parametrize("n,lo,hi", [(1, 2000, 2000), (3, 900, 1500), (40, 1, 700), (7, 33, 64)])
def test_decode_ranges(H_kv, n, lo, hi):
    """Items cut over several ranges, in one and two levels of joins, for every
    number of waves per team; the same bits every time."""
    announce(f"q4 decode ranges H_kv={H_kv} {n} x {lo}-{hi}")
    rng = np.random.default_rng(H_kv + n)
    b = Batch([(int(c), 1) for c in rng.integers(lo, hi + 1, n)], 2 * H_kv, H_kv, 64, varlen=False, seed=n)
    d = b.upload()
    first = b.attend(d)
    check(first.float().cpu(), b.expected(), hi, "bf16")
    ws = torch.full((pb.pa_workspace_size_q4(b.dims(d)),), 0xA5, dtype=torch.uint8, device="cuda")
    for fill in (0xA5, 0xFF):
        ws.fill_(fill)
        assert torch.equal(b.attend(d, workspace=ws), first)
    for _ in range(3):
        assert torch.equal(b.attend(d, workspace=ws), first)


@pytest.mark.parametrize("B,ctx", [(8192, 4224), (9000, 40)])
def test_many_sequences_share_their_pages(B, ctx):
    """More sequences than a launch takes; and ranges of more units than a table
    holds.  All sequences read the same pages and a few different queries."""
    announce(f"q4 decode {B} sequences of {ctx}")
    one = Batch([(ctx, 1)], 1, 1, 64, varlen=False)
    d = one.upload()
    q = one.cuda(one.round(np.random.default_rng(1).standard_normal((8, 1, 64)))).to(torch.bfloat16)
    which = torch.arange(B, device="cuda") * 7 % 8
    d["q"] = q[which].contiguous()
    d["bt"] = d["bt"].expand(B, -1).contiguous()
    d["cl"] = d["cl"].expand(B).contiguous()
    out = one.attend(d)
    ref = [q4.attention(q[i:i + 1].float().cpu().numpy(), one.k, one.v, one.bt, one.ctx, one.scale) for i in range(8)]
    ref = [np.concatenate([r[j] for r in ref]) for j in range(5)]
    for i in range(8):
        mine = out[which == i].float().cpu()
        check(mine, [np.repeat(r[i:i + 1], len(mine), 0) for r in ref], ctx, "bf16")


def test_mixed_call_with_wrong_max_q_len():
    announce("q4 varlen, chunks longer than max_q_len")
    b = Batch([(40, 9), (33, 1), (64, 4)], 4, 2, 64)
    d = b.upload()
    for most, nan in ((1, (0, 2)), (4, (0,))):
        ref = b.expected()
        for i in nan:
            ref[0][b.qsl[i]:b.qsl[i + 1]] = np.nan
        check(b.attend(d, b.dims(d, max_q_len=most)).float().cpu(), ref, 64, "bf16")


def test_captured_calls_replay():
    """A step recorded once and replayed on other contents, with eager calls on
    the same workspace between the replays."""
    announce("q4 captured step")
    H_q, H_kv, D = 8, 2, 128
    b = Batch([(300, 1), (70, 20), (1000, 1)], H_q, H_kv, D, seed=4)
    d = b.upload()
    rows = torch.zeros((2, b.T, H_kv, D), dtype=torch.bfloat16, device="cuda")
    dims = b.dims(d)
    ws = torch.empty(pb.pa_workspace_size_q4(dims), dtype=torch.uint8, device="cuda")
    out, back = torch.empty_like(d["q"]), torch.empty_like(rows)

    def step():
        pb.pa_kv_append_q4(rows[0], rows[1], d["bt"], d["cl"], d["k"], d["v"], dims, query_start_loc=d["qsl"])
        b.attend(d, dims, out, workspace=ws)
        pb.pa_kv_read_q4(d["k"], d["v"], d["bt"], d["cl"], back[0], back[1], dims, query_start_loc=d["qsl"])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rows.copy_(torch.randn(rows.shape, device="cuda", generator=g))
        d["q"].copy_(torch.randn(d["q"].shape, device="cuda", generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), back.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, got[0]) and torch.equal(back, got[1])
        ref = q4.attention(d["q"].float().cpu().numpy(), d["k"].cpu().numpy(), d["v"].cpu().numpy(), b.bt, b.ctx, b.scale, b.qsl)
        check(got[0].float().cpu(), ref, 1000, "bf16")


@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** -25, 2.0 ** 9, 2.0 ** 60])
@pytest.mark.parametrize("D", [64, 128])
def test_values_of_any_size(D, size):
    """V far outside fp16's range, in all or some of the units."""
    announce(f"q4 attention, V of size {size} D={D}")
    b = Batch([(100, 20), (90, 1), (33, 1)], 8, 2, D, seed=1)
    for page in b.bt[0, ::2].tolist() + b.bt[1].tolist():
        at = [q4.scale_byte_of(D, t, j) for t in range(16) for j in range(D // 32)]
        b.v[page][:, at] = np.clip(b.v[page][:, at].astype(int) + int(np.log2(size)), 2, 252)
    check(b.attend(b.upload()).float().cpu(), b.expected(), 100, "bf16")


@pytest.mark.parametrize("D", [64, 128])
def test_queries_of_any_size(D):
    """Queries from the smallest to large ones, and of very different sizes in one row."""
    announce(f"q4 decode, queries of any size D={D}")
    b = Batch([(100, 1)] * 8, 8, 2, D, seed=2, varlen=False)
    for i, f in enumerate([0.0, 2.0 ** -130, 2.0 ** -60, 2.0 ** -10, 1.0, 30.0, 1.0, 1.0]):
        b.q[i] *= f
    b.q[6] *= np.exp2(-np.arange(D) / 4.0).astype(np.float32)
    b.q[7, :, ::2] *= 2.0 ** -20
    b.q = b.round(b.q)
    check(b.attend(b.upload()).float().cpu(), b.expected(), 100, "bf16")


# --- workgroups that share V (large calls) -----------------------------------

FAR = 1 << 20  # a declared context that makes a call's work large enough for them


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_q,H_kv", [(34, 34), (68, 34), (8, 2), (6, 1), (16, 2)])
@pytest.mark.parametrize("lens", [
    [(100, 7), (64, 64), (16, 1), (90, 33), (1, 1), (0, 0), (200, 50)],
    [(130, 130), (150, 65)],
    [(300, 40)],
], ids=["mixed", "chunks", "one"])
def test_shared(D, H_q, H_kv, lens):
    """The sizes where such a workgroup can go wrong, its kernel chosen by a declared
    context far above the real ones."""
    announce(f"q4 shared D={D} heads={H_q}/{H_kv} {lens}")
    b = Batch(lens, H_q, H_kv, D, seed=len(lens))
    d = b.upload()
    b.widen(d, FAR)
    check(b.attend(d, b.dims(d, max_context_len=FAR)).float().cpu(), b.expected_gpu(), max(c for c, _ in lens), "bf16")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_q,H_kv", [(32, 8), (48, 8), (8, 1)])
@pytest.mark.parametrize("lens", [
    [(1000, 256)] * 9 + [(300, 1), (1, 1)],      # whole items
    [(5000, 100), (4700, 120), (33, 2)],          # items in parts
    [(2600, 2600)],
], ids=["items", "parts", "prompt"])
def test_shared_at_size(D, H_q, H_kv, lens):
    announce(f"q4 shared at size D={D} heads={H_q}/{H_kv} {lens[0]}")
    b = Batch(lens, H_q, H_kv, D, seed=9)
    check(b.attend(b.upload()).float().cpu(), b.expected_gpu(), max(c for c, _ in lens), "bf16")


@pytest.mark.parametrize("D", [64, 128])
def test_shared_nan_blocks_and_any_size(D):
    """A NaN block reaches the rows that see it, units outside fp16's window are exact
    beside it, and a page outside the pool reaches the rows that see it."""
    announce(f"q4 shared, NaN blocks and V of any size D={D}")
    b = Batch([(170, 140), (64, 1), (100, 90)], 8, 2, D, seed=3)
    d = b.upload()
    b.v[b.bt[0, 2], 1, q4.scale_byte_of(D, 13, 1)] = 255   # token 45: rows from 15 on
    b.k[b.bt[2, 1], 0, q4.scale_byte_of(D, 4, 0)] = 255    # token 20: rows from 10 on
    for page, e in ((b.bt[0, 5], 60), (b.bt[2, 0], -40), (b.bt[1, 1], 20)):
        at = [q4.scale_byte_of(D, t, j) for t in range(16) for j in range(D // 32)]
        b.v[page][:, at] = np.clip(b.v[page][:, at].astype(int) + e, 2, 252)
    ref = b.expected()
    assert np.isnan(ref[0]).any() and not np.isnan(ref[0][:15]).any()
    bt = b.bt.copy()
    bt[2, 4] = b.num_pages  # tokens 64 .. 79: rows from 54 on
    ref[0][141 + 54:] = np.nan
    d.update(k=b.cuda(b.k), v=b.cuda(b.v), bt=b.cuda(bt))
    b.widen(d, FAR)
    check(b.attend(d, b.dims(d, max_context_len=FAR)).float().cpu(), ref, 170, "bf16")
