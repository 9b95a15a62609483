"""What a serving step does with new rows when the cache is held in 8 bits, each
operator through the public binding: rotary positions of q and k (``pa_rope``), the
rows quantised into the cache (``pa_kv_append_q8``) and read back
(``pa_kv_read_q8``), and attention over it for decode rows (``paged_attn_q8``) and
for prompt chunks beside them (``paged_attn_varlen_q8``).

With ``own`` false the same results come from elementary torch operations in 32
bits (angles in 64).  ``listed()`` names the fixed cases and ``draw(rng)`` gives
another one of the same ranges.  Context and chunk lengths follow from a case alone
(``lens`` seeds them), so its work is known without its inputs, while every number
in the inputs, and the place of every page, comes from the seed that ``prepare``
takes.

The rotation: pair i of a vector's first ``rot`` dims, (x, y), at position p becomes
f (x cos a - y sin a, y cos a + x sin a) with a = p w_i; the pair is dims i and
i + rot / 2 or, interleaved, dims 2 i and 2 i + 1.  w is given in 64 bits.

The cache: the 16 tokens of a page share, per KV head and for K and V each, a
power-of-two scale; elements are e4m3 (4 exponent bits, bias 7; 3 mantissa bits;
codes 127 and 255 are NaN; the largest is 448).  With a = max |x| over the finite x of
the tokens that the page holds, a = m 2^k, 1 <= m < 2, the scale is 2^e with e = k - 8
where m <= 1.75 and k - 7 otherwise, kept within -110 .. 119, stored as the byte
e + 127 of scales [page][KV head][K, V].  x is held as x / 2^e to the nearest e4m3,
ties to even, at most 448 in magnitude; what is not finite is held as NaN.  A token
written to a page that holds earlier ones raises the scale where its own needs more;
the earlier ones' values are then rounded to the new scale.  Byte of token t and dim d
of a (page, KV head) tile of 16 D:
  K  ((d / 16) 16 + t) 16 + d mod 16
  V  (d / 64) 1024 + ((t / 4) 16 + d mod 32 / 2) 16 + (d / 32 mod 2) 8 + (d mod 2) 4 + t mod 4
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
E_LOW, E_HIGH = -110, 119


# --- the cases ---------------------------------------------------------------

def _case(name, kind, dtype="bf16", H_q=32, H_kv=8, D=128, chunks=0, chunk=(1, 1), prior=(0, 0), B=0, ctx=(1, 1), rot=128,
          interleaved=False, packed=False, stretch=1, lens=1):
    c = dict(name=name, kind=kind, dtype=dtype, H_q=H_q, H_kv=H_kv, D=D, chunks=chunks, chunk_lo=chunk[0], chunk_hi=chunk[1],
             prior_lo=prior[0], prior_hi=prior[1], B=B, ctx_lo=ctx[0], ctx_hi=ctx[1], lens=lens)
    if kind == "rope":  # packed: q and k lie in rows of q, k and v; stretch: how often the trained length fits the context
        c.update(rot=rot, interleaved=interleaved, packed=packed, stretch=stretch)
    return c if name else {k: v for k, v in c.items() if k != "name"}


def listed():
    return [
        # a decode step's new rows: one for each of 256 sequences, out of the joint projection
        _case("rope-step-256", "rope", B=256, ctx=(512, 2048), packed=True),
        # prompts at the far end of long contexts, half of each vector rotated, the other layout
        _case("rope-prompts-far", "rope", chunks=8, chunk=(100, 2048), prior=(0, 120000), rot=64, interleaved=True, stretch=32),
        # the cache write of a decode step: one new token for each of 256 sequences
        _case("append-step-256", "append", B=256, ctx=(512, 2048)),
        # the cache write of a prefill-heavy step: prompts of any length, some behind a cached prefix
        _case("append-prompts", "append", chunks=8, chunk=(100, 2048), prior=(0, 1000)),
        # one conversation leaves the cache (or is branched): all of its rows read back
        _case("read-1x4001", "read", B=1, ctx=(4001, 4001)),
        # a batch's caches read back for 32-bit work, the other head dim
        _case("read-d64-fp32-64", "read", dtype="fp32", D=64, B=64, ctx=(512, 2048)),
        # one user, a short conversation: the launch and its latency are all there is
        _case("decode-b1-ctx200", "decode", B=1, ctx=(200, 200)),
        # a full decode batch (Mixtral-8x7B heads, 256 sequences)
        _case("decode-mixtral-256", "decode", B=256, ctx=(512, 2048)),
        # a few very long contexts; 32-bit queries, the other head dim, a wide group
        _case("decode-long-d64-fp32-4", "decode", dtype="fp32", H_q=64, D=64, B=4, ctx=(8192, 32768)),
        # one prompt of odd length arrives alone: the time to its first token
        _case("prefill-1x700", "varlen", chunks=1, chunk=(700, 700)),
        # a prefill-heavy step, the largest work
        _case("prefill-8x2048", "varlen", chunks=8, chunk=(2048, 2048), prior=(0, 2048)),
        # the mixed step of continuous batching
        _case("mixed-8x512-512", "varlen", chunks=8, chunk=(512, 512), prior=(0, 1536), B=512, ctx=(256, 4096)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    lens = rng.randrange(1 << 20)
    H_kv = rng.choice([1, 2, 4, 8, 8, 8])
    H_q = H_kv * rng.choice([1, 2, 4, 4, 6, 8])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    heads = dict(dtype=dtype, H_q=H_q, H_kv=H_kv, D=rng.choice([64, 128, 128]), lens=lens)
    row = H_kv * heads["D"]
    r = rng.random()
    if r < 0.15:
        more = dict(rot=rng.choice([heads["D"], heads["D"], heads["D"] // 2, 32, 2 * rng.randint(1, heads["D"] // 2)]),
                    interleaved=rng.random() < 0.4, packed=rng.random() < 0.4, stretch=rng.choice([1, 1, 4, 32]))
        prior = _log_int(rng, 1, 1000000)
        if rng.random() < 0.4:
            return _case("", "rope", B=_log_int(rng, 1, 512), ctx=(max(1, prior // 3), prior), **more, **heads)
        chunk = _log_int(rng, 2, 2048)
        return _case("", "rope", chunks=max(1, min(_log_int(rng, 1, 16), 8 * 2048 * 5120 // (chunk * (H_q + H_kv) * heads["D"]))),
                     chunk=(max(1, chunk // 3), chunk), prior=(0, prior), B=rng.randint(0, 40), ctx=(1, prior), **more, **heads)
    if r < 0.3:
        if rng.random() < 0.5:
            return _case("", "append", B=_log_int(rng, 1, 512), ctx=(1, _log_int(rng, 20, 4000)), **heads)
        chunk = _log_int(rng, 2, 2048)
        return _case("", "append", chunks=max(1, min(_log_int(rng, 1, 16), 8192 * 1024 // (chunk * row))),
                     chunk=(max(1, chunk // 3), chunk), prior=(0, _log_int(rng, 1, 2000)), B=rng.randint(0, 40), ctx=(1, 500), **heads)
    mean = _log_int(rng, 20, 20000)
    if r < 0.42:
        B = max(1, min(_log_int(rng, 1, 256), 64 * 1280 * 512 // (mean * row)))
        return _case("", "read", B=B, ctx=(max(1, mean // 3), mean + mean // 2), **heads)
    if r < 0.7:
        B = max(1, min(_log_int(rng, 1, 512), 256 * 1280 * 1024 // (mean * row)))
        return _case("", "decode", B=B, ctx=(max(1, mean // 3), mean + mean // 2), **heads)
    # what chunks cost is bounded by their (row, key) pairs
    chunk, prior = _log_int(rng, 2, 2048), rng.choice([0, 0, _log_int(rng, 16, 4096)])
    pairs = (8 * 2048 * 2048 if dtype == "bf16" else 2048 * 2048) * 32 / H_q
    chunks = max(1, min(_log_int(rng, 1, 16), int(pairs / (chunk * (chunk / 2 + prior)))))
    B = 0 if r < 0.85 else min(_log_int(rng, 1, 256), 256 * 1024 * 1024 // (2000 * row))
    return _case("", "varlen", chunks=chunks, chunk=(max(2, chunk - chunk // 4), chunk), prior=(prior // 2, prior), B=B, ctx=(1, 2000), **heads)


# --- lengths and work --------------------------------------------------------

def _lengths(case):
    """(context length, rows) of each sequence: the chunks, then the others (one
    row each, or for a read all of them)."""
    r = random.Random(case["lens"])
    rows = [r.randint(case["chunk_lo"], case["chunk_hi"]) for _ in range(case["chunks"])]
    ctx = [n + r.randint(case["prior_lo"], case["prior_hi"]) for n in rows]
    more = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["B"])]
    return ctx + more, rows + (more if case["kind"] == "read" else [1] * len(more))


def _page_rows(ctx, rows):
    """Rows of the pages that an append writes, from each sequence's first such page on."""
    return [n + (c - n) % PAGE for c, n in zip(ctx, rows)]


def work(case):
    ctx, rows = _lengths(case)
    es = 2 if case["dtype"] == "bf16" else 4
    H_q, H_kv, D = case["H_q"], case["H_kv"], case["D"]
    T = sum(rows)
    if case["kind"] == "rope":
        return {"bytes": float(2 * T * (H_q + H_kv) * D * es + 8 * len(ctx) + 4 * case["rot"]), "flops": 3.0 * T * (H_q + H_kv) * case["rot"]}
    # a page's entry, and its scales per KV head
    pages = sum((c + PAGE - 1) // PAGE for c in ctx)
    table = (4 + 2 * H_kv) * pages + 8 * len(ctx)
    if case["kind"] == "append":
        # rows in, their codes out; and the values of the pages that they lie in, read back
        back = _page_rows(ctx, rows)
        table = (4 + 4 * H_kv) * sum((n + PAGE - 1) // PAGE for n in back) + 8 * len(ctx)
        return {"bytes": float(2 * H_kv * D * (T * (es + 1) + sum(back) * (es + 1)) + table), "flops": 0.0}
    if case["kind"] == "read":
        return {"bytes": float(2 * T * H_kv * D * (es + 1) + table), "flops": 0.0}
    pairs = sum(L * (C - L) + L * (L + 1) // 2 for C, L in zip(ctx, rows))
    return {"bytes": float(2 * sum(ctx) * H_kv * D + 2 * T * H_q * D * es + table), "flops": 4.0 * D * H_q * pairs}


# --- the plain form ----------------------------------------------------------

def _k_bytes(D, device):
    """[token][dim] -> byte of a K tile; _v_bytes: of a V tile."""
    t, d = torch.arange(PAGE, device=device)[:, None], torch.arange(D, device=device)
    return (d // 16 * 16 + t) * 16 + d % 16


def _v_bytes(D, device):
    t, d = torch.arange(PAGE, device=device)[:, None], torch.arange(D, device=device)
    return d // 64 * 1024 + (t // 4 * 16 + d % 32 // 2) * 16 + d // 32 % 2 * 8 + d % 2 * 4 + t % 4


def _power(e):
    """2^e in 32 bits, -126 <= e <= 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _needed(x):
    """Exponents [...] that x [..., tokens, D] needs."""
    a = torch.where(torch.isfinite(x), x.abs(), 0).amax((-2, -1))
    return (((a.view(torch.int32) + 0x1FFFFF) >> 23) - 135).clamp(E_LOW, E_HIGH)


def _codes(x, e):
    """Codes (uint8) of x [..., tokens, D] with scales 2^e."""
    y = (x * _power(-e)[..., None, None]).clamp(-448, 448)
    return torch.where(torch.isfinite(x), y, math.nan).to(torch.float8_e4m3fn).view(torch.uint8)


def _values(codes, e):
    return codes.view(torch.float8_e4m3fn).float() * _power(e)[..., None, None]


def _pack(x, places):
    """Tiles [N, H_kv, 16 D] and exponents [N, H_kv] of x [N, H_kv, 16, D]."""
    e = _needed(x)
    return _codes(x, e).flatten(-2)[..., torch.argsort(places.flatten())].contiguous(), e


def _unpack(tiles, places):
    """Codes [..., 16, D] of tiles [..., 16 D]."""
    return tiles[..., places.flatten()].unflatten(-1, (PAGE, -1))


def _write(st, name, which, x):
    """The rows x [T, H_kv, D] into the pages that st lists."""
    pool, places, page = st[name], st[name + "_places"], st["page"]
    held, e0 = _unpack(pool[page], places), st["scales"][page, :, which].int() - 127
    early = torch.arange(PAGE, device=page.device) < st["first"][:, None]
    fresh = st["row"] >= 0
    old = torch.where(early[:, None, :, None], _values(held, e0), 0)
    new = x.float()[st["row"].clamp(min=0)].transpose(1, 2)
    new = torch.where(fresh[:, None, :, None], new, 0)
    e = _needed(new)
    e = torch.where((st["first"] > 0)[:, None], torch.maximum(e, e0), e)
    codes = torch.where(fresh[:, None, :, None], _codes(new, e), torch.where(early[:, None, :, None], _codes(old, e), held))
    pool[page] = codes.flatten(-2)[..., torch.argsort(places.flatten())]
    st["scales"][page, :, which] = (e + 127).to(torch.uint8)


def _read(st, name, which, page, slot):
    """[T, H_kv, D] in 32 bits, of slot[T] of page[T]."""
    pool, places = st[name], st[name + "_places"]
    g = torch.arange(pool.shape[1], device=page.device)[None, :, None]
    codes = pool[page[:, None, None], g, places[slot][:, None]]
    return _values(codes[:, :, None], st["scales"][page, :, which].int() - 127)[:, :, 0]


def _whole(st, name, which, pages):
    """[n, H_kv, tokens, D] in 32 bits, of the pages [n, P]."""
    x = _values(_unpack(st[name][pages], st[name + "_places"]), st["scales"][pages][..., which].int() - 127)
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)


def _attend(st, group):
    """Attention rows of the sequences of `group`, padded to its longest."""
    case = st["case"]
    H_kv, D, s = case["H_kv"], case["D"], case["H_q"] // case["H_kv"]
    pages, rows, L = group["pages"], group["rows"], group["rows"].shape[1]
    k = _whole(st, "k", 0, pages)
    q = st["q"][rows].float().view(-1, L, H_kv, s, D).permute(0, 2, 3, 1, 4).reshape(-1, H_kv, s * L, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(st["scale"]).view(-1, H_kv, s, L, k.shape[2])
    hidden = torch.arange(k.shape[2], device=k.device) > group["last"][:, :, None]
    x.masked_fill_(hidden[:, None, None], -math.inf)
    x -= x.amax(-1, keepdim=True)
    x.exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(-1, H_kv, s * L, k.shape[2]), _whole(st, "v", 1, pages)).view(-1, H_kv, s, L, D)
    o = (o / total).permute(0, 3, 1, 2, 4).reshape(-1, case["H_q"], D)
    st["out"][rows.flatten()[group["real"]]] = o[group["real"]].to(st["out"].dtype)


def _rotate(x, cos, sin, interleaved):
    """x [T, H, D] with its first pairs rotated; cos, sin [T, 1, pairs]."""
    n = cos.shape[-1]
    f = x.float()
    a, b = (f[..., 0:2 * n:2], f[..., 1:2 * n:2]) if interleaved else (f[..., :n], f[..., n:2 * n])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([turned, f[..., 2 * n:]], -1).to(x.dtype)


# --- inputs ------------------------------------------------------------------

def _frequencies(case):
    """The pairs' angles per token, and the factor of the rotated values: base 10000,
    or for a context `stretch` times the trained 4096 tokens the pairs that turn less
    than once in those slowed by it, those of 32 turns or more left, between them a
    ramp."""
    n, stretch = case["rot"] // 2, case["stretch"]
    w = [10000.0 ** (-i / n) for i in range(n)]
    if stretch == 1:
        return w, 1.0
    keep = [min(1.0, max(0.0, (4096 * x / (2 * math.pi) - 1) / 31)) for x in w]
    return [x * (k + (1 - k) / stretch) for x, k in zip(w, keep)], 0.1 * math.log(stretch) + 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    H_q, H_kv, D = case["H_q"], case["H_kv"], case["D"]
    ctx, rows = _lengths(case)
    B, T = len(ctx), sum(rows)

    def normal(*shape):
        return torch.randn(shape, dtype=dt, device="cuda", generator=g)

    starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    pos = np.concatenate([np.arange(c - n, c) for c, n in zip(ctx, rows)])
    st = dict(case=case, ctx=ctx, n_rows=rows, starts=starts, cl=torch.tensor(ctx, dtype=torch.int32, device="cuda"),
              qsl=torch.from_numpy(starts).cuda(), max_ctx=max(ctx), max_q=max(rows), scale=1.0 / math.sqrt(D))
    if case["kind"] == "rope":
        if case["packed"]:
            joint = normal(T, H_q + 2 * H_kv, D)
            st["q"], st["k"] = joint[:, :H_q], joint[:, H_q:H_q + H_kv]
        else:
            st["q"], st["k"] = normal(T, H_q, D), normal(T, H_kv, D)
        st["q_out"], st["k_out"] = (torch.empty((T, H, D), dtype=dt, device="cuda") for H in (H_q, H_kv))
        w, st["factor"] = _frequencies(case)
        st["w"] = torch.tensor(w, dtype=torch.float64, device="cuda")
        st["pos"] = torch.from_numpy(pos).cuda()
        return st

    n_pages = [(c + PAGE - 1) // PAGE for c in ctx]
    need, width = sum(n_pages), max(n_pages)
    num_pages = max(need + 1, math.ceil(1.25 * need))
    # keys vary in size from channel to channel, tokens of either from one to the next
    channels = torch.exp(0.6 * torch.randn((H_kv, 1, D), device="cuda", generator=g))
    perm = torch.randperm(num_pages, device="cuda", generator=g).to(torch.int32).cpu().numpy()
    table = np.full((B, width), perm[need], np.int32)  # unused entries: a page nobody owns
    at = 0
    for b, n in enumerate(n_pages):
        table[b, :n] = perm[at:at + n]
        at += n
    st.update(k_places=_k_bytes(D, "cuda"), v_places=_v_bytes(D, "cuda"), table=table, bt=torch.from_numpy(table).cuda())

    def tokens():
        return torch.exp(0.3 * torch.randn((num_pages, H_kv, PAGE, 1), device="cuda", generator=g))

    st["scales"] = torch.empty((num_pages, H_kv, 2), dtype=torch.uint8, device="cuda")
    for which, (name, size) in enumerate((("k", channels), ("v", 1.0))):
        x = torch.randn((num_pages, H_kv, PAGE, D), device="cuda", generator=g)
        x *= size
        x *= tokens()
        st[name], e = _pack(x, st[name + "_places"])
        st["scales"][:, :, which] = (e + 127).to(torch.uint8)
        del x
    if case["kind"] in ("append", "read"):
        if case["kind"] == "append":
            more = torch.exp(0.3 * torch.randn((2, T, H_kv, 1), device="cuda", generator=g))
            st["k_new"] = (channels.view(H_kv, D) * normal(T, H_kv, D) * more[0]).to(dt)
            st["v_new"] = (normal(T, H_kv, D) * more[1]).to(dt)
            # the pages written: where, the first slot written, the row of each slot
            page, first, row = [], [], []
            for b, (c, n) in enumerate(zip(ctx, rows)):
                for p in range((c - n) // PAGE, n_pages[b]):
                    page.append(table[b, p])
                    first.append(max(0, c - n - p * PAGE))
                    t = np.arange(p * PAGE, (p + 1) * PAGE)
                    row.append(np.where((t >= c - n) & (t < c), starts[b] + t - (c - n), -1))
            st["page"] = torch.tensor(np.array(page, np.int64), device="cuda")
            st["first"] = torch.tensor(first, device="cuda")
            st["row"] = torch.from_numpy(np.stack(row)).cuda()
            back = _page_rows(ctx, rows)
        else:
            back = rows
        st["back"] = torch.from_numpy(np.concatenate([[0], np.cumsum(back)]).astype(np.int32)).cuda()
        st["max_back"] = max(back)
        st["k_out"], st["v_out"] = (torch.empty((sum(back), H_kv, D), dtype=dt, device="cuda") for _ in range(2))
        pos = np.concatenate([np.arange(c - n, c) for c, n in zip(ctx, back)])
        st["back_page"] = torch.from_numpy(table[np.repeat(np.arange(B), back), pos // PAGE].astype(np.int64)).cuda()
        st["back_slot"] = torch.from_numpy(pos % PAGE).cuda()
        return st
    st["q"] = normal(T, H_q, D)
    st["out"] = torch.empty_like(st["q"])
    # the plain form's batches: the chunks, and the single rows
    st["groups"] = []
    for lo, hi in ((0, case["chunks"]), (case["chunks"], B)):
        if lo < hi:
            n, c = np.array(rows[lo:hi])[:, None], np.array(ctx[lo:hi])[:, None]
            j = np.arange(n.max())
            real = j < n
            row, last = np.where(real, starts[lo:hi, None] + j, 0), np.where(real, c - n + j, 0)
            pages = table[lo:hi, :(c.max() + PAGE - 1) // PAGE].astype(np.int64)
            st["groups"].append(dict(pages=torch.from_numpy(pages).cuda(), rows=torch.from_numpy(row).cuda(), last=torch.from_numpy(last).cuda(),
                                     real=torch.from_numpy(np.flatnonzero(real)).cuda()))
    st["ws"] = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    return st


# --- one pass ----------------------------------------------------------------

def _run_own(st):
    from paper_2504_09345_amd import binding as pb
    kind = st["case"]["kind"]
    if kind == "rope":
        varlen = st["max_q"] > 1
        dims = pb.make_dims_rope(st["q"], st["k"], st["max_ctx"], num_q_rows=st["q"].shape[0] if varlen else 0, num_seqs=len(st["ctx"]))
        pb.pa_rope(st["q"], st["k"], st["cl"], st["w"], st["q_out"], st["k_out"], dims, query_start_loc=st["qsl"] if varlen else None,
                   interleaved=st["case"]["interleaved"], factor=st["factor"])
        return dict(q=st["q_out"], k=st["k_out"])
    pool, cache = (st["k"], st["v"], st["scales"]), (st["bt"], st["cl"])
    if kind in ("append", "read"):
        if kind == "append":
            varlen = st["max_q"] > 1
            dims = pb.make_dims_q8(st["k_new"], st["k"], st["bt"], st["max_ctx"], num_q_rows=st["k_new"].shape[0] if varlen else 0, max_q_len=st["max_q"])
            pb.pa_kv_append_q8(st["k_new"], st["v_new"], *cache, *pool, dims, query_start_loc=st["qsl"] if varlen else None)
        dims = pb.make_dims_q8(st["k_out"], st["k"], st["bt"], st["max_ctx"], num_q_rows=st["k_out"].shape[0], max_q_len=st["max_back"])
        pb.pa_kv_read_q8(*pool, *cache, st["k_out"], st["v_out"], dims, query_start_loc=st["back"])
        return dict(k=st["k_out"], v=st["v_out"])
    if kind == "decode":
        dims = pb.make_dims_q8(st["q"], st["k"], st["bt"], st["max_ctx"])
        pb.paged_attn_q8(st["q"], *pool, *cache, st["scale"], st["out"], dims, workspace=st["ws"])
    else:
        dims = pb.make_dims_q8(st["q"], st["k"], st["bt"], st["max_ctx"], num_q_rows=st["q"].shape[0], max_q_len=st["max_q"])
        pb.paged_attn_varlen_q8(st["q"], *pool, *cache, st["qsl"], st["scale"], st["out"], dims, workspace=st["ws"])
    return dict(out=st["out"])


def run(st):
    if own:
        return _run_own(st)
    case = st["case"]
    if case["kind"] == "rope":
        angle = (st["pos"].double()[:, None] * st["w"])[:, None]
        cos, sin = ((f(angle) * st["factor"]).float() for f in (torch.cos, torch.sin))
        st["q_out"].copy_(_rotate(st["q"], cos, sin, case["interleaved"]))
        st["k_out"].copy_(_rotate(st["k"], cos, sin, case["interleaved"]))
        return dict(q=st["q_out"], k=st["k_out"])
    if case["kind"] in ("append", "read"):
        if case["kind"] == "append":
            _write(st, "k", 0, st["k_new"])
            _write(st, "v", 1, st["v_new"])
        for which, name in enumerate(("k", "v")):
            st[name + "_out"].copy_(_read(st, name, which, st["back_page"], st["back_slot"]))
        return dict(k=st["k_out"], v=st["v_out"])
    [_attend(st, group) for group in st["groups"]]
    return dict(out=st["out"])


# --- the same in 64 bits -----------------------------------------------------

def _power64(e):
    """2^e in float64, from its bits (torch's pow is off by a bit on some)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest64(y):
    """y to the nearest e4m3 value in float64: a multiple of the spacing at its
    magnitude, 2^-9 below 2^-6; torch.round goes to the even multiple."""
    spacing = _power64(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return (torch.round(y / spacing) * spacing).clamp(-448, 448)


def _exponent64(a):
    """The exponent that a largest magnitude needs."""
    m, k = torch.frexp(a)  # a = m 2^k, 1/2 <= m < 1
    return torch.where(a > 0, k - 9 + (m > 0.875).int(), E_LOW).clamp(E_LOW, E_HIGH)


def _e4m3_64(device):
    """The values of the 256 codes."""
    c = torch.arange(256, device=device)
    e, m = c // 8 % 16, (c % 8).double()
    x = torch.where(e > 0, (1 + m / 8) * _power64(e - 7), m / 8 * 2.0 ** -6)
    return torch.where(c % 128 == 127, math.nan, torch.where(c >= 128, -x, x))


def exact(case, seed):
    """What ``run`` returns for these inputs, from plain torch in float64."""
    st = prepare(case, seed)
    H_q, H_kv, D, s = case["H_q"], case["H_kv"], case["D"], case["H_q"] // case["H_kv"]
    if case["kind"] == "rope":
        angle = torch.outer(st["pos"].double(), st["w"])
        res = {}
        for name in ("q", "k"):
            x = st[name].double()
            turn = torch.polar(torch.full_like(angle, st["factor"]), angle)[:, None]
            n = case["rot"] // 2
            first = torch.arange(n, device="cuda") * (2 if case["interleaved"] else 1)
            second = first + (1 if case["interleaved"] else n)
            z = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = z.real, z.imag
            res[name] = x
        return res
    lut = _e4m3_64("cuda")
    order = dict(
        k=torch.tensor([[(d // 16 * 16 + t) * 16 + d % 16 for d in range(D)] for t in range(PAGE)], device="cuda"),
        v=torch.tensor([[d // 64 * 1024 + (t // 4 * 16 + d % 32 // 2) * 16 + d // 32 % 2 * 8 + d % 2 * 4 + t % 4 for d in range(D)]
                        for t in range(PAGE)], device="cuda"))

    def dense(name, which, pages):
        pages = torch.from_numpy(pages.astype(np.int64)).cuda()
        x = lut[st[name][pages][..., order[name]].long()]
        x *= _power64(st["scales"][pages][..., which].int() - 127)[..., None, None]
        return x.transpose(0, 1).reshape(H_kv, -1, D)

    if case["kind"] in ("append", "read"):
        res = dict(k=[], v=[])
        for b, (C, n) in enumerate(zip(st["ctx"], st["n_rows"])):
            from_page = (C - n) // PAGE
            for which, name in enumerate(("k", "v")):
                x = dense(name, which, st["table"][b, from_page:(C + PAGE - 1) // PAGE])[:, :C - from_page * PAGE]
                if case["kind"] == "append":
                    e0 = st["scales"][int(st["table"][b, from_page]), :, which].int() - 127
                    early, at = (C - n) % PAGE, int(st["starts"][b])
                    x[:, early:] = st[name + "_new"][at:at + n].double().transpose(0, 1)
                    x = torch.nn.functional.pad(x, (0, 0, 0, -x.shape[1] % PAGE)).view(H_kv, -1, PAGE, D)
                    new = x.clone()
                    new[:, 0, :early] = 0
                    e = _exponent64(new.abs().amax((-2, -1)))
                    if early:
                        e[:, 0] = torch.maximum(e[:, 0], e0)
                    p = _power64(e)[..., None, None]
                    x = (_nearest64(x / p) * p).view(H_kv, -1, D)[:, :early + n]
                res[name].append(x.transpose(0, 1))
        return {name: torch.cat(x) for name, x in res.items()}
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    for b, (C, L) in enumerate(zip(st["ctx"], st["n_rows"])):
        r0 = int(st["starts"][b])
        pages = st["table"][b, :(C + PAGE - 1) // PAGE]
        k, v = dense("k", 0, pages)[:, :C], dense("v", 1, pages)[:, :C]
        visible = torch.arange(C, device="cuda")[None, :] <= torch.arange(C - L, C, device="cuda")[:, None]
        for g in range(H_kv):
            q = st["q"][r0:r0 + L, g * s:(g + 1) * s].double().transpose(0, 1).reshape(s * L, D)
            x = torch.matmul(q, k[g].t().contiguous()).view(s, L, C) * st["scale"]
            p = torch.softmax(x.masked_fill_(~visible, -math.inf), dim=-1).view(s * L, C)
            out[r0:r0 + L, g * s:(g + 1) * s] = torch.matmul(p, v[g].contiguous()).view(s, L, D).transpose(0, 1)
    return dict(out=out)
