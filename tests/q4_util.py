"""Batches on a 4-bit cache for the tests, and the attention's error bound."""
import numpy as np

from oracle import q4
from paper_2504_09345_amd import binding as pb


class Batch:
    """Seeded sequences of (context, rows) on a pool whose pages are dealt at
    random and whose unused bytes (the slots past a context, the pages of nobody)
    hold anything, scales of NaN among them."""

    def __init__(self, lens, H_q=8, H_kv=2, D=128, dtype="bf16", seed=0, varlen=True, spare=3, k_size=1.0):
        rng = np.random.default_rng(seed)
        self.ctx = np.array([c for c, _ in lens], np.int32)
        self.n_rows = [n for _, n in lens] if varlen else [1] * len(lens)
        self.qsl = np.concatenate([[0], np.cumsum(self.n_rows)]).astype(np.int32) if varlen else None
        self.T, self.H_q, self.H_kv, self.D, self.dtype = sum(self.n_rows), H_q, H_kv, D, dtype
        pages = [-(-int(c) // 16) for c in self.ctx]
        self.num_pages = sum(pages) + spare
        width = max(pages + [1])
        perm = rng.permutation(self.num_pages).astype(np.int32)
        self.bt = np.full((len(lens), width), perm[-1], np.int32)
        self.k = rng.integers(0, 256, (self.num_pages, H_kv, q4.tile_bytes(D)), dtype=np.uint8)
        self.v = rng.integers(0, 256, self.k.shape, dtype=np.uint8)
        at = 0
        for b, n in enumerate(pages):
            self.bt[b, :n] = perm[at:at + n]
            at += n
        channels = np.exp(0.6 * rng.standard_normal((H_kv, 1, D))) * k_size
        live = np.zeros((self.num_pages, 16), bool)
        for b, c in enumerate(self.ctx):
            for p in range(pages[b]):
                live[self.bt[b, p], :min(16, int(c) - 16 * p)] = True
        for which, pool, size in (("k", self.k, channels), ("v", self.v, 1.0)):
            x = rng.standard_normal((self.num_pages, H_kv, 16, D)) * size
            tiles = q4.pack(which, x)
            for t in range(16):
                at = [q4.byte_of(which, D, t, m) for m in range(D // 2)] + [q4.scale_byte_of(D, t, j) for j in range(D // 32)]
                for i in np.flatnonzero(live[:, t]):
                    pool[i][:, at] = tiles[i][:, at]
        self.q = self.round(rng.standard_normal((self.T, H_q, D)))
        self.scale = 1 / np.sqrt(D)

    def round(self, x):
        """x as the call's type holds it, float32."""
        x = np.asarray(x, np.float32)
        if self.dtype == "fp32":
            return x
        u = x.view(np.uint32).astype(np.uint64)
        return (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)

    @property
    def torch_dtype(self):
        import torch
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32

    def cuda(self, x):
        import torch
        return torch.from_numpy(np.ascontiguousarray(x)).cuda()

    def upload(self):
        d = dict(k=self.cuda(self.k), v=self.cuda(self.v), bt=self.cuda(self.bt), cl=self.cuda(self.ctx),
                 q=self.cuda(self.q).to(self.torch_dtype))
        d["qsl"] = None if self.qsl is None else self.cuda(self.qsl)
        return d

    def dims(self, d, rows=None, max_context_len=None, num_q_rows=None, max_q_len=None):
        mcl = max(1, int(self.ctx.max())) if max_context_len is None else max_context_len
        if self.qsl is None:
            return pb.make_dims_q4(d["q"] if rows is None else rows, d["k"], d["bt"], mcl)
        return pb.make_dims_q4(d["q"] if rows is None else rows, d["k"], d["bt"], mcl,
                               num_q_rows=self.T if num_q_rows is None else num_q_rows,
                               max_q_len=max(self.n_rows) if max_q_len is None else max_q_len)

    def attend(self, d, dims=None, out=None, **kw):
        """The call's output, a device tensor (NaN where it wrote nothing)."""
        import torch
        out = torch.full_like(d["q"], float("nan")) if out is None else out
        dims = self.dims(d) if dims is None else dims
        if self.qsl is None:
            pb.paged_attn_q4(d["q"], d["k"], d["v"], d["bt"], d["cl"], self.scale, out, dims, **kw)
        else:
            pb.paged_attn_varlen_q4(d["q"], d["k"], d["v"], d["bt"], d["cl"], d["qsl"], self.scale, out, dims, **kw)
        return out

    def widen(self, d, tokens):
        """The block table with room for contexts of `tokens` (its further entries name
        no page)."""
        import torch
        more = -(-tokens // 16) - d["bt"].shape[1]
        d["bt"] = torch.cat([d["bt"], torch.full((d["bt"].shape[0], more), -1, dtype=torch.int32, device="cuda")], 1)

    def expected(self):
        return q4.attention(self.q, self.k, self.v, self.bt, self.ctx, self.scale, self.qsl)

    def expected_gpu(self):
        """The same, a sequence's rows and keys at once."""
        import torch
        s = self.H_q // self.H_kv
        res = [np.zeros(self.q.shape) for _ in range(3)] + [np.zeros(self.q.shape[:2]) for _ in range(2)]
        for b, C in enumerate(int(c) for c in self.ctx):
            r0, L = (b, 1) if self.qsl is None else (int(self.qsl[b]), self.n_rows[b])
            if L == 0 or C == 0:
                continue
            k, v = (torch.from_numpy(q4.dense(w, p, self.bt, b, C, self.D)).cuda() for w, p in (("k", self.k), ("v", self.v)))
            q = torch.from_numpy(self.q[r0:r0 + L].astype(np.float64)).cuda()
            seen = torch.arange(C, device="cuda")[None, :] <= torch.arange(C - L, C, device="cuda")[:, None]
            for h in range(self.H_q):
                kt, vh = k[h // s].t().contiguous(), v[h // s].contiguous()
                x = (self.scale * torch.matmul(q[:, h].contiguous(), kt)).masked_fill(~seen, -torch.inf)
                w = torch.softmax(x, -1)
                size = (self.scale * torch.matmul(q[:, h].abs().contiguous(), kt.abs())).masked_fill(~seen, 0).amax(-1)
                reach = self.scale * q[:, h].abs().amax(-1) * (seen * kt.abs().sum(0)).amax(-1)
                for to, what in zip(res, (torch.matmul(w, vh), torch.matmul(w, vh.abs()), torch.matmul(seen.double(), vh.abs()), size, reach)):
                    to[r0:r0 + L, h] = what.cpu().numpy()
        return res


def bound(ref, spread, mass, size, reach, keys, dtype, D):
    """How far an output may be from the float64 one.

    The output's rounding, half a step: 2^-8 (bf16) or 2^-24 of it.  A weight is
    off by its score's error: the accumulation, at most (3 D + 2) 2^-24 of sum |q k|
    in whatever order (fp32's queries are three parts, so up to 3 D products), and
    bf16 queries at head_dim 128 as two e4m3 parts, 2^-22 of max |q| sum |k| (half of
    the last step that both parts hold, 2^-15, beside a largest value of 2^7 at
    least); by 2^-22 for the exponential and its argument's rounding (relative to 1 +
    |x|); by its own rounding, 2^-11 (fp16) for bf16 outputs, of small
    ones half of fp16's last step, 2^-25, beside a largest of 2^7 or more: 2^-32 of
    sum |v|; or 2^-24 (three bf16 parts).  Sums over n keys in 32 bits: n 2^-24.  Numerator and denominator carry
    these, hence twice, of sum w |v|.  A normalisation: 2^-22."""
    w = 1.5 * ((3 * D + 2) * 2.0 ** -24 * size + 2.0 ** -22 * reach) + 2.0 ** -22 * (1 + 1.5 * size)
    w = w + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -24) + keys * 2.0 ** -24
    return (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(ref) + (2 * w[..., None] + 2.0 ** -22) * spread + 2.0 ** -32 * mass + 1e-37


def check(out, expected, keys, dtype, what=""):
    """Every output within its bound, and NaN only where the reference is."""
    ref, spread, mass, size, reach = expected
    x = np.asarray(out, np.float64)
    assert np.array_equal(np.isnan(x), np.isnan(ref)), f"{what}: NaN at other places"
    fine = ~np.isnan(ref)
    off = np.abs(x - ref)[fine] / bound(ref, spread, mass, size, reach, keys, dtype, ref.shape[-1])[fine]
    assert off.size == 0 or off.max() <= 1.0, f"{what}: {off.max():.3g} times the bound"
    return 0.0 if off.size == 0 else float(off.max())
