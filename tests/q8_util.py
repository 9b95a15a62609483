"""Batches on an 8-bit cache for the tests."""
import numpy as np

from oracle import q8
from paper_2504_09345_amd import binding as pb
from q4_util import Batch as Q4Batch


class Batch(Q4Batch):
    """Seeded sequences of (context, rows) on a pool whose pages are dealt at random and
    whose unused bytes (the slots past a context, the pages of nobody and their scales)
    hold anything, codes of NaN among them.  (The pages of a context have a scale that
    is one.)"""

    def __init__(self, lens, H_q=8, H_kv=2, D=128, dtype="bf16", seed=0, varlen=True, spare=3, k_size=1.0, v_size=1.0):
        rng = np.random.default_rng(seed)
        self.ctx = np.array([c for c, _ in lens], np.int32)
        self.n_rows = [n for _, n in lens] if varlen else [1] * len(lens)
        self.qsl = np.concatenate([[0], np.cumsum(self.n_rows)]).astype(np.int32) if varlen else None
        self.T, self.H_q, self.H_kv, self.D, self.dtype = sum(self.n_rows), H_q, H_kv, D, dtype
        pages = [-(-int(c) // 16) for c in self.ctx]
        self.num_pages = sum(pages) + spare
        perm = rng.permutation(self.num_pages).astype(np.int32)
        self.bt = np.full((len(lens), max(pages + [1])), perm[-1], np.int32)
        self.k = rng.integers(0, 256, (self.num_pages, H_kv, 16 * D), dtype=np.uint8)
        self.v = rng.integers(0, 256, self.k.shape, dtype=np.uint8)
        self.scales = rng.integers(0, 256, (self.num_pages, H_kv, 2), dtype=np.uint8)
        channels = np.exp(0.6 * rng.standard_normal((H_kv, 1, D))) * k_size
        at = 0
        for b, n in enumerate(pages):
            self.bt[b, :n] = perm[at:at + n]
            at += n
            for p in range(n):
                live = min(16, int(self.ctx[b]) - 16 * p)
                self.put("k", self.bt[b, p], rng.standard_normal((H_kv, 16, D)) * channels * np.exp(0.5 * rng.standard_normal((H_kv, 16, 1))), live)
                self.put("v", self.bt[b, p], rng.standard_normal((H_kv, 16, D)) * v_size * np.exp(0.5 * rng.standard_normal((H_kv, 16, 1))), live)
        self.q = self.round(rng.standard_normal((self.T, H_q, D)))
        self.scale = 1 / np.sqrt(D)

    def put(self, which, page, x, live=16):
        """The first `live` of the tokens x [H_kv][16][D] into a page, with the scale of all."""
        pool, at = self.k if which == "k" else self.v, q8.places(which, self.D)[:live]
        for g in range(self.H_kv):
            e = q8.exponent(x[g])
            pool[page, g, at] = q8.codes(x[g, :live], e)
            self.scales[page, g, 0 if which == "k" else 1] = e + 127

    def upload(self):
        d = super().upload()
        d["scales"] = self.cuda(self.scales)
        return d

    def dims(self, d, rows=None, max_context_len=None, num_q_rows=None, max_q_len=None):
        mcl = max(1, int(self.ctx.max())) if max_context_len is None else max_context_len
        rows = d["q"] if rows is None else rows
        if self.qsl is None:
            return pb.make_dims_q8(rows, d["k"], d["bt"], mcl)
        return pb.make_dims_q8(rows, d["k"], d["bt"], mcl, num_q_rows=self.T if num_q_rows is None else num_q_rows,
                               max_q_len=max(self.n_rows) if max_q_len is None else max_q_len)

    def append(self, d, kn, vn, **kw):
        k, v = (self.cuda(x).to(self.torch_dtype) for x in (kn, vn))
        pb.pa_kv_append_q8(k, v, d["bt"], d["cl"], d["k"], d["v"], d["scales"], self.dims(d, k, **kw), query_start_loc=d["qsl"])

    def read(self, d, out=None, **kw):
        import torch
        out = torch.full((2, self.T, self.H_kv, self.D), -3.0, dtype=self.torch_dtype, device="cuda") if out is None else out
        pb.pa_kv_read_q8(d["k"], d["v"], d["scales"], d["bt"], d["cl"], out[0], out[1], self.dims(d, out[0], **kw), query_start_loc=d["qsl"])
        return out.float().cpu().numpy()

    def attend(self, d, dims=None, out=None, **kw):
        """The call's output, a device tensor (NaN where it wrote nothing)."""
        import torch
        out = torch.full_like(d["q"], float("nan")) if out is None else out
        dims = self.dims(d) if dims is None else dims
        pool = (d["k"], d["v"], d["scales"], d["bt"], d["cl"])
        if self.qsl is None:
            pb.paged_attn_q8(d["q"], *pool, self.scale, out, dims, **kw)
        else:
            pb.paged_attn_varlen_q8(d["q"], *pool, d["qsl"], self.scale, out, dims, **kw)
        return out

    def expected(self):
        """(out, spread, mass, size, reach) as oracle.q4.attention's, a sequence's rows and
        keys at once, in float64 on the GPU.  A NaN of V reaches the rows that see it, in its
        dim; of K, the whole of those rows."""
        import torch
        s = self.H_q // self.H_kv
        res = [np.zeros(self.q.shape) for _ in range(3)] + [np.zeros(self.q.shape[:2]) for _ in range(2)]
        for b, C in enumerate(int(c) for c in self.ctx):
            r0, L = (b, 1) if self.qsl is None else (int(self.qsl[b]), self.n_rows[b])
            if L == 0 or C == 0:
                continue
            k, v = (torch.from_numpy(q8.dense(w, p, self.scales, self.bt, b, C, self.D)).cuda() for w, p in (("k", self.k), ("v", self.v)))
            q = torch.from_numpy(self.q[r0:r0 + L].astype(np.float64)).cuda()
            seen = torch.arange(C, device="cuda")[None, :] <= torch.arange(C - L, C, device="cuda")[:, None]
            for h in range(self.H_q):
                kt, vh = k[h // s].t().contiguous(), v[h // s].contiguous()
                x = (self.scale * torch.matmul(q[:, h].contiguous(), kt)).masked_fill(~seen, -torch.inf)
                w = torch.softmax(x, -1)
                odd = torch.matmul(seen.double(), vh.isnan().double()) > 0
                vh, kt = vh.nan_to_num(0.0), kt.nan_to_num(0.0)
                size = (self.scale * torch.matmul(q[:, h].abs().contiguous(), kt.abs())).masked_fill(~seen, 0).amax(-1)
                reach = self.scale * q[:, h].abs().amax(-1) * (seen * kt.abs().sum(0)).amax(-1)
                out = torch.matmul(w, vh).masked_fill(odd, torch.nan)
                for to, what in zip(res, (out, torch.matmul(w, vh.abs()), torch.matmul(seen.double(), vh.abs()), size, reach)):
                    to[r0:r0 + L, h] = what.cpu().numpy()
        return res

    expected_gpu = expected

    def new_rows(self, seed, odd=False):
        """Rows of widely different sizes, as the call's type holds them."""
        rng = np.random.default_rng(seed)
        x = rng.standard_normal((self.T, self.H_kv, self.D)) * np.exp(2 * rng.standard_normal((self.T, self.H_kv, 1)))
        if odd:
            flat = x.reshape(-1, 32)
            for i, y in enumerate([0.0, -0.0, 1e-38, 2.0 ** -133, np.inf, -np.inf, np.nan]):
                flat[i::37, (5 * i) % 32] = y
            flat[3::41] = 0.0
            flat[4::43] *= 2.0 ** -9
            flat[5::47] = 1.75 * 2.0 ** 5 * np.tanh(rng.standard_normal(flat[5::47].shape))
            flat[5::47, 3] = 1.75 * 2.0 ** 5
        return self.round(x)

    def written(self, kn, vn, keep=None):
        """(k, v, scales) after the append."""
        return q8.append(kn, vn, self.bt, self.ctx, self.k, self.v, self.scales, self.qsl, keep)


def same_bytes(d, expected):
    """The pools and scales on the GPU are the expected bytes, one NaN as good as the other."""
    for name, ref in zip(("k", "v", "scales"), expected):
        got = d[name].cpu().numpy()
        if name != "scales":
            got, ref = (np.where(x & 127 == 127, 127, x) for x in (got, ref))
        if not np.array_equal(got, ref):
            at = np.argwhere(got != ref)
            return f"{name}: {len(at)} bytes differ, the first at {at[0].tolist()}: {got[tuple(at[0])]}, not {ref[tuple(at[0])]}"
    return ""
