"""A paged store and its oracle side by side: the same steps on both, with the
tokens' keys and values kept on the host."""
import numpy as np

from oracle.paged_oracle import PagedOracle, paged_attend, rotary_apply

THETA = 10000.0


class Pair:
    def __init__(self, seqs, pages, P, heads, D, kv_heads=None, dtype="bf16", layers=1, max_tokens=4096, max_rows=1024,
                 block=1, window=0, sinks=0, grid=(1, 1), seed=0, pairs=None, layout="interleaved"):
        import torch
        from paper_2606_10671_amd.paged import PagedCache
        from paper_2606_10671_amd.rotary import Rotary
        self.torch, self.dtype = torch, dtype
        self.td = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.H, self.Hk, self.D, self.layers = heads, heads if kv_heads is None else kv_heads, D, layers
        self.cache = PagedCache(seqs=seqs, pages=pages, page_tokens=P, heads=heads, kv_heads=self.Hk, head_dim=D,
                                dtype=self.td, layers=layers, max_tokens=max_tokens, max_rows=max_rows,
                                block_tokens=block, window=window, sinks=sinks, grid=grid)
        # What no token was written to is NaN: a kernel that reads it shows it.
        for l in range(layers):
            self.cache.pages(l).fill_(float("nan"))
        self.oracle = PagedOracle(seqs, pages, P, max_tokens, block, window, sinks, grid)
        self.kv = [[[] for _ in range(seqs)] for _ in range(layers)]  # per token: (k, v) fp64 [Hk][D]
        self.rng = np.random.default_rng(seed)
        self.rotary = None if pairs is None else Rotary(D, pairs, THETA, layout)
        self.pairs, self.layout = pairs, layout

    def rand(self, rows, heads):
        x = self.torch.from_numpy(self.rng.standard_normal((rows, heads, self.D)).astype(np.float32)).to(self.td)
        return x.cuda(), x.double().numpy()

    def plan(self, kept, added, rows=None, max_new=None):
        rows = max(0, sum(max(0, a) for a in added)) if rows is None else rows
        max_new = max(list(added) + [0]) if max_new is None else max_new
        dev = [self.torch.tensor(x, dtype=self.torch.int32, device="cuda") for x in (kept, added)]
        self.cache.plan(*dev, rows=rows, max_new=max_new)
        ref = self.oracle.plan(kept, added, rows, max_new)
        self.check_plan(ref, rows)
        self.step = dict(ref, kept=list(kept), added=list(added), rows=rows)
        return ref

    def check_plan(self, ref, rows):
        c = self.cache
        assert c.status.tolist() == ref["status"]
        assert c.q_start.tolist() == ref["q_start"]
        assert c.slots[:rows].tolist() == ref["slots"]
        assert [tuple(p) for p in c.pos[:rows].tolist()] == ref["pos"]
        assert c.held.tolist() == ref["held"]
        assert int(c.free[0]) == ref["free"]
        assert np.array_equal(c.table.cpu().numpy(), self.oracle.table_rows())

    def admitted(self):
        st = self.step
        return [(s, st["q_start"][s], st["kept"][s], st["added"][s]) for s in range(self.oracle.seqs)
                if st["status"][s] == 0]

    def insert(self, layer=0, edit=None, pitch=1):
        """edit(k, v) may change the step's keys and values (host fp32 arrays) before they go in."""
        rows = self.step["rows"]
        k, kn = self.rand(rows, self.Hk)
        v, vn = self.rand(rows, self.Hk)
        if edit is not None:
            edit(kn, vn)
            k, v = (self.torch.from_numpy(x.astype(np.float32)).to(self.td).cuda() for x in (kn, vn))
        if pitch > 1:  # the rows of a joint projection's output
            joint = self.torch.zeros((rows, pitch, self.Hk, self.D), dtype=self.td, device="cuda")
            joint[:, 0], joint[:, 1] = k, v
            k, v = joint[:, 0], joint[:, 1]
        self.cache.insert(k, v, layer, rotary=self.rotary)
        if self.rotary is not None:
            turned = self.rotary.apply(k, self.cache.pos[:rows])  # the same rotation, bit for bit
            kn = turned.double().cpu().numpy()
        for s, at, kept, n in self.admitted():
            del self.kv[layer][s][kept:]
            self.kv[layer][s].extend((kn[at + i], vn[at + i]) for i in range(n))
        self.check_pages(layer)

    def check_pages(self, layer=0):
        """Every held token that has a page lies there, bit for bit."""
        pages = self.cache.pages(layer).double().cpu().numpy()
        P = self.oracle.P
        for s in range(self.oracle.seqs):
            for p, (k, v) in enumerate(self.kv[layer][s][:self.oracle.held[s]]):
                page = self.oracle.table[s].get(p // P)
                if page is not None:
                    assert np.array_equal(pages[page, 0, :, p % P], k, equal_nan=True), (s, p)
                    assert np.array_equal(pages[page, 1, :, p % P], v, equal_nan=True), (s, p)

    def attend(self, layer=0, scale=0.0, lse=True, q_scale=1.0, pitch=1, finite=True):
        """One attention call against the oracle; returns the output."""
        torch, rows = self.torch, self.step["rows"]
        q, qn = self.rand(rows, self.H)
        if q_scale != 1.0:
            q = (q.float() * q_scale).to(self.td)
            qn = q.double().cpu().numpy()
        if pitch > 1:
            joint = torch.zeros((rows, pitch, self.H, self.D), dtype=self.td, device="cuda")
            joint[:, 1] = q
            q = joint[:, 1]
        out = torch.full((rows, self.H, self.D), 7.0, dtype=self.td, device="cuda")
        L = torch.full((self.H, rows), 7.0, device="cuda") if lse else None
        self.cache.attend(q, layer, scale=scale, out=out, lse=L)
        got, got_l = out.double().cpu().numpy(), L.double().cpu().numpy() if lse else None
        last = self.step["q_start"][-1]
        assert (got[last:] == 7.0).all() and (not lse or (got_l[:, last:] == 7.0).all()), "rows behind the last sequence"
        seen = np.zeros(rows, bool)
        for s, at, kept, n in self.admitted():
            seen[at:at + n] = True
            if n == 0:
                continue
            held = self.kv[layer][s]
            keys, vals = np.stack([k for k, _ in held]), np.stack([v for _, v in held])
            self.compare(got[at:at + n], got_l[:, at:at + n] if lse else None, qn[at:at + n], keys, vals,
                         range(kept, kept + n), scale or None, (s,), finite)
        assert (got[:last][~seen[:last]] == 0.0).all(), "rows of sequences that were not admitted"
        if lse:
            assert np.isneginf(got_l[:, :last][:, ~seen[:last]]).all()
        return out, L

    def compare(self, got, got_l, q, keys, vals, positions, scale, where, finite=True):
        """Elementwise, with A the weighted mean of |V| and d the error of a score: D products summed in fp32, each
        sum within 2^-24 of the running size, doubled for the exponential's argument.
        bf16: weights and output are rounded once each (2^-8 of A, 2^-8 of the output).
        fp32: weights carry the scores' error twice (theirs and the sum's) and n + 16 fp32 sums.
        LSE: the scores' error and the sum's."""
        with np.errstate(all="ignore"):
            O, L, A = paged_attend(q, keys, vals, positions, self.oracle, scale)
        sc = 1.0 / np.sqrt(self.D) if scale is None else scale
        size = sc * np.abs(q).max() * np.abs(keys[np.isfinite(keys)]).max() * self.D if keys.size else 0.0
        size = min(size, sc * np.sqrt((q**2).sum(-1).max()) * np.sqrt(np.nan_to_num(keys, nan=0, posinf=0, neginf=0)**2).sum(-1).max()
                   if keys.size else 0.0)
        d = 2 * (self.D + 2) * 2.0**-24 * size
        n = len(keys)
        if self.dtype == "bf16":
            tol = 2.0**-8 * (A + np.abs(O)) + (2 * d + (n + 16) * 2.0**-24) * A
        else:
            tol = (2 * d + (n + 16) * 2.0**-24) * A + 2.0**-24 * np.abs(O)
        if finite:
            assert np.isfinite(got).all(), where
        ok = np.isfinite(O)
        assert np.array_equal(np.isfinite(got), ok), (where, "finite")
        with np.errstate(invalid="ignore"):
            err = np.abs(got - O)
        assert (err[ok] <= tol[ok]).all(), (where, float((err - tol)[ok].max()), float(err[ok].max()))
        assert np.array_equal(np.isnan(got), np.isnan(O)) and (got[np.isinf(O)] == O[np.isinf(O)]).all(), where
        if got_l is not None:
            fin = np.isfinite(L)
            assert (np.abs(got_l - L)[fin] <= (d + (n + 16) * 2.0**-24 + 2.0**-22 * np.abs(L))[fin]).all(), (where, "lse")
            assert np.array_equal(np.isnan(got_l), np.isnan(L)), (where, "lse")
