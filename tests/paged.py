"""Inputs and bounds shared by the tests of the cache of pages."""
import numpy as np
import torch

import paper_2604_10103_amd as hf

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}   # a rounding, relative


def f64(t):
    return t.detach().double().cpu().numpy()


class Batch:
    """Sequences of the given new tokens and lengths (the new ones included) in shuffled pages; every buffer on the GPU."""

    def __init__(self, new, lens, heads, heads_kv, d, dtype, page, causal=True, window=0, n_sink=0, scale=0.0, seed=0, rows_behind=0,
                 spare_pages=2, gain=1.0, extra_entries=0):
        g = torch.Generator().manual_seed(seed)
        t = TYPES[dtype]
        self.dtype, self.t, self.page, self.d, self.heads, self.heads_kv = dtype, t, page, d, heads, heads_kv
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
        self.lens = np.array(lens, dtype=np.int64)
        self.n = int(self.cu[-1]) + rows_behind
        count = [max(0, -(-int(x) // page)) for x in lens]
        self.n_pages = sum(count) + spare_pages
        width = max(1, max(count)) + extra_entries
        order = torch.randperm(self.n_pages, generator=g).numpy()
        self.table = np.full((len(lens), width), -1, dtype=np.int32)
        at = 0
        for s, k in enumerate(count):
            self.table[s, :k] = order[at:at + k]
            at += k
        make = lambda *shape: torch.randn(shape, generator=g).to(t)  # noqa: E731
        rows = make(self.n, heads + 2 * heads_kv, d)
        rows[:, :heads] *= gain
        self.rows = rows.to(DEV)
        self.Q, self.K, self.V = self.rows[:, :heads], self.rows[:, heads:heads + heads_kv], self.rows[:, heads + heads_kv:]
        self.K_pages, self.V_pages = make(self.n_pages, heads_kv, page, d).to(DEV), make(self.n_pages, heads_kv, page, d).to(DEV)
        self.mask = dict(causal=causal, window=window, n_sink=n_sink)
        self.scale = scale
        self.cache = hf.make_paged(heads, heads_kv, d, dtype, page, self.n_pages, len(lens), width, softmax_scale=scale, **self.mask)
        self.to_gpu()

    def to_gpu(self):
        ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)  # noqa: E731
        self.cu_d, self.lens_d, self.table_d = ints(self.cu), ints(self.lens), ints(self.table)

    def workspace(self):
        n = hf.hf_paged_workspace_bytes(self.cache, self.n)
        return torch.randint(0, 255, (n,), dtype=torch.uint8, device=DEV) if n else None

    def attend(self, lse=True, O=None, workspace=None):
        O = torch.full((self.n, self.heads, self.d), 7.0, dtype=self.t, device=DEV) if O is None else O
        lse2 = torch.full((self.heads, self.n), 7.0, device=DEV) if lse else None
        ws = self.workspace() if workspace is None else workspace
        hf.hf_paged_attn_fwd(self.cache, self.Q, self.cu_d, self.lens_d, self.K_pages, self.V_pages, self.table_d, O, ws, lse2)
        return O, lse2

    def oracle(self):
        import oracle.paged as orc
        return orc.attend(f64(self.Q), f64(self.K_pages), f64(self.V_pages), self.cu, self.lens, self.table, scale=self.scale, **self.mask)

    def check(self, O, lse2, ref=None):
        """Scores of d products summed in fp32 are off by (d + 8) 2^-24 of the sum of their sizes at most (the scale's and the exponent's
        roundings among the eight), which moves every probability by twice that, relatively; n probabilities and n products are summed in
        fp32, in parts that are rescaled (64 more roundings); bf16: a rounding of each probability and of the output."""
        R, L, spread, size, count = self.oracle() if ref is None else ref
        live = ~np.isnan(R[:, 0, 0])
        delta = (self.d + 8) * 2.0 ** -24 * size[..., None]
        sums = (count[:, None, None] + 64) * 2.0 ** -24
        bound = HALF[self.dtype] * np.abs(R) + spread * ((HALF["bf16"] if self.dtype == "bf16" else 0.0) + 2 * delta + 2 * sums)
        got = f64(O)
        assert np.isfinite(got[live]).all()
        far = np.abs(got - R) - bound
        assert (far[live] <= 0).all(), f"off by {np.abs(got - R)[live].max():.3e}, {(far[live] > 0).mean():.3e} of the values beyond the bound"
        assert (got[~live] == 7.0).all()           # rows behind the last sequence
        assert (got[live][count[live] == 0] == 0).all()
        if lse2 is not None:
            got = f64(lse2)
            some = live & (count > 0)
            assert (np.isposinf(got[:, live & (count == 0)])).all() and (got[:, ~live] == 7.0).all()
            L, far = L[:, some], np.abs(got[:, some] - L[:, some])
            bound = 1.5 * (delta[..., 0].T + 2 * sums[..., 0].T)[:, some] + 2.0 ** -22 * np.abs(L)
            assert (far <= bound).all(), far.max()
