"""Inputs and bounds shared by the tests of norms with rotation and of the pages in 8 bits."""
import numpy as np
import torch

import oracle.e4m3 as orc
import paper_2604_10103_amd as hf
from paged import DEV, HALF, TYPES, Batch, f64  # noqa: F401

UNIT = 2.0 ** -24


def codes_of(pages):
    """Random fp32 pages as (codes, scales): every code of the type may appear, no row is the same."""
    scale = (pages.abs().amax(-1) * (1.0 / 448.0)).clamp_min(2.0 ** -126)
    return (pages / scale[..., None]).to(torch.float8_e4m3fn), scale


def values(codes, scales):
    """What pages stand for, fp64."""
    return codes.cpu().float().double().numpy() * f64(scales)[..., None]


class Batch8(Batch):
    """Batch whose pages are codes and scales; K_pages and V_pages of the base class become these."""

    def __init__(self, *args, spread=0.5, **kw):
        super().__init__(*args, **kw)
        g = torch.Generator().manual_seed(kw.get("seed", 0) + 77)
        make = lambda shape: torch.randn(shape, generator=g) * (spread * torch.randn(shape[:-1] + (1,), generator=g)).exp()  # noqa: E731
        shape = tuple(self.K_pages.shape)
        (self.K_pages, self.K_scales), (self.V_pages, self.V_scales) = ([t.to(DEV) for t in codes_of(make(shape))] for _ in range(2))

    def workspace(self):
        n = hf.hf_paged_e4m3_workspace_bytes(self.cache, self.n)
        return torch.randint(0, 255, (n,), dtype=torch.uint8, device=DEV) if n else None

    def attend(self, lse=True, O=None, workspace=None):
        O = torch.full((self.n, self.heads, self.d), 7.0, dtype=self.t, device=DEV) if O is None else O
        lse2 = torch.full((self.heads, self.n), 7.0, device=DEV) if lse else None
        ws = self.workspace() if workspace is None else workspace
        hf.hf_paged_attn_e4m3_fwd(self.cache, self.Q, self.cu_d, self.lens_d, self.K_pages, self.V_pages, self.K_scales, self.V_scales,
                                  self.table_d, O, ws, lse2)
        return O, lse2

    def oracle(self):
        import oracle.paged as paged
        return paged.attend(f64(self.Q), values(self.K_pages, self.K_scales), values(self.V_pages, self.V_scales), self.cu, self.lens,
                            self.table, scale=self.scale, **self.mask)

    def check(self, O, lse2, ref=None):
        """Batch.check's bound, with what is different here: fp32 queries are three bf16, so that a score is a sum of 3 d products (the
        base class counts d of size |q k|, whose parts sum to at most 1.01 of that); two more roundings of a score, by the key's scale,
        and one of a probability, by the value's.  All are within three times the base class's count: d is tripled there."""
        d = self.d
        self.d = 3 * d + 8
        try:
            super().check(O, lse2, ref)
        finally:
            self.d = d


def norm_bound(x, dtype, y, weight=None, eps=None, positions=None, pairs=None, halves=True, amplitude=1.0, **spectrum):
    """How far hf_norm_rope_fwd may be from y.  The sum of squares is one of positive terms, 16 products a thread and four exchanges, the
    mean and eps: 22 roundings; its root's reciprocal half of that and 2 for itself: 13.  Two products: 15 units of a normalised, weighted
    feature.  Turned: cosine and sine are 2.5 units off and rounded once more by the amplitude, two products and a sum: 21 units of the
    pair's two sizes.  Then a rounding to the type."""
    u = orc.norm(x, eps)[0] if eps is not None else np.asarray(x, dtype=np.float64)
    if weight is not None:
        u = u * (weight[:, None] if weight.ndim == 2 else weight)
    return HALF[dtype] * np.abs(y) + 21 * UNIT * pair_sizes(np.abs(u), pairs, halves, amplitude) + 1e-38


def pair_sizes(a, pairs, halves, amplitude):
    """The sum of a pair's two features at both places (others as they are), times the amplitude."""
    out, P = a.copy(), sum(pairs or [])
    for p in range(P):
        u, v = (p, p + P) if halves else (2 * p, 2 * p + 1)
        out[..., u] = out[..., v] = amplitude * (a[..., u] + a[..., v])
    return out


def rope_of(pairs, halves=True, shared=True, theta=10000.0):
    return hf.make_rope_axes(pairs, theta=theta, layout=hf.HF_ROPE_HALVES if halves else hf.HF_ROPE_ADJACENT,
                             spectrum=hf.HF_ROPE_SHARED if shared else hf.HF_ROPE_PER_AXIS)
