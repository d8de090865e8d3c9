"""Plain 64-bit definitions of what gk_append and gk_attention compute, and the random paged caches that their
tests run on.  Torch, one sequence and one head at a time; nothing here is shared with the library."""
from __future__ import annotations

import math
from dataclasses import dataclass, field

import torch

import paper_2609_39358_b200 as gk

F8 = torch.float8_e4m3fn


@dataclass
class Layout:
    """A paged cache: layers x (K, V) x pages, with room between its parts."""
    H: int
    D: int
    T: int
    fp8: bool = False
    scale_kv: int = 2
    head_major: bool = False
    layers: int = 2
    gap: int = 0              # unused bytes behind every page slab (a multiple of 16)
    scale_gap: int = 0        # unused floats behind every page's scales

    def geom(self) -> gk.Geom:
        return gk.Geom(self.layers, self.H, self.D, self.T, gk.GK_FP8_E4M3 if self.fp8 else gk.GK_BF16,
                       self.scale_kv if self.fp8 else 0, gk.GK_FLAG_HEAD_MAJOR if self.head_major else 0)

    @property
    def elem(self):
        return torch.float8_e4m3fn if self.fp8 else torch.bfloat16


class Paged:
    """The cache's bytes, a gk.Cache over them, and views of one layer as [2, pages, T, H, D]."""

    def __init__(self, lay: Layout, pages: int, seed: int, spread: float = 1.0):
        self.lay, self.pages = lay, pages
        g = torch.Generator(device="cuda").manual_seed(seed)
        E = 1 if lay.fp8 else 2
        slab = lay.T * lay.H * lay.D * E
        self.page_stride = slab + lay.gap
        self.kv_stride = self.page_stride * pages + 64
        self.layer_stride = 2 * self.kv_stride + 128
        self.bytes = torch.randint(0, 127, (lay.layers * self.layer_stride,), dtype=torch.uint8, device="cuda", generator=g)
        self.scales, self.s_page, self.s_kv, self.s_layer = None, 0, 0, 0
        if lay.fp8:
            self.s_page = 4 * (lay.H + lay.scale_gap)
            self.s_kv = self.s_page * pages + 8
            self.s_layer = self.s_kv * lay.scale_kv + 16
            self.scales = torch.rand(lay.layers * self.s_layer // 4, device="cuda", generator=g) * 0.02 + 0.002
        for layer in range(lay.layers):
            for kv in range(2):
                x = torch.randn(pages, lay.T, lay.H, lay.D, device="cuda", generator=g) * spread
                if lay.fp8:
                    x = x / self.scale(layer, kv)[:, None, :, None]
                    x = x.clamp(-448, 448)
                self.layer(layer)[kv].copy_(x.to(lay.elem))

    def cache(self) -> gk.Cache:
        return gk.Cache(self.bytes, self.pages, self.layer_stride, self.kv_stride, self.page_stride, self.scales,
                        self.s_layer, self.s_kv, self.s_page)

    def layer(self, layer: int):
        """[K, V], each a view [pages, T, H, D] of the cache's bytes."""
        lay, E = self.lay, 1 if self.lay.fp8 else 2
        el = self.bytes.view(lay.elem)
        tok, head = (lay.D, lay.T * lay.D) if lay.head_major else (lay.H * lay.D, lay.D)
        return [torch.as_strided(el, (self.pages, lay.T, lay.H, lay.D), (self.page_stride // E, tok, head, 1),
                                 (layer * self.layer_stride + kv * self.kv_stride) // E) for kv in range(2)]

    def scale(self, layer: int, kv: int):
        """View [pages, H] of the K or V scales."""
        lay = self.lay
        off = layer * self.s_layer + (self.s_kv if kv and lay.scale_kv == 2 else 0)
        return torch.as_strided(self.scales, (self.pages, lay.H), (self.s_page // 4, 1), off // 4)

    def values(self, layer: int, kv: int):
        """What the layer's K or V stand for, in 64 bits."""
        x = self.layer(layer)[kv].to(torch.float64)
        return x * self.scale(layer, kv).to(torch.float64)[:, None, :, None] if self.lay.fp8 else x


@dataclass
class Seqs:
    kv: list                 # tokens in the cache, with the new ones
    new: list                # new tokens
    table: torch.Tensor = field(default=None)
    pages: int = 0

    @property
    def n(self):
        return sum(self.new)


def make_seqs(lay: Layout, kv, new, seed: int, spare: int = 3, extra_columns: int = 2) -> Seqs:
    """Random page tables; the entries behind a sequence's pages are no page ids."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-k // lay.T) for k in kv]
    pages = sum(need) + spare
    perm = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(kv), max(need + [1]) + extra_columns), -7, dtype=torch.int32)
    at = 0
    for s, p in enumerate(need):
        table[s, :p] = perm[at:at + p]
        at += p
    return Seqs(list(kv), list(new), table.cuda(), pages)


def batch_of(sq: Seqs, status=None, step_form: bool = False) -> gk.Batch:
    kv = torch.tensor(sq.kv, dtype=torch.int32, device="cuda")
    if step_form:
        assert all(q == 1 for q in sq.new)
        return gk.Batch(sq.table, kv, status=status)
    start = torch.tensor([sum(sq.new[:i]) for i in range(len(sq.new) + 1)], dtype=torch.int32, device="cuda")
    return gk.Batch(sq.table, kv, start, sq.n, max(sq.new), status)


def attention64(p: Paged, layer: int, sq: Seqs, q, scale=None, window=0, causal=True):
    """(out, lse, spread) in 64 bits; spread = sum_t w_t |V_t| / sum_t w_t, by which rounded weights are judged.
    Tokens that a row does not attend to are left out of its sums, whatever they hold."""
    lay = p.lay
    Hq = q.shape[1]
    G = Hq // lay.H
    scale = lay.D ** -0.5 if scale is None else scale
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    spread = torch.zeros_like(out)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    K, V = p.values(layer, 0), p.values(layer, 1)
    at = 0
    for s, (t, n) in enumerate(zip(sq.kv, sq.new)):
        ids = sq.table[s, :-(-t // lay.T)].long()
        k = K[ids].reshape(-1, lay.H, lay.D)[:t]
        v = V[ids].reshape(-1, lay.H, lay.D)[:t]
        for h in range(lay.H):
            kh, vh = k[:, h], v[:, h]
            odd = not bool(torch.isfinite(vh).all())
            x = q[at:at + n, h * G:(h + 1) * G].to(torch.float64)
            pos = torch.arange(t - n, t, device="cuda")[:, None]
            u = torch.arange(t, device="cuda")[None]
            seen = torch.ones(n, t, dtype=torch.bool, device="cuda")
            if causal:
                seen &= u <= pos
            if window:
                seen &= u > pos - window
            w = (x @ kh.t()) * scale
            w = torch.where(seen[:, None], w, -math.inf)
            l = torch.logsumexp(w, -1) if t else torch.full(w.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
            some = seen.any(-1)[:, None].expand(l.shape)
            pr = torch.where(some[..., None], torch.exp(w - l[..., None]), 0.0)
            if odd:
                o = torch.stack([torch.stack([(pr[i, a][seen[i]][:, None] * vh[seen[i]]).sum(0) for a in range(G)])
                                 for i in range(n)]) if n else x
            else:
                o = pr @ vh
            out[at:at + n, h * G:(h + 1) * G] = torch.where(some[..., None], o, 0.0)
            spread[at:at + n, h * G:(h + 1) * G] = pr @ torch.nan_to_num(vh, 0, 0, 0).abs()
            lse[at:at + n, h * G:(h + 1) * G] = torch.where(some, l, -math.inf)
        at += n
    return out, lse, spread


def rotate64(x, cos_sin, rows, interleaved):
    """x [n, heads, D], rows [pairs, n]: the table row that turns each pair of each token."""
    R = cos_sin.shape[1]
    pair = torch.arange(R // 2, device=x.device)[:, None]
    c = cos_sin.to(torch.float64)[rows, pair].t()[:, None]
    s = cos_sin.to(torch.float64)[rows, R // 2 + pair].t()[:, None]
    y = x.to(torch.float64).clone()
    a, b = ((slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R)))
    y[..., a] = x.to(torch.float64)[..., a] * c - x.to(torch.float64)[..., b] * s
    y[..., b] = x.to(torch.float64)[..., b] * c + x.to(torch.float64)[..., a] * s
    return y


def e4m3_round64(x):
    """Nearest e4m3 value, ties to even, |x| <= 464 (a NaN or an infinity gives NaN)."""
    _, e = torch.frexp(x)
    q = torch.exp2((e - 4).clamp(min=-9).to(torch.float64))
    r = torch.round(x / q) * q
    return torch.where(torch.isfinite(x), r, math.nan)
