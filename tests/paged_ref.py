"""The paged cache's operators in 64 bits on the host, from their definitions, and pools of pages to run the library's on."""
from __future__ import annotations

import math
from dataclasses import dataclass, field

import torch

import layout_ref as lr
from paper_2406_13170_amd import binding as B
from paper_2406_13170_amd import device as D

DEV = "cuda:0"
F64 = torch.float64
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}          # of a rounding, relative


def make_ctx(dtype, heads, dim, theta=10000.0):
    return B.Context(d_model=heads * dim, n_heads=heads, head_dim=dim, d_ffn=64, vocab=64, K=1, topk=1, max_tree=1, max_kv=32, batch=1,
                     dtype=D.dtype_code(dtype), rope_theta=theta, device=DEV)


@dataclass
class Pool:
    """Row-major rows of every sequence on the host, and the same in scattered step-tiled pages on the device; NaN where no row is."""
    dtype: str
    n_kv: int
    dim: int
    page: int
    lens: list
    per: int                                    # entries of a table row
    layers: int = 1
    seed: int = 0
    spare: int = 3
    rows_k: list = field(default_factory=list)  # [layer][sequence] -> [n_kv, rows, dim] float32, of the storage type's values

    def __post_init__(self):
        g = torch.Generator().manual_seed(self.seed)
        tdt = D.torch_dtype(self.dtype)
        n, cap = len(self.lens), self.per * self.page
        self.n_pages = n * self.per + self.spare
        self.table = torch.randperm(self.n_pages, generator=g)[:n * self.per].view(n, self.per).to(torch.int32)
        normal = lambda L: torch.randn(self.n_kv, L, self.dim, generator=g).to(tdt)  # noqa: E731
        self.rows_k = [[normal(max(L, 0)) for L in self.lens] for _ in range(self.layers)]
        self.rows_v = [[normal(max(L, 0)) for L in self.lens] for _ in range(self.layers)]
        shape = (self.layers, self.n_pages, self.n_kv, self.page, self.dim)
        k, v = torch.full(shape, math.nan, dtype=tdt), torch.full(shape, math.nan, dtype=tdt)
        for ly in range(self.layers):
            for b, L in enumerate(self.lens):
                for dst, src in ((k, self.rows_k[ly][b]), (v, self.rows_v[ly][b])):
                    whole = torch.full((self.n_kv, cap, self.dim), math.nan, dtype=tdt)
                    whole[:, :max(L, 0)] = src
                    dst[ly, self.table[b].long()] = whole.view(self.n_kv, self.per, self.page, self.dim).transpose(0, 1)
        self.k = lr.keys_to_tiled(k).to(DEV)
        self.v = lr.values_to_tiled(v).to(DEV)
        self.table_d = self.table.to(DEV)
        self.kv = D.paged_pool(self.k, self.v, self.table_d)

    @property
    def cap(self):
        return self.per * self.page

    def rows(self, ly, b):
        """(keys, values) of a sequence as the device has them now, [n_kv, cap, dim] on the host."""
        out = []
        for x, back in ((self.k, lr.tiled_to_keys), (self.v, lr.tiled_to_values)):
            out.append(back(x[ly, self.table[b].long().to(DEV)].cpu()).transpose(0, 1).reshape(self.n_kv, self.cap, self.dim))
        return out


def attn(q, k, v):
    """One sequence: q [heads, dim], k, v [n_kv, L, dim] -> out [heads, dim], weights [n_kv, L], and what errors are bounded by:
    sum_r p |v| [heads, dim], and the largest sum of |q k| of a score, by head."""
    H, (n_kv, L, dim) = q.shape[0], k.shape
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    if L == 0:
        return torch.zeros(H, dim, dtype=F64), torch.zeros(n_kv, 0, dtype=F64), torch.zeros(H, dim, dtype=F64), torch.zeros(H, dtype=F64)
    of = torch.arange(H) // (H // n_kv)
    p = torch.softmax(torch.einsum("hd,hld->hl", q, k[of]) / math.sqrt(dim), -1)
    out, mag = torch.einsum("hl,hld->hd", p, v[of]), torch.einsum("hl,hld->hd", p, v[of].abs())
    reach = torch.einsum("hd,hld->hl", q.abs(), k[of].abs()).amax(-1) / math.sqrt(dim)
    return out, p.view(n_kv, H // n_kv, L).sum(1), mag, reach


def attn_bounds(dtype, out, mag, reach, L, dim):
    """How far an output may be off: its rounding to the storage type; and, relative to sum_r p |v|, what float32 sums and a 16-bit P
    leave.  A score is a sum of dim products with a step of 2^-23 each at most (the matrix core cuts its sums off), relative to the sum of
    the magnitudes, and an exponential errs by its argument's error and two steps; numerator and denominator are sums of L such."""
    score = (dim + 4) * 2.0 ** -23 * reach
    sums = 2 * score + (L + 64) * 2.0 ** -23 + (2.0 ** -16 if dtype == "bf16" else 0.0)
    return HALF_STEP[dtype] * out.abs() + mag * sums[:, None] + 1e-30


def weight_bounds(weights, reach, n_kv, L, dim):
    score = (dim + 4) * 2.0 ** -23 * reach.view(n_kv, -1).amax(1) if L else torch.zeros(n_kv, dtype=F64)
    group = reach.numel() // n_kv
    return weights.abs() * ((2 * score + (L + 64 + group) * 2.0 ** -23)[:, None]) + 1e-30


def turn(x, pos, theta):
    """RoPE of x [..., dim] at positions pos [...]."""
    dim = x.shape[-1]
    x = x.to(F64)
    ang = pos.to(F64)[..., None] * theta ** (-torch.arange(0, dim, 2, dtype=F64) / dim)
    c, s = torch.cos(ang), torch.sin(ang)
    a, b = x[..., :dim // 2], x[..., dim // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def turn_bounds(dtype, x, ref):
    """A rounding to the storage type; the angle, below half a turn, is rounded to float32 (2^-23 of it at most), its sine and cosine err
    by four steps, the two products and their sum by one each."""
    a, b = x[..., :x.shape[-1] // 2].to(F64).abs(), x[..., x.shape[-1] // 2:].to(F64).abs()
    m = torch.cat([a + b, a + b], -1)
    return HALF_STEP[dtype] * ref.abs() + m * (math.pi * 2.0 ** -24 + 7 * 2.0 ** -24)


def evict_rows(w, pos, R, budget, recent):
    """What the rows below the budget hold afterwards: the row that was there, or the one that moved in.  w, pos: lists of one head."""
    if R <= budget:
        return list(range(R))
    top = max(pos[:R]) - recent

    def key(r):
        x = w[r]
        return (0, 0.0, r) if pos[r] > top else (2, 0.0, r) if x != x else (1, -x, r)
    kept = set(sorted(range(R), key=key)[:budget])
    rows, behind = list(range(budget)), sorted(r for r in kept if r >= budget)
    for hole, src in zip((r for r in range(budget) if r not in kept), behind):
        rows[hole] = src
    return rows
