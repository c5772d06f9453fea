"""The measured operators of the paged key-value cache, each through the library's public calls:

  append   amph_paged_append: rotates new queries and keys and writes keys and values into the sequences' pages
  attn     amph_paged_attn: one new token of every sequence attends to its pages, optionally adding up what every row got
  evict    amph_paged_evict: keeps a budget of rows by those weights and the newest ones

Pages hold K and V step-tiled, as the library's other caches do.  The plain forms read and write the same pages.
Sequences' pages lie scattered over the pool; weights and caches are seeded on the device.
"""
import math

import torch

own = False
DEV = "cuda:0"
THETA = 10000.0


def _case(kind, name=None, dtype="bf16", heads=32, kv_heads=8, dim=128, seqs=1, rows=1024, page=64, unequal=False, weights=False, new=1,
          far=0, layers=1, budget=0, recent=0, steady=False):
    c = dict(kind=kind, dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, seqs=seqs, rows=rows, page=page, unequal=unequal,
             weights=weights, new=new, far=far, layers=layers, budget=budget, recent=recent, steady=steady)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest attention: the float32 miniature's heads, two short sequences, an odd length
        _case("attn", "attn_tiny_f32", dtype="f32", heads=4, kv_heads=4, dim=64, seqs=2, rows=101, page=32),
        # plain decoding of one sequence at 7B widths, the context that the benchmark uses, one row more
        _case("attn", "attn_7b", kv_heads=32, rows=1025),
        # a serving batch with shared key heads: 32 sequences between a handful of rows and 4096
        _case("attn", "attn_shared_b32_unequal", seqs=32, rows=4096, unequal=True),
        # the largest: one sequence with a context of 131072 rows
        _case("attn", "attn_long", rows=131072, page=256),
        # 13B widths, four sequences, the weights of every row added up for an eviction
        _case("attn", "attn_13b_b4_weights", heads=40, kv_heads=40, seqs=4, rows=2011, weights=True),
        # eight query heads a key head, eight unequal sequences, weights
        _case("attn", "attn_shared_b8_weights", heads=64, seqs=8, rows=8191, page=128, unequal=True, weights=True),
        # one decoding step's new rows: 16 sequences, far positions
        _case("append", "append_token", seqs=16, rows=700, unequal=True, far=100000),
        # four prompts of up to 1024 rows into their pages, some of them shorter
        _case("append", "append_prompts_7b", kv_heads=32, seqs=4, rows=0, new=1024, unequal=True),
        # float32, an odd chunk behind an odd length
        _case("append", "append_chunk_f32", dtype="f32", heads=4, kv_heads=4, dim=64, seqs=3, rows=77, new=45, page=32),
        # a decoding step that holds a cache to its budget: one row too many everywhere, rows in the order that earlier steps left
        _case("evict", "evict_step_7b", kv_heads=32, seqs=4, rows=1024, layers=2, budget=1024, recent=64, steady=True),
        # long prompts cut to a quarter
        _case("evict", "evict_prompts", seqs=2, rows=8191, layers=2, budget=2048, recent=512, unequal=True),
        # the float32 miniature, an odd budget
        _case("evict", "evict_tiny_f32", dtype="f32", heads=4, kv_heads=4, dim=64, seqs=2, rows=200, page=32, layers=2, budget=101, recent=7),
    ]


SHAPES = [("f32", 4, 4, 64), ("bf16", 4, 4, 128), ("bf16", 32, 32, 128), ("bf16", 32, 8, 128), ("bf16", 40, 40, 128), ("bf16", 64, 8, 128),
          ("bf16", 52, 52, 128), ("bf16", 28, 4, 128), ("bf16", 32, 8, 64), ("bf16", 16, 1, 128), ("f32", 16, 4, 128), ("bf16", 20, 4, 64)]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    dtype, heads, kv_heads, dim = rng.choice(SHAPES)
    kind = rng.choice(["attn", "attn", "attn", "append", "evict"])
    row = 2 * kv_heads * dim * (4 if dtype == "f32" else 2)
    c = dict(dtype=dtype, heads=heads, kv_heads=kv_heads, dim=dim, page=rng.choice([32, 64, 128, 256]))
    if kind == "attn":
        seqs = log(1, 64)
        weights = rng.random() < 0.4
        most = min(65536, int(3e8 / (row * seqs)))
        return _case("attn", seqs=seqs, rows=log(1, max(most, 40)), unequal=rng.random() < 0.5, weights=weights, **c)
    if kind == "append":
        seqs = log(1, 32)
        new = 1 if rng.random() < 0.5 else log(2, min(2048, max(int(5e7 / (row * seqs)), 4)))
        return _case("append", seqs=seqs, rows=log(1, 2000) - 1, new=new, unequal=rng.random() < 0.5, far=rng.choice([0, 0, 100000]), **c)
    seqs, layers = log(1, 8), rng.randint(1, 3)
    rows = log(64, min(8192, max(int(1e8 / (row * seqs * layers)), 100)))
    budget = rng.choice([rows, rng.randint(max(rows // 8, 1), rows)])
    return _case("evict", seqs=seqs, layers=layers, rows=rows, budget=budget, recent=rng.randint(0, budget // 2), unequal=rng.random() < 0.4,
                 steady=rng.random() < 0.5, **c)


# ---- what a program has in hand -----------------------------------------------------------------------------------------

def _lens(c):
    """Rows that every sequence has before the new ones: the longest first, then down to a sixteenth."""
    if not c["unequal"] or c["seqs"] == 1:
        return [c["rows"]] * c["seqs"]
    return [c["rows"] - (15 * c["rows"] // 16) * b // (c["seqs"] - 1) for b in range(c["seqs"])]


def _news(c):
    """New rows of every sequence, of c["new"] at most: an append with unequal sequences has shorter ones, and in long batches an idle one."""
    if c["kind"] == "attn":
        return [0] * c["seqs"]
    if c["kind"] == "evict":
        return [1] * c["seqs"]
    if not c["unequal"] or c["seqs"] == 1:
        return [c["new"]] * c["seqs"]
    return [c["new"] - (c["new"] * b // c["seqs"]) if c["new"] > 1 else int(b != 2) for b in range(c["seqs"])]


def _pages_each(c):
    return (c["rows"] + (c["new"] if c["kind"] != "attn" else 0) + c["page"] - 1) // c["page"]


class _State:
    pass


def prepare(case, seed):
    c, s = case, _State()
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    tdt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    n, H, Hk, D, P, Ly = c["seqs"], c["heads"], c["kv_heads"], c["dim"], c["page"], c["layers"]
    per = _pages_each(c)
    n_pages = n * per + 3
    normal = lambda *shape, std=1.0: (torch.randn(shape, generator=g, device=DEV) * std).to(tdt)  # noqa: E731
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s.case, s.lens, s.news = c, _lens(c), _news(c)
    s.k_pages, s.v_pages = normal(Ly, n_pages, Hk, P, D), normal(Ly, n_pages, Hk, P, D)
    s.table = torch.randperm(n_pages, generator=g, device=DEV)[:n * per].view(n, per).to(torch.int32).contiguous()
    s.kv_len, s.n_valid = i32(s.lens), i32(s.news)
    R = per * P
    s.weights_in = s.weights = s.row_pos = None
    if c["kind"] == "attn":
        s.q = normal(n, H, D, std=2.0)                       # peaked scores, as trained heads have
        s.out = torch.empty(n, H, D, dtype=tdt, device=DEV)
        if c["weights"]:
            s.weights_in = torch.rand(Ly, n, Hk, R, generator=g, device=DEV)
            s.weights = torch.zeros_like(s.weights_in)
    elif c["kind"] == "append":
        # one projection's output: queries, keys and values of a row side by side
        s.qkv = normal(n, c["new"], (H + 2 * Hk) * D)
        s.q_out = torch.zeros(n, c["new"], H, D, dtype=tdt, device=DEV)
        s.pos = (s.kv_len[:, None] + c["far"] + torch.arange(c["new"], device=DEV, dtype=torch.int32)).contiguous()
        s.weights = torch.rand(n, Hk, R, generator=g, device=DEV)
        s.row_pos = torch.zeros(n, Hk, R, dtype=torch.int32, device=DEV)
    else:
        # accumulated weights spread over decades; every ninth row has never been attended to
        w = torch.exp(2.5 * torch.randn(Ly, n, Hk, R, generator=g, device=DEV) - 6.0)
        s.weights_in = torch.where(torch.rand(Ly, n, Hk, R, generator=g, device=DEV) < 0.11, torch.zeros_like(w), w)
        pos = torch.arange(R, device=DEV, dtype=torch.int32).expand(Ly, n, Hk, R)
        if c["steady"]:                                     # rows where earlier evictions put them; the newest is the last
            old = torch.argsort(torch.rand(Ly, n, Hk, R, generator=g, device=DEV), dim=-1).to(torch.int32)
            new = pos - (s.kv_len + s.n_valid - 1)[None, :, None, None]
            pos = torch.where(new >= 0, R + new, old)
        s.row_pos_in = pos.contiguous()
        s.weights, s.row_pos = torch.zeros_like(s.weights_in), torch.zeros_like(s.row_pos_in)
        s.kv_len_out = torch.zeros_like(s.kv_len)
    if own:
        from paper_2406_13170_amd import binding as B
        from paper_2406_13170_amd import device as L
        s.ctx = B.Context(d_model=H * D, n_heads=H, head_dim=D, d_ffn=64, vocab=64, K=1, topk=1, max_tree=1, max_kv=32, batch=1,
                          dtype=L.dtype_code(c["dtype"]), rope_theta=THETA, device=DEV)
        s.kv = L.paged_pool(s.k_pages, s.v_pages, s.table)
        s.workspace = torch.empty(s.ctx.amph_paged_workspace_bytes(s.kv, Ly), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(s):
    c = s.case
    if not own:
        return {"attn": _plain_attn, "append": _plain_append, "evict": _plain_evict}[c["kind"]](s)
    if c["kind"] == "attn":
        s.ctx.amph_paged_attn(s.kv, 0, s.q, c["heads"] * c["dim"], 0, None, s.kv_len, s.out, s.weights_in, s.weights, s.workspace)
        return {"out": s.out} if s.weights is None else {"out": s.out, "weights": s.weights}
    if c["kind"] == "append":
        H, Hk, D, ld = c["heads"], c["kv_heads"], c["dim"], s.qkv.shape[2]
        s.ctx.amph_paged_append(s.kv, 0, c["new"], s.n_valid, s.kv_len, s.pos, s.qkv, ld, s.qkv[:, :, H * D:], ld,
                                s.qkv[:, :, (H + Hk) * D:], ld, s.q_out, s.weights, s.row_pos)
        return {"q": s.q_out, "k": s.k_pages, "v": s.v_pages, "weights": s.weights, "row_pos": s.row_pos}
    s.ctx.amph_paged_evict(s.kv, c["layers"], c["budget"], c["recent"], 1, None, s.kv_len, s.kv_len_out, s.weights_in, s.weights,
                           s.row_pos_in, s.row_pos, s.workspace)
    return {"k": s.k_pages, "v": s.v_pages, "weights": s.weights, "row_pos": s.row_pos, "kv_len": s.kv_len_out}


def _places(c):
    """Where row r, dim d of a page and head lies in its step-tiled keys and values: two index tables [page rows, dims]."""
    e = 4 if c["dtype"] == "f32" else 2
    P, D = 16 // e, c["dim"]
    r, d = torch.arange(c["page"], device=DEV)[:, None], torch.arange(D, device=DEV)[None, :]
    step, kk, piece = r // (4 * P), r % (4 * P), 64 // e
    tile, slot = (kk % P) // 4, (kk // P) * 4 + kk % 4
    k = ((step * (P // 4) + tile) * (D // piece) + d // piece) * 16 * piece + slot * piece + d % piece
    v = (step * (D // 16) + d // 16) * 16 * piece + (d % 16) * piece + kk
    return k, v


def _plain_attn(s):
    c = s.case
    n, H, Hk, D = c["seqs"], c["heads"], c["kv_heads"], c["dim"]
    k_at, v_at = _places(c)
    t = s.table.long()
    gather = lambda pages, at: pages[0].flatten(2)[t].permute(0, 2, 1, 3)[:, :, :, at].flatten(2, 3).float()  # noqa: E731
    q = s.q.float().view(n, Hk, H // Hk, D)
    live = torch.arange(t.shape[1] * c["page"], device=DEV) < s.kv_len[:, None]
    sc = torch.matmul(q, gather(s.k_pages, k_at).transpose(2, 3).contiguous()) / math.sqrt(D)
    sc = torch.where(live[:, None, None], sc, torch.full_like(sc, -math.inf))
    p = torch.exp(sc - sc.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    out = torch.matmul(p, gather(s.v_pages, v_at)).view(n, H, D).to(s.q.dtype)
    if s.weights is None:
        return {"out": out}
    return {"out": out, "weights": torch.where(live[None, :, None], s.weights_in + p.sum(2)[None], s.weights)}


def _plain_append(s):
    c = s.case
    n, H, Hk, D, N = c["seqs"], c["heads"], c["kv_heads"], c["dim"], c["new"]
    k_at, v_at = _places(c)
    b, j = torch.nonzero(torch.arange(N, device=DEV) < s.n_valid[:, None], as_tuple=True)
    x = s.qkv[b, j].float()
    q, k, v = x[:, :H * D].view(-1, H, D), x[:, H * D:(H + Hk) * D].view(-1, Hk, D), x[:, (H + Hk) * D:].view(-1, Hk, D)
    angle = s.pos[b, j].double()[:, None] * THETA ** (-2.0 * torch.arange(D // 2, device=DEV, dtype=torch.float64) / D)
    cs, sn = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turn(y):
        lo, hi = y[..., :D // 2], y[..., D // 2:]
        return torch.cat([lo * cs - hi * sn, hi * cs + lo * sn], -1).to(s.qkv.dtype)

    row = s.kv_len[b].long() + j
    page, at = s.table[b, row // c["page"]].long()[:, None, None], row % c["page"]
    head = torch.arange(Hk, device=DEV)[None, :, None]
    s.k_pages[0].flatten(2)[page, head, k_at[at][:, None]] = turn(k)
    s.v_pages[0].flatten(2)[page, head, v_at[at][:, None]] = v.to(s.qkv.dtype)
    s.q_out[b, j] = turn(q)
    s.weights[b[:, None], head[:, :, 0], row[:, None]] = 0.0
    s.row_pos[b[:, None], head[:, :, 0], row[:, None]] = s.pos[b, j][:, None].expand(-1, Hk)
    return {"q": s.q_out, "k": s.k_pages, "v": s.v_pages, "weights": s.weights, "row_pos": s.row_pos}


def _plain_evict(s):
    c = s.case
    k_at, v_at = _places(c)
    R, most, far = s.weights_in.shape[-1], c["budget"], torch.iinfo(torch.int64).max
    at = torch.arange(R, device=DEV)
    rows = (s.kv_len + s.n_valid).long()[None, :, None, None]
    live = at < rows
    pos = torch.where(live, s.row_pos_in.long(), torch.full_like(s.row_pos_in, -1).long())
    kept = live & (pos > pos.amax(-1, keepdim=True) - c["recent"])
    rank = torch.where(kept, torch.full_like(s.weights_in, math.inf), torch.where(live, s.weights_in, torch.full_like(s.weights_in, -math.inf)))
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(live.expand_as(rank)).scatter(-1, order[..., :most], True) & live
    # ascending: the holes below the budget, and the kept rows behind it
    holes = torch.sort(torch.where(~kept & live & (at < most), at, far), dim=-1).values
    from_ = torch.sort(torch.where(kept & (at >= most), at, far), dim=-1).values
    ly, b, h, i = torch.nonzero((from_ < far), as_tuple=True)
    dst, src = holes[ly, b, h, i], from_[ly, b, h, i]
    page = lambda r: s.table[b, r // c["page"]].long()[:, None]  # noqa: E731
    for pages, places in ((s.k_pages, k_at), (s.v_pages, v_at)):
        flat = pages.flatten(3)
        flat[ly[:, None], page(dst), h[:, None], places[dst % c["page"]]] = flat[ly[:, None], page(src), h[:, None], places[src % c["page"]]]
    stay = live & (at < most)
    for new, old in ((s.weights, s.weights_in), (s.row_pos, s.row_pos_in)):
        torch.where(stay, old, new, out=new)
        new[ly, b, h, dst] = old[ly, b, h, src]
    s.kv_len_out.copy_(torch.minimum(rows.view(-1), torch.tensor(most, device=DEV)))
    return {"k": s.k_pages, "v": s.v_pages, "weights": s.weights, "row_pos": s.row_pos, "kv_len": s.kv_len_out}


# ---- the same from the definitions, in 64 bits ----------------------------------------------------------------------------

def _untile(x, values):
    """Step-tiled rows [..., rows, dims] as they are numbered."""
    P = 64 // x.element_size()
    *lead, R, D = x.shape
    m = len(lead)
    if values:
        y = x.reshape(*lead, R // P, D // 16, 16, P).permute(*range(m), m, m + 3, m + 1, m + 2)
    else:
        y = x.reshape(*lead, R // P, P // 16, D // P, 4, 4, P).permute(*range(m), m, m + 3, m + 1, m + 4, m + 2, m + 5)
    return y.reshape(*lead, R, D)


def _tile(x, values, size):
    P = 64 // size
    *lead, R, D = x.shape
    m = len(lead)
    if values:
        y = x.reshape(*lead, R // P, P, D // 16, 16).permute(*range(m), m, m + 2, m + 3, m + 1)
    else:
        y = x.reshape(*lead, R // P, 4, P // 16, 4, D // P, P).permute(*range(m), m, m + 2, m + 4, m + 1, m + 3, m + 5)
    return y.reshape(*lead, R, D)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    H, Hk, D, P = c["heads"], c["kv_heads"], c["dim"], c["page"]
    if c["kind"] == "attn":
        out, weights = torch.zeros_like(s.q, dtype=torch.float64), None if s.weights is None else s.weights.double()
        for b, L in enumerate(s.lens):
            pages = s.table[b].long()
            for h in range(Hk):
                k = _untile(s.k_pages[0, pages, h], False).flatten(0, 1)[:L].double()
                v = _untile(s.v_pages[0, pages, h], True).flatten(0, 1)[:L].double()
                group = slice(h * (H // Hk), (h + 1) * (H // Hk))
                p = torch.softmax(s.q[b, group].double() @ k.T * D ** -0.5, dim=-1)
                out[b, group] = p @ v
                if weights is not None:
                    weights[0, b, h, :L] = s.weights_in[0, b, h, :L].double() + p.sum(0)
        return {"out": out} if weights is None else {"out": out, "weights": weights}
    k_rows, v_rows = _untile(s.k_pages, False).double(), _untile(s.v_pages, True).double()
    if c["kind"] == "append":
        q = s.q_out.double()
        weights = s.weights.double()
        turns = torch.complex(*(f(s.pos.double()[:, :, None] / THETA ** (torch.arange(0, D, 2, device=DEV).double() / D)) for f in (torch.cos, torch.sin)))
        for b, (L, N) in enumerate(zip(s.lens, s.news)):
            if N == 0:
                continue
            new = s.qkv[b, :N].double().view(N, H + 2 * Hk, D)
            z = torch.complex(new[:, :H + Hk, :D // 2].contiguous(), new[:, :H + Hk, D // 2:].contiguous()) * turns[b, :N, None]
            turned = torch.cat([z.real, z.imag], -1)
            q[b, :N] = turned[:, :H]
            weights[b, :, L:L + N] = 0
            s.row_pos[b, :, L:L + N] = s.pos[b, :N]
            for r0 in range(0, N):
                if r0 and (L + r0) % P:
                    continue
                r1 = min(N, r0 + P - (L + r0) % P)            # rows of one page
                page, at = int(s.table[b, (L + r0) // P]), (L + r0) % P
                k_rows[0, page, :, at:at + r1 - r0] = turned[r0:r1, H:].transpose(0, 1)
                v_rows[0, page, :, at:at + r1 - r0] = new[r0:r1, H + Hk:].transpose(0, 1)
        e = s.k_pages.element_size()
        return {"q": q, "k": _tile(k_rows, False, e), "v": _tile(v_rows, True, e), "weights": weights, "row_pos": s.row_pos}
    weights, row_pos, most = s.weights.double(), s.row_pos, c["budget"]
    w_host, p_host, table = s.weights_in.cpu(), s.row_pos_in.cpu(), s.table.cpu()
    lens = []
    for b, (L, N) in enumerate(zip(s.lens, s.news)):
        R = L + N
        lens.append(min(R, most))
        for ly in range(c["layers"]):
            for h in range(Hk):
                w, p = w_host[ly, b, h, :R].numpy(), p_host[ly, b, h, :R].numpy()
                top, idx = p.max() - c["recent"], list(range(R))
                idx = sorted(idx, key=lambda r: (0 if p[r] > top else 1, 0.0 if p[r] > top else -w[r], r))[:most]  # noqa: B023
                have = set(idx)
                dst = [r for r in range(min(most, R)) if r not in have]
                src = sorted(r for r in idx if r >= most)
                rows = list(range(min(most, R)))
                for a, z in zip(dst, src):
                    rows[a] = z
                rows = torch.tensor(rows)
                weights[ly, b, h, :len(rows)] = s.weights_in[ly, b, h][rows.to(DEV)].double()
                row_pos[ly, b, h, :len(rows)] = s.row_pos_in[ly, b, h][rows.to(DEV)]
                if src:
                    a, z = torch.tensor(dst), torch.tensor(src)
                    for x in (k_rows, v_rows):
                        x[ly, table[b, a // P].long().to(DEV), h, (a % P).to(DEV)] = x[ly, table[b, z // P].long().to(DEV), h, (z % P).to(DEV)]
    e = s.k_pages.element_size()
    return {"k": _tile(k_rows, False, e), "v": _tile(v_rows, True, e), "weights": weights, "row_pos": row_pos,
            "kv_len": torch.tensor(lens, dtype=torch.int32)}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------

def work(case):
    c = case
    e, H, Hk, D = 4 if c["dtype"] == "f32" else 2, c["heads"], c["kv_heads"], c["dim"]
    lens, news = _lens(c), _news(c)
    if c["kind"] == "attn":
        rows = sum(lens)
        return {"bytes": 2 * rows * Hk * D * e + 2 * c["seqs"] * H * D * e + (8 * rows * Hk if c["weights"] else 0), "flops": 4 * rows * H * D}
    if c["kind"] == "append":
        rows = sum(news)
        return {"bytes": rows * ((2 * H + 4 * Hk) * D * e + 8 * Hk + 4), "flops": 3 * rows * (H + Hk) * D}
    total, moved, left = 0, 0, 0
    for L, N in zip(lens, news):
        R = L + N
        total, left = total + R, left + min(R, c["budget"])
        behind = max(R - c["budget"], 0)                      # kept rows among them: the newest, and their share of the others
        safe = min(c["recent"], c["budget"])
        rest = (c["budget"] - safe) / max(R - safe, 1)
        near = min(safe, behind) if not c["steady"] else min(1, behind, safe)
        moved += near + (behind - near) * rest if behind else 0
    heads = c["layers"] * Hk
    return {"bytes": heads * (8 * total + 8 * left + moved * 4 * D * e), "flops": heads * total}
