"""The paged cache's append, attention and eviction against their definitions in 64 bits (paged_ref.py), alone and as a decoding loop uses
them.  Rows that no sequence has hold NaN throughout."""
import ctypes as C
import math

import pytest
import torch

import layout_ref as lr
import paged_ref as pr
import synth_inputs as si
from gpu_common import say
from paged_ref import DEV, F64, Pool
from paper_2406_13170_amd import binding as B
from paper_2406_13170_amd import device as D

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def workspace(ctx, kv, n_layers=0):
    """Exactly as many bytes as the library asks for, NaN in all of them."""
    return torch.full((ctx.amph_paged_workspace_bytes(kv, n_layers),), 0xff, dtype=torch.uint8, device=DEV)


def off_by(x, floats):
    """The same values in a tensor that begins `floats` elements behind an aligned address."""
    buf = torch.empty(x.numel() + floats, dtype=x.dtype, device=DEV)
    buf[floats:] = x.reshape(-1)
    return buf[floats:].view(x.shape)


# ---- attention ------------------------------------------------------------------------------------------------------------

def attn_case(dtype, heads, n_kv, dim, lens, page=32, per=None, weights=None, layers=1, layer=0, ld_extra=0, scale=2.0, seed=0, max_pages=None):
    per = per or max(1, (max(lens) + page - 1) // page)
    pool = Pool(dtype, n_kv, dim, page, lens, per, layers=layers, seed=seed)
    if max_pages:
        pool.kv.max_pages = max_pages
    ctx = pr.make_ctx(dtype, heads, dim)
    g = torch.Generator().manual_seed(seed + 1)
    tdt, n = D.torch_dtype(dtype), len(lens)
    q = (torch.randn(n, heads * dim + ld_extra, generator=g) * scale).to(tdt)
    out = torch.full((n, heads, dim), 7.0, dtype=tdt, device=DEV)
    w_in = torch.rand(n, n_kv, pool.cap, generator=g) if weights == "add" else None
    w_out = torch.full((n, n_kv, pool.cap), -3.0, device=DEV) if weights else None
    w_in_d = w_in.to(DEV) if w_in is not None else None
    ctx.amph_paged_attn(pool.kv, layer, q.to(DEV), heads * dim + ld_extra, 0, None, i32(lens), out, w_in_d, w_out,
                        workspace(ctx, pool.kv, 1 if weights else 0))
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    worst, off, rounding, norm = 0.0, 0.0, 0.0, 0.0
    for b, L in enumerate(lens):
        ref, w, mag, reach = pr.attn(q[b, :heads * dim].view(heads, dim), pool.rows_k[layer][b], pool.rows_v[layer][b])
        err, most = (out[b].cpu().to(F64) - ref).abs(), pr.attn_bounds(dtype, ref, mag, reach, L, dim)
        assert bool((err <= most).all()), (b, L, float((err / most).max()))
        worst = max(worst, float((err / most).max()))
        off, rounding, norm = (x + float(y.square().sum()) for x, y in ((off, err), (rounding, ref.to(tdt).to(F64) - ref), (norm, ref)))
        if weights:
            want = w + (w_in[b, :, :L].to(F64) if w_in is not None else 0.0)
            err, most = (w_out[b, :, :L].cpu().to(F64) - want).abs(), pr.weight_bounds(w, reach, n_kv, L, dim) + 2.0 ** -23 * want.abs()
            assert bool((err <= most).all()), (b, L)
            assert bool((w_out[b, :, L:] == -3.0).all())
    # As a whole it is the output's rounding that counts: P has 16 bits and the sums 24, and their errors have either sign.
    assert math.sqrt(off) <= 1.05 * math.sqrt(rounding) + (2.0 ** -15 if dtype == "bf16" else 2.0 ** -17) * math.sqrt(norm)
    say(f"  {dtype} {heads}/{n_kv} x {dim}, rows {lens[:6]}: {worst:.2f} of the bound, error {math.sqrt(off / max(norm, 1e-300)):.1e}")
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,n_kv,dim", [(4, 4, 64), (4, 4, 128), (8, 2, 128), (7, 1, 128), (16, 1, 64), (17, 1, 128), (33, 1, 64), (12, 4, 64),
                                            (64, 2, 128)])
def test_attention_head_layouts(dtype, heads, n_kv, dim):
    """Groups of 1 to 33 query heads a key head: one and two blocks of queries, one and two query groups, none of them full."""
    if heads * dim % 64:
        pytest.skip("not a model width")
    attn_case(dtype, heads, n_kv, dim, [70, 1, 300], weights="add")
    attn_case(dtype, heads, n_kv, dim, [1500, 3, 0, 47], weights="new", seed=2)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("L", [1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 511, 512, 513, 2047, 2048, 2049, 8200])
def test_attention_lengths(dtype, dim, L):
    attn_case(dtype, 8, 2, dim, [L], page=64, weights="add", seed=L)


@pytest.mark.parametrize("page,per", [(32, 40), (96, 13), (160, 9), (1024, 2)])
def test_attention_pages_of_other_sizes(page, per):
    """Pages that are no power of two, and a table longer than any sequence needs."""
    attn_case("bf16", 8, 8, 128, [1111, 5, 640, 32], page=page, per=per, weights="add")
    attn_case("f32", 4, 2, 64, [1111, 5, 640, 32], page=page, per=per)


def test_attention_of_many_sequences():
    """As many as a call takes, most of them short or empty; 300 in another."""
    lens = [(7 * b) % 13 for b in range(1024)]
    lens[0], lens[500], lens[1023] = 0, 900, 33
    attn_case("bf16", 2, 1, 64, lens, per=29)
    attn_case("f32", 4, 4, 64, [(b * b) % 90 for b in range(300)], weights="add")
    for n in (63, 64, 65, 256, 257):
        attn_case("bf16", 2, 1, 64, [(13 * b) % 40 for b in range(n - 1)] + [700], weights="new", per=22)


def test_attention_of_every_sequence_empty():
    attn_case("bf16", 8, 2, 128, [0, 0, 0], per=1, weights="add")
    attn_case("bf16", 8, 2, 128, [0, 0, 0], per=64, weights="add")


def test_attention_long_and_spread():
    """More key steps a wave than it looks up at once (64), over 512 workgroups and over few."""
    attn_case("bf16", 4, 1, 128, [70000], page=128, weights="add")
    attn_case("bf16", 32, 32, 64, [9000, 8000, 5], page=256)


def test_attention_sharp_and_flat():
    """Scores that one row takes whole, and scores that are all the same."""
    attn_case("bf16", 8, 2, 128, [777], scale=200.0, weights="add")
    attn_case("bf16", 8, 2, 128, [777], scale=0.0, weights="add")
    attn_case("f32", 8, 2, 64, [777], scale=200.0, weights="add")


def test_attention_row_distance_layer_and_bound():
    attn_case("bf16", 8, 2, 128, [300, 41], ld_extra=512, layers=3, layer=2, weights="add")
    attn_case("bf16", 8, 2, 128, [60, 41], per=40, max_pages=2, weights="add")       # a tight bound: one workgroup a walk
    attn_case("bf16", 8, 2, 128, [600, 41], per=40, max_pages=19)


def test_attention_new_rows_count():
    """kv_len and the rows since: n_new, and n_valid where sequences differ (an idle one among them)."""
    pool, ctx = Pool("bf16", 2, 128, 32, [40, 77, 0], 4), pr.make_ctx("bf16", 8, 128)
    q = torch.randn(3, 8, 128, device=DEV, dtype=torch.bfloat16)
    ws = workspace(ctx, pool.kv)

    def run(n_new, n_valid, lens):
        out = torch.zeros(3, 8, 128, device=DEV, dtype=torch.bfloat16)
        ctx.amph_paged_attn(pool.kv, 0, q, 1024, n_new, n_valid, i32(lens), out, workspace=ws)
        return out
    want = run(0, None, [40, 77, 0])
    assert torch.equal(run(3, i32([2, 7, 0]), [38, 74, 0]), want) and torch.equal(run(5, i32([1, 0, -4]), [39, 77, 0]), want)
    two = run(2, None, [38, 75, 0])
    assert torch.equal(two[:2], want[:2])
    torch.cuda.synchronize()
    assert ctx.device_status() == 0                       # (the third sequence then has rows of NaN, which are rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_special_values(dtype):
    """NaN and infinities in a row's key or value reach that sequence's head alone; a score of -inf has no weight; rows all of -inf give
    zeros."""
    lens = [100, 100, 100, 100, 90]
    pool, ctx, tdt = Pool(dtype, 2, 64, 32, lens, 40), pr.make_ctx(dtype, 2, 64), D.torch_dtype(dtype)

    def put(x, back, to, b, h, row, value):
        rows = back(x[0, pool.table[b].long().to(DEV)].cpu())           # [per, n_kv, page, dim]
        rows[row // 32, h, row % 32] = value
        x[0, pool.table[b].long().to(DEV)] = to(rows).to(DEV)
    q = torch.ones(5, 2, 64, device=DEV, dtype=tdt)
    put(pool.k, lr.tiled_to_keys, lr.keys_to_tiled, 0, 0, 7, math.nan)
    put(pool.v, lr.tiled_to_values, lr.values_to_tiled, 1, 1, 99, math.inf)
    put(pool.v, lr.tiled_to_values, lr.values_to_tiled, 4, 0, 0, -math.inf)
    put(pool.k, lr.tiled_to_keys, lr.keys_to_tiled, 2, 0, 50, -math.inf)
    for r in range(100):
        put(pool.k, lr.tiled_to_keys, lr.keys_to_tiled, 3, 1, r, -math.inf)
    out, w = torch.zeros(5, 2, 64, device=DEV, dtype=tdt), torch.zeros(5, 2, pool.cap, device=DEV)
    for most in (pool.per, 4):                             # the keys dealt out, and one workgroup a head
        pool.kv.max_pages = most
        ctx.amph_paged_attn(pool.kv, 0, q, 128, 0, None, i32(lens), out, None, w, workspace(ctx, pool.kv, 1))
        torch.cuda.synchronize()
        assert ctx.device_status() == 0
        assert out[0, 0].isnan().all() and out[0, 1].isfinite().all() and w[0, 0, :100].isnan().all()
        assert bool((out[1, 1] == math.inf).all()) and out[1, 0].isfinite().all()
        assert bool((out[4, 0] == -math.inf).all()) and out[4, 1].isfinite().all()
        keep = [r for r in range(100) if r != 50]
        ref = pr.attn(q[2, :1].cpu(), pool.rows_k[0][2][:1, keep], pool.rows_v[0][2][:1, keep])
        assert bool(((out[2, :1].cpu().to(F64) - ref[0]).abs() <= pr.attn_bounds(dtype, ref[0], ref[2], ref[3], 100, 64)).all())
        assert float(w[2, 0, 50]) == 0.0 and out[2].isfinite().all()
        assert bool((out[3, 1] == 0).all()) and bool((w[3, 1, :100] == 0).all())


def test_attention_bad_lengths_and_pages():
    """Nothing is written for them, the others are served, and the flag says so."""
    lens = [50, 700, 60, 640, 33]
    for cap_pages in (24, 4):                              # several workgroups a walk, and one
        ls = [min(L, cap_pages * 32) for L in lens]
        pool, ctx = Pool("bf16", 2, 128, 32, ls, cap_pages), pr.make_ctx("bf16", 8, 128)
        q = torch.randn(5, 8, 128, device=DEV, dtype=torch.bfloat16)
        good, w_good = torch.zeros(5, 8, 128, device=DEV, dtype=torch.bfloat16), torch.zeros(5, 2, pool.cap, device=DEV)
        ws = workspace(ctx, pool.kv, 1)
        ctx.amph_paged_attn(pool.kv, 0, q, 1024, 0, None, i32(ls), good, None, w_good, ws)
        assert ctx.device_status() == 0
        for lens_now, entry, bits, hit in [([-1, ls[1], cap_pages * 32 + 1, ls[3], ls[4]], None, B.AMPH_DEV_KV_OVERFLOW, {0, 2}),
                                           (ls, (1, 0, -1), B.AMPH_DEV_BAD_PAGE, {1}), (ls, (3, (ls[3] - 1) // 32, pool.n_pages), B.AMPH_DEV_BAD_PAGE, {3}),
                                           (ls, (4, 2, 10 ** 9), 0, set())]:                     # (behind the sequence's last row)
            pool.table_d.copy_(pool.table)
            if entry:
                pool.table_d[entry[0], entry[1]] = entry[2]
            out, w = torch.full_like(good, 7.0), torch.full_like(w_good, -3.0)
            ctx.amph_paged_attn(pool.kv, 0, q, 1024, 0, None, i32(lens_now), out, None, w, ws)
            assert ctx.device_status() == bits
            for b in range(5):
                if b in hit:
                    assert bool((out[b] == 7.0).all()) and bool((w[b] == -3.0).all()), (entry, b)
                else:
                    assert torch.equal(out[b], good[b]) and torch.equal(w[b, :, :ls[b]], w_good[b, :, :ls[b]]), (entry, b)


def test_attention_shared_pages():
    """Two sequences with a prefix in common, and the same page twice in one of them."""
    pool, ctx = Pool("bf16", 4, 64, 32, [96, 96, 64], 3), pr.make_ctx("bf16", 4, 64)
    pool.table[1, :2] = pool.table[0, :2]
    pool.table[2, 1] = pool.table[2, 0]
    pool.table_d.copy_(pool.table)
    q = torch.randn(3, 4, 64).to(torch.bfloat16)
    out = torch.zeros(3, 4, 64, device=DEV, dtype=torch.bfloat16)
    ctx.amph_paged_attn(pool.kv, 0, q.to(DEV), 256, 0, None, i32([96, 96, 64]), out, workspace=workspace(ctx, pool.kv))
    for b in range(3):
        k, v = pool.rows(0, b)
        L = [96, 96, 64][b]
        ref, _, mag, reach = pr.attn(q[b], k[:, :L], v[:, :L])
        assert bool(((out[b].cpu().to(F64) - ref).abs() <= pr.attn_bounds("bf16", ref, mag, reach, L, 64)).all())


def test_attention_adds_in_place_and_twice_the_same():
    pool, ctx = Pool("bf16", 2, 128, 64, [900, 31], 20), pr.make_ctx("bf16", 8, 128)
    q, lens = torch.randn(2, 8, 128, device=DEV, dtype=torch.bfloat16), i32([900, 31])
    w, ws = torch.rand(2, 2, pool.cap, device=DEV), workspace(ctx, pool.kv, 1)
    outs = [torch.zeros(2, 8, 128, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
    apart = torch.zeros_like(w)
    ctx.amph_paged_attn(pool.kv, 0, q, 1024, 0, None, lens, outs[0], w, apart, ws)
    ctx.amph_paged_attn(pool.kv, 0, q, 1024, 0, None, lens, outs[1], w, w, ws)
    assert torch.equal(*outs) and torch.equal(w[0, :, :900], apart[0, :, :900]) and torch.equal(w[1, :, :31], apart[1, :, :31])


def test_attention_beyond_32_bits():
    """Pages beyond 4 GiB of a pool, as bytes and as elements."""
    page, dim = 64, 128
    n_pages = (9 << 30) // (page * dim * 2) // 2 * 2
    k, v = (torch.empty(1, n_pages, 1, page, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ids = [n_pages - 1, 0, n_pages // 2 + 1, n_pages // 4 + 1]
    rows = [torch.randn(4, page, dim, dtype=torch.bfloat16) for _ in range(2)]
    for i, p in enumerate(ids):
        k[0, p, 0] = lr.keys_to_tiled(rows[0][i]).to(DEV)
        v[0, p, 0] = lr.values_to_tiled(rows[1][i]).to(DEV)
    table = i32([ids])
    kv, ctx = D.paged_pool(k, v, table), pr.make_ctx("bf16", 2, dim)
    q = torch.randn(1, 2, dim).to(torch.bfloat16)
    out = torch.zeros(1, 2, dim, device=DEV, dtype=torch.bfloat16)
    ctx.amph_paged_attn(kv, 0, q.to(DEV), 2 * dim, 0, None, i32([250]), out, workspace=workspace(ctx, kv))
    ref, _, mag, reach = pr.attn(q[0], *(r.reshape(1, 4 * page, dim)[:, :250] for r in rows))
    assert bool(((out[0].cpu().to(F64) - ref).abs() <= pr.attn_bounds("bf16", ref, mag, reach, 250, dim)).all())
    # an appended row, and an evicted one, out there
    w, pos = torch.zeros(1, 1, 4 * page, device=DEV), torch.arange(4 * page, device=DEV, dtype=torch.int32).view(1, 1, -1).contiguous()
    w[0, 0, 3] = -1.0
    new = torch.randn(1, 1, dim).to(torch.bfloat16)
    ctx.amph_paged_append(kv, 0, 1, None, i32([250]), i32([[0]]), None, 0, new.to(DEV), dim, new.to(DEV), dim, None, w, pos)
    n = i32([0])
    ctx.amph_paged_evict(kv, 1, 250, 1, 1, None, i32([250]), n, w, w, pos, pos, workspace(ctx, kv, 1))
    assert int(n) == 250 and ctx.device_status() == 0
    assert torch.equal(lr.tiled_to_keys(k[0, ids[0], 0].cpu())[3], new[0, 0]) and torch.equal(lr.tiled_to_values(v[0, ids[0], 0].cpu())[3], new[0, 0])


def test_attention_over_the_most_rows():
    """2^24 rows: keys that are all the same, so that the output is the values' mean and every row has the same weight."""
    L, page, dim = 1 << 24, 1 << 14, 64
    g = torch.Generator(device=DEV).manual_seed(1)
    k = torch.zeros(1, L // page, 1, page, dim, dtype=torch.bfloat16, device=DEV)
    v = torch.randn(k.shape, dtype=torch.bfloat16, device=DEV, generator=g) + 1.0
    table = torch.randperm(L // page, device=DEV, generator=g).to(torch.int32).view(1, -1).contiguous()
    kv, ctx = D.paged_pool(k, v, table), pr.make_ctx("bf16", 2, dim)
    out, w = torch.zeros(1, 2, dim, device=DEV, dtype=torch.bfloat16), torch.zeros(1, 1, L, device=DEV)
    q = torch.randn(1, 2, dim, device=DEV, dtype=torch.bfloat16)
    ctx.amph_paged_attn(kv, 0, q, 2 * dim, 1, None, i32([L - 1]), out, None, w, workspace(ctx, kv, 1))
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    mean = v.view(-1, dim // 16, 16, 32).double().mean((0, 3)).view(dim).cpu()          # [step, block of dims, dim, row of the step]
    mag = v.view(-1, dim // 16, 16, 32).float().abs().mean((0, 3)).view(dim).double().cpu()
    # 512 pieces of four waves, 256 key steps each, one sum after the other: (256 + 4 + 512) sums with a step of 2^-23 each
    assert bool(((out[0].cpu().double() - mean).abs() <= 2.0 ** -8 * mean.abs() + mag * (2.0 ** -16 + 800 * 2.0 ** -22)).all())
    assert bool(((w * (L / 2) - 1).abs() <= 800 * 2.0 ** -22).all())


@pytest.mark.parametrize("cfg,L", [(si.MINI, 77), (si.MINI, 700), (si.TINY, 130)])
def test_attention_over_the_step_s_caches(cfg, L):
    """The caches of the verification attention read as pages: a tree that is a root only, and the same token as plain decoding."""
    d_h, n_h, bsz, max_kv = cfg.head_dim, cfg.n_heads, 2, 768
    ctx = B.Context(d_model=n_h * d_h, n_heads=n_h, head_dim=d_h, d_ffn=64, vocab=64, K=4, topk=4, max_tree=1, max_kv=max_kv, batch=bsz,
                    dtype=D.dtype_code(cfg.dtype), device=DEV)
    tdt = D.torch_dtype(cfg.dtype)
    k, v = (torch.randn(2, bsz, n_h, max_kv, d_h).to(tdt) for _ in range(2))
    kc, vc = lr.keys_to_tiled(k).to(DEV), lr.values_to_tiled(v).to(DEV)
    q, lens = torch.randn(bsz, 1, n_h, d_h).to(tdt), [L, L // 3]
    a, b = torch.zeros(bsz, 1, n_h, d_h, dtype=tdt, device=DEV), torch.zeros(bsz, 1, n_h, d_h, dtype=tdt, device=DEV)
    ctx.amph_verify_attn(B.Tree([], 4), q.to(DEV), kc[1], vc[1], i32(lens), a)
    for page in (32, 128, 768):
        kv, table = D.paged_caches(kc, vc, page)
        ctx.amph_paged_attn(kv, 1, q.to(DEV), n_h * d_h, 1, None, i32(lens), b, workspace=workspace(ctx, kv))
        for i, n in enumerate(lens):
            ref, _, mag, reach = pr.attn(q[i, 0], k[1, i, :, :n + 1], v[1, i, :, :n + 1])
            most = pr.attn_bounds(cfg.dtype, ref, mag, reach, n, d_h)
            assert bool(((b[i, 0].cpu().to(F64) - ref).abs() <= most).all())
            extra = mag * 2.0 ** -8 if cfg.dtype == "bf16" else 0.0    # that attention's P has bf16's 8 bits
            assert bool(((a[i, 0].cpu().to(F64) - b[i, 0].cpu().to(F64)).abs() <= 2 * most + extra).all())
    assert ctx.device_status() == 0


# ---- append ---------------------------------------------------------------------------------------------------------------

def append_case(dtype, heads, n_kv, dim, lens, n_new, valid=None, page=32, far=0, fused=True, with_q=True, theta=10000.0, layers=1, layer=0, seed=0):
    news = [min(max(x, 0), n_new) for x in valid] if valid else [n_new] * len(lens)
    per = max(1, max((L + n + page - 1) // page for L, n in zip(lens, news)))
    pool, ctx, n = Pool(dtype, n_kv, dim, page, lens, per, layers=layers, seed=seed), pr.make_ctx(dtype, heads, dim, theta), len(lens)
    g, tdt = torch.Generator().manual_seed(seed + 1), D.torch_dtype(dtype)
    H, W = heads * dim, n_kv * dim
    if fused:
        qkv = torch.randn(n, n_new, H + 2 * W, generator=g).to(tdt)
        q, k, v = qkv[..., :H], qkv[..., H:H + W], qkv[..., H + W:]
        d = qkv.to(DEV)
        args = (d, H + 2 * W, d[..., H:], H + 2 * W, d[..., H + W:], H + 2 * W)
    else:
        q, k, v = (torch.randn(n, n_new, m, generator=g).to(tdt) for m in (H, W, W))
        args = (q.to(DEV), H, k.to(DEV), W, v.to(DEV), W)
    if not with_q:
        args = (None, 0) + args[2:]
    pos = (torch.tensor(lens)[:, None] + far + torch.arange(n_new)).to(torch.int32) if far else None
    q_out = torch.full((n, n_new, heads, dim), 7.0, dtype=tdt, device=DEV) if with_q else None
    w, rp = torch.full((n, n_kv, pool.cap), -3.0, device=DEV), torch.full((n, n_kv, pool.cap), -5, dtype=torch.int32, device=DEV)
    before = [pool.rows(ly, b) for ly in range(layers) for b in range(n)]
    rest = pool.k.clone(), pool.v.clone()
    ctx.amph_paged_append(pool.kv, layer, n_new, i32(valid) if valid else None, i32(lens), pos.to(DEV) if far else None, *args, q_out, w, rp)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    worst = 0.0
    touched = torch.zeros(layers, pool.n_pages, dtype=torch.bool)
    for b, (L, m) in enumerate(zip(lens, news)):
        p = (pos[b] if far else L + torch.arange(n_new))[:m]
        touched[layer, pool.table[b].long()] = True
        for ly in range(layers):
            now, was = pool.rows(ly, b), before[ly * n + b]
            fresh = slice(L, L + m) if ly == layer else slice(0, 0)
            keep = torch.ones(pool.cap, dtype=torch.bool)
            keep[fresh] = False
            for x, y in zip(now, was):
                assert torch.equal(torch.nan_to_num(x[:, keep].float(), 9e9), torch.nan_to_num(y[:, keep].float(), 9e9)), (b, ly)
            if ly != layer:
                continue
            assert torch.equal(now[1][:, fresh].transpose(0, 1), v[b, :m].view(m, n_kv, dim))
            for got, src in ((now[0][:, fresh].transpose(0, 1), k[b, :m].view(m, n_kv, dim)),
                             (q_out[b, :m].cpu() if with_q else None, q[b, :m].view(m, heads, dim))):
                if got is None:
                    continue
                ref = pr.turn(src, p[:, None], theta)
                err, most = (got.to(F64) - ref).abs(), pr.turn_bounds(dtype, src, ref)
                assert bool((err <= most).all()), (b, float((err / most).max()))
                worst = max(worst, float((err / most).max()) if m else 0.0)
        assert bool((w[b, :, L:L + m] == 0).all()) and bool((rp[b, :, L:L + m].cpu() == p.to(torch.int32)).all())
        for x, mark in ((w, -3.0), (rp, -5)):
            assert bool((x[b, :, :L] == mark).all()) and bool((x[b, :, L + m:] == mark).all())
        if with_q:
            assert bool((q_out[b, m:] == 7.0).all())
    for x, y in zip((pool.k, pool.v), rest):
        assert torch.equal(torch.nan_to_num(x[~touched.to(DEV)].float(), 9e9), torch.nan_to_num(y[~touched.to(DEV)].float(), 9e9))
    say(f"  {dtype} {heads}/{n_kv} x {dim}, {n_new} new rows behind {lens[:5]}: {worst:.2f} of the bound")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,n_kv,dim", [(4, 4, 64), (4, 4, 128), (8, 2, 128), (7, 1, 64), (40, 40, 128), (33, 1, 64)])
def test_append_one_row(dtype, heads, n_kv, dim):
    append_case(dtype, heads, n_kv, dim, [0, 31, 32, 500], 1)
    append_case(dtype, heads, n_kv, dim, [9, 16, 15, 63], 1, valid=[1, 0, 1, -2], far=70000, fused=False)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("L,n_new", [(0, 2), (0, 32), (0, 33), (31, 2), (31, 33), (31, 34), (15, 18), (1, 64), (17, 100), (63, 257)])
def test_append_rows(dtype, dim, L, n_new):
    """Whole key steps, parts of them at either end, both."""
    append_case(dtype, 6, 2, dim, [L, 0, L + 3], n_new, valid=[n_new, n_new - 1, n_new + 9], page=64, far=1000 if n_new % 2 else 0, seed=n_new)


def test_append_positions_and_bases():
    append_case("f32", 4, 4, 128, [5, 40], 3, far=2 ** 24 - 100)
    append_case("f32", 4, 4, 64, [5, 40], 3, far=2 ** 30, theta=500000.0)
    append_case("bf16", 4, 2, 128, [5, 40], 40, far=999999, theta=1e6)


def test_append_without_queries_and_in_layers():
    append_case("bf16", 8, 2, 128, [33, 90], 40, with_q=False, layers=3, layer=1)
    append_case("bf16", 8, 2, 128, [33, 90], 1, with_q=False, layers=3, layer=2, fused=False)


def test_append_queries_in_place():
    pool, ctx = Pool("bf16", 2, 128, 32, [5, 40], 3), pr.make_ctx("bf16", 8, 128)
    q, kv = torch.randn(2, 9, 8, 128, device=DEV).to(torch.bfloat16), torch.randn(2, 9, 2, 128, device=DEV).to(torch.bfloat16)
    apart = torch.zeros_like(q)
    args = (i32([5, 40]), None, q, 1024, kv, 256, kv, 256)
    ctx.amph_paged_append(pool.kv, 0, 9, None, *args, apart)
    ctx.amph_paged_append(pool.kv, 0, 9, None, *args, q)
    assert torch.equal(q, apart)


def test_append_bad_lengths_and_pages():
    lens = [30, 96, -1, 64, 97]
    pool, ctx = Pool("bf16", 2, 64, 32, [30, 96, 0, 64, 96], 3), pr.make_ctx("bf16", 4, 64)
    pool.table_d[0, 1] = pool.n_pages                       # sequence 0's rows 32.. : its rows 30 and 31 are written
    kv, q = torch.randn(5, 4, 2, 64).to(torch.bfloat16), torch.randn(5, 4, 4, 64, device=DEV).to(torch.bfloat16)
    q_out, d = torch.full_like(q, 7.0), kv.to(DEV)
    before = [pool.rows(0, b) for b in range(5)]
    ctx.amph_paged_append(pool.kv, 0, 4, None, i32(lens), None, q, 256, d, 128, d, 128, q_out)
    assert ctx.device_status() == B.AMPH_DEV_KV_OVERFLOW | B.AMPH_DEV_BAD_PAGE
    for b in range(5):
        fresh = [30, 31] if b == 0 else [64, 65, 66, 67] if b == 3 else []
        _, v = pool.rows(0, b)
        keep = [r for r in range(96) if r not in fresh]
        assert torch.equal(torch.nan_to_num(v[:, keep].float(), 9e9), torch.nan_to_num(before[b][1][:, keep].float(), 9e9))
        assert torch.equal(v[:, fresh].transpose(0, 1), kv[b, :len(fresh)])
        assert bool((q_out[b, len(fresh):] == 7.0).all()) and not bool((q_out[b, :len(fresh)] == 7.0).any(-1).any())


# ---- eviction -------------------------------------------------------------------------------------------------------------

def evict_case(dtype, n_kv, dim, lens, budget, recent, page=32, layers=2, new=1, valid=None, weights="spread", positions="rows", in_place=False,
               seed=0, per=None, shift=0):
    """lens: rows before the new ones."""
    news = [min(max(x, 0), new) for x in valid] if valid else [new] * len(lens)
    rows = [L + m for L, m in zip(lens, news)]
    per = per or max(1, (max(rows) + page - 1) // page)
    pool, ctx, n = Pool(dtype, n_kv, dim, page, rows, per, layers=layers, seed=seed), pr.make_ctx(dtype, n_kv, dim), len(lens)
    g = torch.Generator().manual_seed(seed + 1)
    shape = (layers, n, n_kv, pool.cap)
    w = {"spread": lambda: torch.exp(3 * torch.randn(shape, generator=g)), "ties": lambda: torch.randint(0, 3, shape, generator=g).float(),
         "same": lambda: torch.full(shape, 0.25), "close": lambda: 1.0 + torch.randint(0, 9, shape, generator=g) * 2.0 ** -23,
         "wild": lambda: torch.tensor([0.0, -0.0, 1e-42, -1.5, math.inf, -math.inf, math.nan, 3e38])[torch.randint(0, 8, shape, generator=g)]}[weights]()
    pos = torch.arange(pool.cap, dtype=torch.int32).expand(shape).contiguous()
    if positions == "mixed":
        pos = (torch.argsort(torch.rand(shape, generator=g), -1) * 3 - 50).to(torch.int32)
    elif positions == "extreme":
        pos = torch.where(torch.rand(shape, generator=g) < 0.5, -2 ** 31, 2 ** 31 - 1).to(torch.int32)
    w_in, p_in = off_by(w.to(DEV), shift), off_by(pos.to(DEV), shift)
    w_out, p_out = (w_in, p_in) if in_place else (off_by(torch.full_like(w_in, -3.0), shift), off_by(torch.full_like(p_in, -5), shift))
    kv_len = i32(lens)
    len_out = kv_len if in_place else i32([-7] * n)
    before = [[pool.rows(ly, b) for b in range(n)] for ly in range(layers)]
    ctx.amph_paged_evict(pool.kv, layers, budget, recent, new, i32(valid) if valid else None, kv_len, len_out, w_in, w_out, p_in, p_out,
                         workspace(ctx, pool.kv, layers))
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    assert len_out.tolist() == [min(R, budget) for R in rows]
    w_now, p_now = w_out.cpu(), p_out.cpu()
    bits = lambda t: t.view(torch.int16 if t.element_size() == 2 else torch.int32)  # noqa: E731
    for ly in range(layers):
        for b, R in enumerate(rows):
            k_now, v_now = pool.rows(ly, b)
            for h in range(n_kv):
                at = pr.evict_rows(w[ly, b, h].tolist(), pos[ly, b, h].tolist(), R, budget, recent)
                m, where = len(at), torch.tensor(at, dtype=torch.long)
                assert torch.equal(bits(w_now[ly, b, h, :m]), bits(w[ly, b, h, where])), (ly, b, h, R)
                assert torch.equal(p_now[ly, b, h, :m], pos[ly, b, h, where])
                tail = (w[ly, b, h, m:], pos[ly, b, h, m:]) if in_place else (torch.full((pool.cap - m,), -3.0), torch.full((pool.cap - m,), -5))
                assert torch.equal(bits(w_now[ly, b, h, m:]), bits(tail[0])) and torch.equal(p_now[ly, b, h, m:], tail[1].to(torch.int32))
                for now, was in ((k_now, before[ly][b][0]), (v_now, before[ly][b][1])):
                    assert torch.equal(bits(now[h, :m]), bits(was[h, where])) and torch.equal(bits(now[h, m:]), bits(was[h, m:]))
    return pool


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("lens,budget,recent", [([100, 99, 101, 0], 100, 7), ([64, 300, 1], 33, 0), ([200, 200], 1, 1), ([200, 31], 199, 199),
                                                ([511, 640], 320, 64)])
def test_evict(dtype, dim, lens, budget, recent):
    evict_case(dtype, 3, dim, lens, budget, recent)
    evict_case(dtype, 2, dim, lens, budget, recent, positions="mixed", in_place=True, seed=1)


@pytest.mark.parametrize("weights", ["ties", "same", "close", "wild"])
@pytest.mark.parametrize("positions", ["rows", "mixed", "extreme"])
def test_evict_equal_and_special_weights(weights, positions):
    evict_case("bf16", 2, 64, [700, 260], 257, 40, weights=weights, positions=positions, seed=3)
    evict_case("f32", 2, 64, [130, 64], 100, 100, weights=weights, positions=positions, in_place=True)
    evict_case("bf16", 2, 64, [256, 255], 256, 9, weights=weights, positions=positions, in_place=True)
    evict_case("bf16", 2, 128, [700], 700, 0, weights=weights, positions=positions, seed=5)


def test_evict_long():
    evict_case("bf16", 1, 64, [20011], 5000, 1000, layers=1, page=256)
    evict_case("bf16", 1, 64, [9000, 40], 8999, 1, layers=1, page=128, weights="ties")
    evict_case("f32", 1, 64, [17000, 300], 400, 0, layers=1, page=256, in_place=True, weights="ties")
    evict_case("bf16", 1, 64, [16999], 16999, 3, layers=1, page=1024, in_place=True)
    evict_case("bf16", 1, 64, [66000, 100], 20000, 500, layers=1, page=1024, in_place=True)
    evict_case("bf16", 1, 64, [66000], 65990, 0, layers=1, page=1024, weights="ties")
    evict_case("f32", 1, 64, [40000, 30000], 30000, 1, layers=1, page=1024, weights="wild", in_place=True)
    evict_case("bf16", 1, 128, [32767, 9000], 16000, 7000, layers=1, page=1024, weights="ties", positions="mixed", in_place=True)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("L,budget,per", [(700, 333, 11), (1999, 1000, None), (1999, 700, 100), (5000, 1111, None), (12000, 2900, None)])
def test_evict_many_moves(dtype, dim, L, budget, per):
    """More than the choosing workgroup moves itself: by key steps below the budget, the last of them cut by it; one sequence drops a single
    row, one none."""
    evict_case(dtype, 1, dim, [L, budget, budget // 2], budget, budget // 3, page=64, per=per, layers=1, in_place=True)
    evict_case(dtype, 2, dim, [L], budget, 0, page=64, per=per, layers=1, weights="ties", positions="mixed")


def test_evict_new_rows_and_tables():
    """Several new rows, sequences that have none, a table with room, no row to drop at all."""
    evict_case("bf16", 2, 128, [90, 100, 3], 100, 5, new=20, valid=[20, 0, -1], per=9)
    evict_case("bf16", 2, 128, [90, 100, 3], 200, 5, new=20, valid=[25, 7, 1])
    evict_case("bf16", 2, 128, [90, 100, 3], 90, 0, new=0)


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_weights_and_positions_anywhere(shift):
    """Weights and positions begin on any element, as the header allows."""
    evict_case("bf16", 3, 64, [300, 200, 20], 128, 7, shift=shift, page=64)
    evict_case("f32", 3, 64, [3000, 128], 128, 7, shift=shift, page=64, layers=1, in_place=True)
    pool, ctx = Pool("bf16", 2, 64, 32, [70, 200], 7), pr.make_ctx("bf16", 4, 64)
    q, out = torch.randn(2, 4, 64, device=DEV).to(torch.bfloat16), torch.zeros(2, 4, 64, device=DEV, dtype=torch.bfloat16)
    a, b = off_by(torch.rand(2, 2, pool.cap, device=DEV), shift), torch.zeros(2, 2, pool.cap, device=DEV)
    ctx.amph_paged_attn(pool.kv, 0, q, 256, 0, None, i32([70, 200]), out, a, b, workspace(ctx, pool.kv, 1))
    ctx.amph_paged_attn(pool.kv, 0, q, 256, 0, None, i32([70, 200]), out, a, a, workspace(ctx, pool.kv, 1))
    assert torch.equal(a[0, :, :70], b[0, :, :70]) and torch.equal(a[1, :, :200], b[1, :, :200])


def test_evict_bad_lengths_and_pages():
    pool, ctx = Pool("bf16", 2, 64, 32, [96, 96, 96, 60], 3, layers=2), pr.make_ctx("bf16", 2, 64)
    pool.table_d[2, 1] = -1
    w, pos = torch.rand(2, 4, 2, 96, device=DEV), torch.arange(96, dtype=torch.int32, device=DEV).expand(2, 4, 2, 96).contiguous()
    w_out, p_out, n = torch.full_like(w, -3.0), torch.full_like(pos, -5), i32([0] * 4)
    k, v = pool.k.clone(), pool.v.clone()
    ctx.amph_paged_evict(pool.kv, 2, 50, 3, 1, None, i32([-4, 96, 80, 49]), n, w, w_out, pos, p_out, workspace(ctx, pool.kv, 2))
    assert ctx.device_status() == B.AMPH_DEV_KV_OVERFLOW | B.AMPH_DEV_BAD_PAGE
    assert n.tolist() == [-4, 96, 80, 50]
    assert bool((w_out[:, :3] == -3.0).all()) and bool((p_out[:, :3] == -5).all()) and torch.equal(w_out[:, 3, :, :50], w[:, 3, :, :50])
    assert torch.equal(pool.k.view(torch.int16), k.view(torch.int16)) and torch.equal(pool.v.view(torch.int16), v.view(torch.int16))


# ---- together ---------------------------------------------------------------------------------------------------------------

def decode(dtype, heads, n_kv, dim, prompts, budget, recent, steps, layers, per, graph=False, page=32):
    """A decoding loop: prompts, then a token a step in every layer, the cache held to a budget.  The reference follows row by row, by position;
    it takes the device's weights for the choice, once they have been found right."""
    ctx, n, theta = pr.make_ctx(dtype, heads, dim), len(prompts), 10000.0
    pool = Pool(dtype, n_kv, dim, page, [0] * n, per, layers=layers)
    g, tdt, H, W = torch.Generator().manual_seed(7), D.torch_dtype(dtype), heads * dim, n_kv * dim
    w, rp = torch.full((layers, n, n_kv, pool.cap), -3.0, device=DEV), torch.full((layers, n, n_kv, pool.cap), -5, dtype=torch.int32, device=DEV)
    kv_len, pos, valid = i32([0] * n), torch.zeros(n, 1, dtype=torch.int32, device=DEV), i32([1] * n)
    ws = workspace(ctx, pool.kv, layers)
    longest = max(prompts)
    first = torch.randn(layers, n, longest, H + 2 * W, generator=g).to(tdt)
    d = first.to(DEV)
    for ly in range(layers):
        ctx.amph_paged_append(pool.kv, ly, longest, i32(prompts), kv_len, None, None, 0, d[ly, ..., H:], H + 2 * W, d[ly, ..., H + W:], H + 2 * W,
                              None, w[ly], rp[ly])
    ctx.amph_paged_evict(pool.kv, layers, budget, recent, longest, i32(prompts), kv_len, kv_len, w, w, rp, rp, ws)
    # the reference: per (layer, sequence) the rows by position, per head which position a row has and its weight
    keys = [[pr.turn(first[ly, b, :, H:H + W].view(-1, n_kv, dim), torch.arange(longest)[:, None], theta).to(tdt) for b in range(n)] for ly in range(layers)]
    vals = [[first[ly, b, :, H + W:].reshape(-1, n_kv, dim) for b in range(n)] for ly in range(layers)]
    keys, vals = ([[list(x[b][:prompts[b]]) for b in range(n)] for x in y] for y in (keys, vals))
    held = [[[list(range(p)) for _ in range(n_kv)] for p in prompts] for _ in range(layers)]
    mass = [[[[0.0] * p for _ in range(n_kv)] for p in prompts] for _ in range(layers)]

    def cut(ly, b, h, R):
        at = pr.evict_rows(mass[ly][b][h], held[ly][b][h], R, budget, recent)
        held[ly][b][h], mass[ly][b][h] = [held[ly][b][h][r] for r in at], [mass[ly][b][h][r] for r in at]
    lens = []
    for b in range(n):
        for ly in range(layers):
            for h in range(n_kv):
                cut(ly, b, h, prompts[b])
        lens.append(min(prompts[b], budget))
    qkv, q_out = torch.zeros(layers, n, 1, H + 2 * W, dtype=tdt, device=DEV), torch.zeros(layers, n, 1, heads, dim, dtype=tdt, device=DEV)
    out = torch.zeros(layers, n, heads, dim, dtype=tdt, device=DEV)

    def step():
        for ly in range(layers):
            x = qkv[ly]
            ctx.amph_paged_append(pool.kv, ly, 1, valid, kv_len, pos, x, H + 2 * W, x[..., H:], H + 2 * W, x[..., H + W:], H + 2 * W, q_out[ly],
                                  w[ly], rp[ly])
            ctx.amph_paged_attn(pool.kv, ly, q_out[ly], H, 1, valid, kv_len, out[ly], w[ly], w[ly], ws)
        ctx.amph_paged_evict(pool.kv, layers, budget, recent, 1, valid, kv_len, kv_len, w, w, rp, rp, ws)
    run = step
    if graph:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        ctx.set_stream(side.cuda_stream)
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured, stream=side):
            step()
        run = captured.replay
    for t in range(steps):
        x = torch.randn(layers, n, H + 2 * W, generator=g).to(tdt)
        live = [0 if (b == 1 and t % 3 == 1) else 1 for b in range(n)]                 # one sequence idles now and then
        at = [len(keys[0][b]) for b in range(n)]
        qkv.copy_(x[:, :, None].to(DEV))
        pos.copy_(i32(at)[:, None])
        valid.copy_(i32(live))
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        w_now, p_now = w.cpu(), rp.cpu()
        for b in range(n):
            R = lens[b] + live[b]
            lens[b] = min(R, budget)
            for ly in range(layers):
                if live[b]:
                    keys[ly][b].append(pr.turn(x[ly, b, H:H + W].view(n_kv, dim), torch.full((n_kv,), at[b]), theta).to(tdt))
                    vals[ly][b].append(x[ly, b, H + W:].view(n_kv, dim))
                    q = pr.turn(x[ly, b, :H].view(heads, dim), torch.full((heads,), at[b]), theta).to(tdt)
                else:
                    q = q_out[ly, b, 0].cpu()                                            # an idle one attends with what was there
                for h in range(n_kv):
                    if live[b]:
                        held[ly][b][h].append(at[b])
                        mass[ly][b][h].append(0.0)
                    k, v = (torch.stack([x_[ly][b][p][h] for p in held[ly][b][h]])[None] for x_ in (keys, vals))
                    group = slice(h * (heads // n_kv), (h + 1) * (heads // n_kv))
                    ref, share, mag, reach = pr.attn(q[group], k, v)
                    # queries and keys of either side are a rounding apart at most now and then: a storage step of each in the scores
                    near = 2 * 2 * pr.HALF_STEP[dtype] * reach
                    most = pr.attn_bounds(dtype, ref, mag, reach, R, dim) + 2 * mag * near[:, None]
                    err = (out[ly, b, group].cpu().to(F64) - ref).abs()
                    assert bool((err <= most).all()), (t, ly, b, h, float((err / most).max()))
                    mass[ly][b][h] = [a + float(s) for a, s in zip(mass[ly][b][h], share[0])]
                    slack = 4 * float(near.max()) + (R + 200) * 2.0 ** -20
                    # the device's rows after its eviction, by position: right weights, and then its own choice is made again from them
                    rows = {int(p_now[ly, b, h, r]): float(w_now[ly, b, h, r]) for r in range(lens[b])}
                    assert len(rows) == lens[b] and set(rows) <= set(held[ly][b][h])
                    for i, p in enumerate(held[ly][b][h]):
                        if p in rows:
                            assert abs(rows[p] - mass[ly][b][h][i]) <= slack * max(mass[ly][b][h][i], 1e-3) * (t + 1), (t, p)
                            mass[ly][b][h][i] = rows[p]
                    gone = [i for i, p in enumerate(held[ly][b][h]) if p not in rows]
                    if gone:                                # one row went: no heavier than the lightest that could have gone
                        assert len(gone) == 1 and held[ly][b][h][gone[0]] <= max(held[ly][b][h]) - recent
                        free = [m for m, p in zip(mass[ly][b][h], held[ly][b][h]) if p <= max(held[ly][b][h]) - recent]
                        assert mass[ly][b][h][gone[0]] <= min(free) * (1 + slack * (t + 1)) + 1e-3 * slack * (t + 1)
                        mass[ly][b][h][gone[0]] = -1.0
                    cut(ly, b, h, R)
                    assert held[ly][b][h] == p_now[ly, b, h, :lens[b]].tolist()
        assert kv_len.tolist() == lens
    assert ctx.device_status() == 0


def test_decoding_with_a_budget_bf16():
    decode("bf16", 8, 2, 128, [37, 5, 120], budget=64, recent=8, steps=40, layers=2, per=4)


def test_decoding_with_a_budget_f32():
    decode("f32", 4, 4, 64, [10, 90], budget=50, recent=1, steps=30, layers=1, per=3)


def test_decoding_captured_and_replayed():
    """The same loop as one graph a step, its lengths, positions and idle sequences changing between replays; several workgroups a walk."""
    decode("bf16", 8, 2, 64, [700, 30], budget=600, recent=20, steps=8, layers=2, per=24, graph=True)


@pytest.mark.parametrize("cfg,lens,budget", [(si.MINI, [77, 200, 5], 64), (si.TINY, [130, 100, 131], 100)])
def test_the_step_s_caches_appended_to_evicted_and_verified(cfg, lens, budget):
    """The caches of amph_target_forward, three layers of them: rows appended where they lie, every head held to a budget, and the tree attention
    over what is left, with a tree whose rows come behind it."""
    d_h, n_h, bsz, max_kv, layers, n_new = cfg.head_dim, cfg.n_heads, 3, 256, 3, 3
    ctx = B.Context(d_model=n_h * d_h, n_heads=n_h, head_dim=d_h, d_ffn=64, vocab=64, K=4, topk=4, max_tree=8, max_kv=max_kv, batch=bsz,
                    dtype=D.dtype_code(cfg.dtype), device=DEV)
    tdt, tree = D.torch_dtype(cfg.dtype), B.Tree(si.tree_paths(8, (4, 2, 2, 2)), 4)
    g = torch.Generator().manual_seed(11)
    k, v = (torch.randn(layers, bsz, n_h, max_kv, d_h, generator=g).to(tdt) for _ in range(2))
    kc, vc = lr.keys_to_tiled(k).to(DEV), lr.values_to_tiled(v).to(DEV)
    kv, table = D.paged_caches(kc, vc, 64)
    w = torch.rand(layers, bsz, n_h, max_kv, generator=g)
    pos = torch.arange(max_kv, dtype=torch.int32).expand(layers, bsz, n_h, max_kv).contiguous()
    w_d, p_d, n, out_n = w.to(DEV), pos.to(DEV), i32(lens), i32([0] * bsz)
    new = torch.randn(layers, bsz, n_new, 2 * n_h * d_h, generator=g).to(tdt)
    d = new.to(DEV)
    for ly in range(layers):
        x = d[ly]
        ctx.amph_paged_append(kv, ly, n_new, None, n, None, None, 0, x, 2 * n_h * d_h, x[..., n_h * d_h:], 2 * n_h * d_h, None, w_d[ly], p_d[ly])
    k, v = lr.tiled_to_keys(kc.cpu()), lr.tiled_to_values(vc.cpu())        # (the appended rows: checked here against the new ones)
    for b, L in enumerate(lens):
        rows = new[:, b, :, :n_h * d_h].view(layers, n_new, n_h, d_h)
        ref = pr.turn(rows, (L + torch.arange(n_new))[:, None].expand(n_new, n_h), 10000.0)
        assert bool(((k[:, b, :, L:L + n_new].transpose(1, 2).to(F64) - ref).abs() <= pr.turn_bounds(cfg.dtype, rows, ref)).all())
        assert torch.equal(v[:, b, :, L:L + n_new].transpose(1, 2), new[:, b, :, n_h * d_h:].view(layers, n_new, n_h, d_h))
        w[:, b, :, L:L + n_new] = 0.0
    ctx.amph_paged_evict(kv, layers, budget, 10, n_new, None, n, out_n, w_d, w_d, p_d, p_d, workspace(ctx, kv, layers))
    q, out = torch.randn(bsz, 8, n_h, d_h, generator=g).to(tdt), torch.zeros(bsz, 8, n_h, d_h, dtype=tdt, device=DEV)
    assert out_n.tolist() == [min(L + n_new, budget) for L in lens]
    mask = torch.from_numpy(tree.mask_bool())
    for ly in range(layers):
        ctx.amph_verify_attn(tree, q.to(DEV), kc[ly], vc[ly], out_n, out)
        k_now, v_now = lr.tiled_to_keys(kc[ly].cpu()), lr.tiled_to_values(vc[ly].cpu())
        for b, L in enumerate(lens):
            for h in range(n_h):
                at = pr.evict_rows(w[ly, b, h].tolist(), pos[ly, b, h].tolist(), L + n_new, budget, 10)
                m = len(at)
                keys = torch.cat([k[ly, b, h, torch.tensor(at)], k_now[b, h, m:m + 8]])        # (the tree's rows: whatever lies there)
                vals = torch.cat([v[ly, b, h, torch.tensor(at)], v_now[b, h, m:m + 8]])
                for node in range(8):
                    see = torch.cat([torch.ones(m, dtype=torch.bool), mask[node]])
                    ref, _, mag, reach = pr.attn(q[b, node, h:h + 1], keys[None, see], vals[None, see])
                    most = pr.attn_bounds(cfg.dtype, ref, mag, reach, m + 8, d_h) + (mag * 2.0 ** -8 if cfg.dtype == "bf16" else 0.0)
                    assert bool(((out[b, node, h:h + 1].cpu().to(F64) - ref).abs() <= most).all()), (ly, b, h, node)
    assert ctx.device_status() == 0


def test_two_streams_with_workspaces_of_their_own():
    """Two contexts on two streams at once, each captured and replayed many times, against their own eager results."""
    sides = []
    for seed, lens in ((1, [3000, 17]), (2, [900, 2500])):
        pool, ctx = Pool("bf16", 2, 128, 64, lens, 48, seed=seed), pr.make_ctx("bf16", 8, 128)
        q, out = torch.randn(2, 8, 128, device=DEV).to(torch.bfloat16), torch.zeros(2, 8, 128, device=DEV, dtype=torch.bfloat16)
        w, ws, n = torch.zeros(2, 2, pool.cap, device=DEV), workspace(ctx, pool.kv, 1), i32(lens)
        call = lambda ctx=ctx, pool=pool, q=q, n=n, out=out, w=w, ws=ws: ctx.amph_paged_attn(pool.kv, 0, q, 1024, 0, None, n, out, None, w, ws)  # noqa: E731
        call()
        torch.cuda.synchronize()
        want = out.clone(), w.clone()
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        ctx.set_stream(stream.cuda_stream)
        with torch.cuda.graph(graph, stream=stream):
            call()
        sides.append((graph, stream, out, w, want, (pool, ctx, q, ws, n)))
    for _ in range(5):
        for graph, stream, out, w, *_ in sides:
            out.zero_()
            w.zero_()
        torch.cuda.synchronize()
        for _ in range(10):
            for graph, stream, *_ in sides:
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for graph, stream, out, w, want, _ in sides:
            assert torch.equal(out, want[0]) and torch.equal(w, want[1])


def test_graphs_that_share_a_workspace():
    """An attention with weights and an eviction, captured apart over one workspace, replayed in turn on one stream with eager calls in between:
    nothing of a call is left there for the next."""
    pools = [Pool("bf16", 2, 128, 64, lens, 20, seed=i) for i, lens in enumerate(([1200, 60], [300, 1100]))]
    ctx, n = pr.make_ctx("bf16", 8, 128), [i32([1200, 60]), i32([300, 1100])]
    ws, q = workspace(ctx, pools[0].kv, 1), torch.randn(2, 8, 128, device=DEV).to(torch.bfloat16)
    outs, ws_w = [torch.zeros_like(q) for _ in range(2)], [torch.zeros(1, 2, 2, 1280, device=DEV) for _ in range(2)]
    pos, kept = torch.arange(1280, device=DEV, dtype=torch.int32).expand(1, 2, 2, 1280).contiguous(), [torch.zeros(1, 2, 2, 1280, device=DEV) for _ in range(2)]
    places, left = [torch.zeros_like(pos) for _ in range(2)], [i32([0, 0]) for _ in range(2)]
    mass = torch.rand(1, 2, 2, 1280, device=DEV)                      # what the evictions go by: the same in every pass

    def attend(i):
        ctx.amph_paged_attn(pools[i].kv, 0, q, 1024, 0, None, n[i], outs[i], None, ws_w[i], ws)

    def drop(i):
        ctx.amph_paged_evict(pools[i].kv, 1, 256, 10, 0, None, n[i], left[i], mass, kept[i], pos, places[i], ws)
    attend(0), attend(1), drop(0), drop(1)
    torch.cuda.synchronize()
    # (rows moved below the budget: from here on every pass sees the same caches, as the same rows move to the same places again)
    attend(0), attend(1), drop(0), drop(1)
    torch.cuda.synchronize()
    want = [x.clone() for x in outs + ws_w + kept + places + left]
    stream, graphs = torch.cuda.Stream(), []
    ctx.set_stream(stream.cuda_stream)
    for call, i in ((attend, 0), (attend, 1), (drop, 0), (drop, 1)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(i)
        graphs.append(graph)
    for turn in range(4):
        with torch.cuda.stream(stream):
            for x in outs + kept + places:
                x.zero_()
            for graph in graphs:
                graph.replay()
            if turn % 2:
                attend(1)
        torch.cuda.synchronize()
        for x, y in zip(outs + ws_w + kept + places + left, want):
            assert torch.equal(x, y), turn
    assert ctx.device_status() == 0


def test_refusals():
    pool, ctx = Pool("bf16", 2, 64, 32, [10, 10], 2, layers=2), pr.make_ctx("bf16", 4, 64)
    q = torch.zeros(2, 3, 256, device=DEV, dtype=torch.bfloat16)
    out, w, pos, n = torch.zeros_like(q), torch.zeros(2, 2, 2, 64, device=DEV), torch.zeros(2, 2, 2, 64, device=DEV, dtype=torch.int32), i32([10, 10])
    ws, kv = workspace(ctx, pool.kv, 2), pool.kv

    def refused(status, f, *a, **k):
        with pytest.raises(B.AmphError) as e:
            f(*a, **k)
        assert e.value.status == status and len(str(e.value)) > 20, str(e.value)

    def other(**kw):
        c = B.amph_paged_kv.from_buffer_copy(kv)
        for k, x in kw.items():
            setattr(c, k, x)
        return c
    A, P, E = ctx.amph_paged_attn, ctx.amph_paged_append, ctx.amph_paged_evict
    shape, inval = B.AMPH_ESHAPE, B.AMPH_EINVAL
    att = dict(layer=0, q=q, ld_q=256, n_new=0, n_valid=None, kv_len=n, out=out, workspace=ws)
    for kw, st in [(dict(q=None), inval), (dict(out=None), inval), (dict(kv_len=None), inval), (dict(workspace=None), inval), (dict(out=q), inval),
                   (dict(weights_in=w), inval), (dict(layer=-1), inval), (dict(n_new=-1), inval), (dict(n_new=65), shape), (dict(ld_q=255), inval),
                   (dict(ld_q=-256), inval), (dict(q=q.data_ptr() + 2), inval), (dict(out=out.data_ptr() + 8), inval),
                   (dict(workspace=ws.data_ptr() + 4), inval), (dict(kv_len=n.data_ptr() + 1), inval), (dict(weights_out=w.data_ptr() + 2), inval)]:
        refused(st, A, kv, **{**att, **kw})
    for bad, st in [(other(n_kv_heads=3), shape), (other(page_rows=16), shape), (other(max_pages=3), shape), (other(n_seq=0), inval),
                    (other(k_pages=0), inval), (other(page_stride=4), inval), (other(n_seq=1025), shape)]:
        refused(st, A, bad, **att)
        refused(st, P, bad, 0, 1, None, n, None, q, 256, q, 128, q, 128, out)
        refused(st, E, bad, 1, 5, 0, 0, None, n, n, w, w, pos, pos, ws)
        refused(st, ctx.amph_paged_workspace_bytes, bad)
    app = dict(layer=0, n_new=3, n_valid=None, kv_len=n, pos=None, q=q, ld_q=256, k=q, ld_k=128, v=q, ld_v=128, q_out=out)
    for kw, st in [(dict(k=None), inval), (dict(v=None), inval), (dict(kv_len=None), inval), (dict(q=None), inval), (dict(q_out=None), inval),
                   (dict(layer=-2), inval), (dict(n_new=0), inval), (dict(n_new=-3), inval), (dict(n_new=65), shape), (dict(ld_k=120), shape),
                   (dict(ld_v=64), shape), (dict(ld_q=128), shape), (dict(ld_k=132), inval), (dict(q_out=q, ld_q=512), inval),
                   (dict(k=q.data_ptr() + 2), inval), (dict(weights=w.data_ptr() + 1), inval)]:
        refused(st, P, kv, **{**app, **kw})
    ev = dict(n_layers=2, budget=5, recent=2, n_new=1, n_valid=None, kv_len=n, kv_len_out=n, weights_in=w, weights_out=w, row_pos_in=pos,
              row_pos_out=pos, workspace=ws)
    for kw, st in [(dict(n_layers=0), inval), (dict(budget=0), inval), (dict(recent=-1), inval), (dict(recent=6), inval), (dict(n_new=-1), inval),
                   (dict(n_new=65), shape), (dict(kv_len=None), inval), (dict(kv_len_out=None), inval), (dict(weights_in=None), inval),
                   (dict(weights_out=None), inval), (dict(row_pos_in=None), inval), (dict(row_pos_out=None), inval), (dict(workspace=None), inval),
                   (dict(workspace=ws.data_ptr() + 8), inval)]:
        refused(st, E, kv, **{**ev, **kw})
    c = C.c_size_t()
    assert B.lib().amph_paged_bytes(ctx.handle, C.byref(kv), 0, None) == inval and B.lib().amph_paged_bytes(ctx.handle, C.byref(kv), 0, C.byref(c)) == 0
    torch.cuda.synchronize()
    assert ctx.device_status() == 0 and n.tolist() == [10, 10] and bool((out == 0).all())
