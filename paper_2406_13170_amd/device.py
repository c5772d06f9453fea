"""Host->device marshalling of synthetic tensors (data movement and layout only, no arithmetic)."""
from __future__ import annotations

from typing import Dict

import numpy as np
import torch

from .binding import (AMPH_BF16, AMPH_F32, AMPH_PACK_DOWN, AMPH_PACK_GATEUP, AMPH_PACK_LMHEAD, AMPH_PACK_QKV,
                      AMPH_PACK_WO, amph_layer_tiled, amph_paged_kv)


def dtype_code(name: str) -> int:
    return AMPH_BF16 if name == "bf16" else AMPH_F32


def torch_dtype(name: str):
    return torch.bfloat16 if name == "bf16" else torch.float32


def to_device(t, device="cuda:0") -> torch.Tensor:
    """synth_inputs.Tensor -> device tensor holding exactly the same values (bf16 patterns or float32)."""
    if t.dtype == "bf16":
        return torch.from_numpy(t.dev.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(t.dev)).to(device)


def layer_to_device(lw: Dict[str, object], device="cuda:0") -> Dict[str, torch.Tensor]:
    return {k: to_device(v, device) for k, v in lw.items()}


def draft_to_device(dw: Dict[str, object], device="cuda:0") -> Dict[str, object]:
    out = {}
    for k, v in dw.items():
        if k == "sal":
            out[k] = [layer_to_device(l, device) for l in v]
        elif k == "fc":
            out[k] = [to_device(x, device) for x in v]
        else:
            out[k] = to_device(v, device)
    return out


def _kv_check(ctx, t: torch.Tensor) -> int:
    """Number of [max_kv, head_dim] caches in t (all leading dimensions); shape and type must be the context's."""
    assert t.is_contiguous() and t.shape[-2] == ctx.cfg.max_kv and t.shape[-1] == ctx.cfg.head_dim, tuple(t.shape)
    assert t.dtype == (torch.bfloat16 if ctx.cfg.dtype == AMPH_BF16 else torch.float32)
    return t.numel() // (t.shape[-2] * t.shape[-1])


def pack_kv(ctx, k_rows: torch.Tensor, v_rows: torch.Tensor):
    """Row-major caches [..., max_kv, head_dim] -> their step-tiled storage (amph_pack_kv); same shapes."""
    k_t, v_t = torch.empty_like(k_rows), torch.empty_like(v_rows)
    n = _kv_check(ctx, k_rows)
    assert _kv_check(ctx, v_rows) == n
    ctx.amph_pack_kv(k_rows, v_rows, k_t, v_t, n)
    return k_t, v_t


def unpack_kv(ctx, k_tiled: torch.Tensor, v_tiled: torch.Tensor):
    """Step-tiled caches -> row-major [..., max_kv, head_dim] (amph_unpack_kv)."""
    k_r, v_r = torch.empty_like(k_tiled), torch.empty_like(v_tiled)
    n = _kv_check(ctx, k_tiled)
    assert _kv_check(ctx, v_tiled) == n
    ctx.amph_unpack_kv(k_tiled, v_tiled, k_r, v_r, n)
    return k_r, v_r


def pack_layer(ctx, lw: Dict[str, torch.Tensor]):
    """Tiled copies of one target layer's matrices (amph_pack_weights).  Returns (amph_layer_tiled, tensors):
    the caller keeps `tensors` alive as long as the struct is used."""
    dev = lw["wq"].device

    def buf(role):
        return torch.empty(ctx.amph_tiled_bytes(role), dtype=torch.uint8, device=dev)

    t = {"qkv": buf(AMPH_PACK_QKV), "wo": buf(AMPH_PACK_WO), "gate_up": buf(AMPH_PACK_GATEUP), "down": buf(AMPH_PACK_DOWN)}
    ctx.amph_pack_weights(AMPH_PACK_QKV, lw["wq"], lw["wk"], lw["wv"], t["qkv"])
    ctx.amph_pack_weights(AMPH_PACK_WO, lw["wo"], None, None, t["wo"])
    ctx.amph_pack_weights(AMPH_PACK_GATEUP, lw["w_gate"], lw["w_up"], None, t["gate_up"])
    ctx.amph_pack_weights(AMPH_PACK_DOWN, lw["w_down"], None, None, t["down"])
    s = amph_layer_tiled(*[t[k].data_ptr() for k in ("qkv", "wo", "gate_up", "down")])
    return s, t


def pack_lm_head(ctx, lm_head: torch.Tensor) -> torch.Tensor:
    out = torch.empty(ctx.amph_tiled_bytes(AMPH_PACK_LMHEAD), dtype=torch.uint8, device=lm_head.device)
    ctx.amph_pack_weights(AMPH_PACK_LMHEAD, lm_head, None, None, out)
    return out


def paged_pool(k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, max_pages: int | None = None) -> amph_paged_kv:
    """A pool of pages [n_layers, n_pages, n_kv_heads, page_rows, head_dim] (step-tiled) and its table [n_seq, table_pages] int32 as the
    paged calls take them.  The caller keeps the tensors alive as long as the struct is used."""
    assert k_pages.shape == v_pages.shape and k_pages.dim() == 5 and k_pages.is_contiguous() and v_pages.is_contiguous()
    assert k_pages.dtype == v_pages.dtype and table.dtype == torch.int32 and table.dim() == 2 and table.is_contiguous()
    _, n_pages, n_kv, rows, d_h = k_pages.shape
    page = rows * d_h
    return amph_paged_kv(k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), table.shape[0], n_kv, rows, n_pages, table.shape[1],
                         table.shape[1] if max_pages is None else max_pages, n_kv * page, page, n_pages * n_kv * page)


def paged_caches(k_caches: torch.Tensor, v_caches: torch.Tensor, page_rows: int):
    """The caches of amph_target_forward, [n_layers, B, n_heads, max_kv, head_dim] (step-tiled), as pages of page_rows rows where they
    lie.  Returns (amph_paged_kv, table): the caller keeps the table and the caches alive as long as the struct is used."""
    assert k_caches.shape == v_caches.shape and k_caches.dim() == 5 and k_caches.is_contiguous() and v_caches.is_contiguous()
    assert k_caches.dtype == v_caches.dtype and k_caches.shape[3] % page_rows == 0
    _, batch, n_h, max_kv, d_h = k_caches.shape
    per = max_kv // page_rows
    first = torch.arange(batch, dtype=torch.int32, device=k_caches.device) * (n_h * per)
    table = (first[:, None] + torch.arange(per, dtype=torch.int32, device=k_caches.device)).contiguous()
    return amph_paged_kv(k_caches.data_ptr(), v_caches.data_ptr(), table.data_ptr(), batch, n_h, page_rows, batch * n_h * per, per, per,
                         page_rows * d_h, max_kv * d_h, batch * n_h * max_kv * d_h), table
