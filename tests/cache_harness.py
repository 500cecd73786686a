"""A paged cache for the tests of the calls that fill and read it: pool, page
table and the host's view of the rows."""
from __future__ import annotations

import numpy as np
import torch

DEV = "cuda"


def bf16(x):
    """float64 values rounded to bf16, as (torch tensor on the GPU, float64)."""
    t = torch.from_numpy(np.asarray(x, dtype=np.float32)).bfloat16()
    return t.to(DEV), t.double().numpy()


def f64(t):
    return t.detach().double().cpu().numpy()


class Cache:
    """One layer (of `layers`) of a paged pool, every byte preset to `fill`
    (0xff: NaN in bf16, a NaN block in 4 bits), pages scattered."""

    def __init__(self, E, rng, fmt, B, H, d, page, room, layers=1, layer=0, spare=3, fill=0xff,
                 gap=0, **cfg):
        self.E, self.fmt, self.H, self.d, self.page, self.layer = E, fmt, H, d, page, layer
        self.cfg = E.default_cfg(batch=B, n_layers=layers, n_kv_heads=H, head_dim=d,
                                 page_size=page, kv_format=fmt, **cfg)
        self.row = E.kv_row_bytes(self.cfg)
        width = -(-max(room, 1) // page)
        n_pages = B * width + spare
        self.bytes = torch.full((layers, 2, n_pages, page * self.row + gap), fill,
                                dtype=torch.uint8, device=DEV)
        ids = rng.permutation(n_pages)[:B * width].reshape(B, width).astype(np.int32)
        self.table_host = ids
        self.table = torch.from_numpy(ids).to(DEV)
        self.ld_pt = width
        s = self.bytes.stride()
        self.pool = E.Pool(self.bytes.data_ptr(), s[0], s[1], s[2], n_pages)

    def put(self, b, kv, first, rows):
        """Raw rows [n][row] uint8 at slots first..."""
        host = torch.from_numpy(np.ascontiguousarray(rows)).to(DEV)
        for i in range(rows.shape[0]):
            pg, at = self.table_host[b, (first + i) // self.page], (first + i) % self.page
            self.bytes[self.layer, kv, int(pg), at * self.row:(at + 1) * self.row] = host[i]

    def fill_rows(self, b, kv, rows):
        """Slots 0.. of a sequence, page by page."""
        for m in range(0, rows.shape[0], self.page):
            part = np.ascontiguousarray(rows[m:m + self.page]).reshape(-1)
            self.bytes[self.layer, kv, int(self.table_host[b, m // self.page]),
                       :part.size] = torch.from_numpy(part).to(DEV)

    def rows(self, b, kv, n):
        """Raw rows [n][row] of slots 0..n-1."""
        host = self.bytes[self.layer, kv].cpu().numpy()
        out = np.empty((n, self.row), dtype=np.uint8)
        for i in range(n):
            at = i % self.page
            out[i] = host[self.table_host[b, i // self.page], at * self.row:(at + 1) * self.row]
        return out

    def encode(self, x):
        """float64 [n][H][d] as raw rows, and the values they hold."""
        import oracle.cache_ref as R
        n = x.shape[0]
        if self.fmt == self.E.KV_BF16:
            t = torch.from_numpy(x.astype(np.float32)).bfloat16().reshape(n, self.H * self.d)
            return t.view(torch.uint8).numpy(), t.double().numpy().reshape(x.shape)
        codes, byte = quick_encode(x.reshape(n, self.H * self.d))
        row = R.mxfp4_pack(codes, byte, self.row)
        return row, R.mxfp4_decode(row, self.H * self.d).reshape(x.shape)


def quick_encode(x):
    """The oracle's 4-bit encoding, whole arrays at a time (checked against
    it on the CPU)."""
    import oracle.cache_ref as R
    x = np.asarray(x, dtype=np.float64)
    blk = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    m = np.abs(blk).max(-1)
    good = np.isfinite(m)
    safe = np.where(good & (m > 0), m, 1.0)
    e = np.floor(np.log2(safe)) - 2
    e += safe > 7 * 2.0 ** e
    e = np.where(m == 0, -126, np.maximum(e, -126))
    mid = (R.E2M1[1:] + R.E2M1[:-1]) / 2
    with np.errstate(invalid="ignore", over="ignore"):
        a = np.abs(blk) / 2.0 ** e[..., None]
        code = np.zeros(a.shape, dtype=np.uint8)
        for i, t in enumerate(mid):
            code += (a > t) if i % 2 == 0 else (a >= t)
    code = np.where(good[..., None], code | (np.signbit(blk) << 3), 0).astype(np.uint8)
    byte = np.where(good, e + 127, 255).astype(np.uint8)
    return code.reshape(x.shape), byte
