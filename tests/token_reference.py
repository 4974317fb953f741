"""Plain 64-bit forms of the operators for several tokens per user, and caches in every storage layout (test infrastructure: torch
indexing and numpy only)."""
import numpy as np
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # of a rounding, relative


class Cache:
    """Rows k[u], v[u] ([len, H, d], any device) stored in a layout, with room for `room` more tokens, and a view of it.
    layout: hnd, nhd, exact (a buffer of its own size per user), tables (hnd, device pointer tables), paged_hnd16, paged_nhd64, ..."""

    def __init__(self, spd, k, v, layout, device, seed=0, fill=float("nan")):
        self.layout, n = layout, len(k)
        H, d, dt = k[0].shape[1], k[0].shape[2], k[0].dtype
        self.lens = np.array([t.shape[0] for t in k], np.int32)
        self.table, self.page = None, 0
        if layout.startswith("paged"):
            self.head_major, self.page = "hnd" in layout, int(layout.lstrip("pagednh_"))
            B = self.page
            pages = [-(-int(x) // B) for x in self.lens]
            order = np.random.default_rng(seed).permutation(sum(pages) + 2).astype(np.int32)
            bad = order[-1]                                  # a page that no token lies in: what a table's unused entries name
            table, at = np.full((n, max(pages + [1]) + 1), bad, np.int32), 0
            for u, p in enumerate(pages):
                table[u, :p] = order[at:at + p]
                at += p
            shape = (len(order), H, B, d) if self.head_major else (len(order), B, H, d)
            self.k, self.v = (torch.full(shape, fill, dtype=dt, device=device) for _ in range(2))
            self.table = table
            strides = (d, B * d) if self.head_major else (H * d, d)
            table_dev = torch.from_numpy(table).to(device)
            self.view = spd.KVView(self.lens, *strides, k_pool=self.k, v_pool=self.v, block_table=table_dev, block_size=B, block_stride=H * B * d)
        elif layout == "exact":
            self.head_major = True
            self.k, self.v = ([torch.full((H, int(x), d), fill, dtype=dt, device=device) for x in self.lens] for _ in range(2))
            self.view = spd.KVView(self.lens, d, 0, k=self.k, v=self.v, head_strides=self.lens.astype(np.int64) * d)
        else:
            self.head_major = layout in ("hnd", "tables")
            room = int(max(self.lens)) + 5
            shape = (n, H, room, d) if self.head_major else (n, room, H, d)
            self.k, self.v = (torch.full(shape, fill, dtype=dt, device=device) for _ in range(2))
            strides = (d, room * d) if self.head_major else (H * d, d)
            self.view = spd.KVView(self.lens, *strides, k=list(self.k), v=list(self.v), device_pointer_tables=layout == "tables")
        for u in range(n):
            self.put(u, 0, k[u], v[u])

    def _place(self, store, u, t):
        if self.page:
            page, at = int(self.table[u, t // self.page]), t % self.page
            return store[page, :, at] if self.head_major else store[page, at]
        return store[u][:, t] if self.head_major else store[u][t]

    def put(self, u, first, k, v):
        n = k.shape[0]
        if self.page:
            at = np.arange(first, first + n)
            page, at = torch.from_numpy(self.table[u, at // self.page]).long(), torch.from_numpy(at % self.page)
            for store, rows in ((self.k, k), (self.v, v)):
                page, at = page.to(store.device), at.to(store.device)
                if self.head_major:
                    store[page, :, at] = rows.to(store.device)
                else:
                    store[page, at] = rows.to(store.device)
        elif n:
            for store, rows in ((self.k, k), (self.v, v)):
                rows = rows.to(store[u].device)
                if self.head_major:
                    store[u][:, first:first + n] = rows.transpose(0, 1)
                else:
                    store[u][first:first + n] = rows

    def bits(self):
        return [t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16).cpu() for s in (self.k, self.v)
                for t in (s if isinstance(s, list) else [s])]


def visible(n, held, q_pos, k_pos, causal=False, window=0, prefix=None, ranges=None):
    """[n, held] bool, from the definition."""
    q, k = (q_pos + np.arange(n))[:, None], (k_pos + np.arange(held))[None]
    see = np.ones((n, held), bool)
    if causal:
        see &= k <= q
    if window:
        see &= np.abs(q - k) < window
    if prefix is not None:
        see |= k < prefix
    if ranges is not None:
        see &= (k >= ranges[:, :1]) & (k < ranges[:, 1:])
    return see


def attend(q, k, v, see, scale, cap=0.0, slopes=None, distance=None):
    """One user in 64 bits: q [n, Hq, d], k and v [held, H, d] -> A [n, Hq, d], lse [n, Hq], sum of p |v|, and the largest sum of |q_c k_c| * |scale|."""
    n, Hq, d = q.shape
    H, G = k.shape[1], Hq // k.shape[1]
    a = torch.zeros((n, Hq, d), dtype=torch.float64)
    b, lse, most = torch.zeros_like(a), torch.full((n, Hq), -np.inf, dtype=torch.float64), 0.0
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    see = torch.from_numpy(see)
    if k.shape[0] == 0 or n == 0:
        return a, lse, b, most
    for h in range(Hq):
        x = q[:, h] @ k[:, h // G].t() * scale
        most = max(most, float((q[:, h].abs() @ k[:, h // G].abs().t())[see].max()) * abs(scale) if see.any() else 0.0)
        if cap:
            x = cap * torch.tanh(x / cap)
        if slopes is not None:
            x = x - float(slopes[h]) * distance
        x = torch.where(see, x, -np.inf)
        lse[:, h] = torch.logsumexp(x, 1)
        p = torch.where(see, torch.exp(x - torch.where(torch.isinf(lse[:, h:h + 1]), 0.0, lse[:, h:h + 1])), 0.0)
        a[:, h], b[:, h] = p @ v[:, h // G], p @ v[:, h // G].abs()
    return a, lse, b, most


def turn(x, positions, inv_freq, pair_axis, adjacent, amplitude=1.0, transposed=False):
    """Rotary positions in 64 bits: x [T, H, d], positions [axes, T]."""
    P = inv_freq.numel()
    angle = positions.double().cpu()[torch.from_numpy(np.asarray(pair_axis)).long()].t() * inv_freq.double().cpu()
    c, s = (amplitude * f(angle)[:, None] for f in (torch.cos, torch.sin))
    if transposed:
        s = -s
    y = x.double().cpu().clone()
    i, j = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if adjacent else (slice(0, P), slice(P, 2 * P))
    x0, x1 = y[..., i].clone(), y[..., j].clone()
    y[..., i], y[..., j] = x0 * c - x1 * s, x0 * s + x1 * c
    return y, x0.abs() + x1.abs()
