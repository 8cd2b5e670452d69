"""Plain 64-bit forms of the paged-cache operators and of the verification, and cases for their tests."""
import numpy as np
import torch

LEAST = -100


def quantise(x):
    """float64 rows [..., d] -> (values that an 8-bit row holds, exponent), element by element from the definition."""
    x = np.asarray(x, dtype=np.float64)
    fin = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    e = np.full(fin.shape, LEAST, dtype=np.int64)
    while True:                                       # the smallest e with max <= 448 * 2^e
        more = fin > 448.0 * np.exp2(e.astype(np.float64))
        if not more.any():
            break
        e = e + more
    unit = np.exp2(e.astype(np.float64))[..., None]
    most = np.where(e == 120, 240.0, 448.0)[..., None]           # 256 * 2^120 is no fp32 number
    y = np.clip(np.where(np.isnan(x), 0.0, x) / unit, -most, most)
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -30))), -6.0) - 3.0)
    return np.where(np.isnan(x).any(-1, keepdims=True), np.nan, np.round(y / step) * step * unit), e


class Case:
    """Sequences of rows[s] new rows behind kv[s] positions, pages anywhere in a pool whose unwritten slots are NaN."""

    def __init__(self, b, rows, kv, kv_heads=2, dim=128, page=16, kind="bf16", dtype=torch.float32, seed=0, extra_pages=3, pad_rows=2, lead_rows=0,
                 amplitude=1.0):
        g = torch.Generator().manual_seed(seed)
        self.b, self.rows, self.kv, self.H, self.D, self.P, self.dtype = b, list(rows), list(kv), kv_heads, dim, page, dtype
        need = [-(-(r + n) // page) for r, n in zip(rows, kv)]
        n_pages = sum(need) + extra_pages
        order = torch.randperm(n_pages, generator=g).int()
        table = torch.full((len(rows), max(max(need), 1)), -5, dtype=torch.int32)      # entries behind a sequence's pages are not ids
        at = 0
        for s, n in enumerate(need):
            table[s, :n] = order[at:at + n]
            at += n
        self.table = table
        self.start = np.concatenate([[0], np.cumsum(rows)]) + lead_rows
        self.total = int(self.start[-1]) + pad_rows
        # float64 values of every sequence's keys and values, as a pool of this kind holds them
        self.keys, self.vals = [], []
        for s, (r, n) in enumerate(zip(rows, kv)):
            k, v = (torch.randn(n + r, kv_heads, dim, generator=g) * amplitude * torch.exp(0.7 * torch.randn(n + r, kv_heads, 1, generator=g)) for _ in range(2))
            k, v = k.to(dtype), v.to(dtype)
            self.keys.append(k)
            self.vals.append(v)
        self.pool = b.KvPool.empty(n_pages, page, kv_heads, dim, torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn)
        for t in (self.pool.k, self.pool.v):
            t.view(torch.uint8).fill_(0xFF)           # NaN in both kinds
        if kind != "bf16":
            self.pool.k_exp.fill_(255)
            self.pool.v_exp.fill_(255)
        self.kind = kind

    def held(self, x):
        x = x.double().numpy()
        return torch.from_numpy(x).bfloat16().double().numpy() if self.kind == "bf16" else quantise(x)[0]

    def batch(self, rows=None, kv=None, start=None, total=None, max_rows=None):
        start = self.start if start is None else start
        return self.b.PagedBatch(self.table.cuda(), torch.tensor(np.asarray(start), dtype=torch.int32).cuda(),
                                 torch.tensor(self.kv if kv is None else kv, dtype=torch.int32).cuda(), self.total if total is None else total,
                                 max(max(self.rows), 1) if max_rows is None else max_rows)

    def packed(self, parts, lead=None):
        """[total, heads, d] on the GPU with NaN in rows that belong to no sequence."""
        H, D = parts[0].shape[1:]
        out = torch.full((self.total, H, D), float("nan"), dtype=self.dtype)
        for s, p in enumerate(parts):
            out[self.start[s]:self.start[s] + len(p)] = p.to(self.dtype)
        return out.cuda()

    def fill(self):
        """Writes positions 0 .. kv and then the new rows, as two appends; returns the batch of the new rows."""
        if sum(self.kv):
            start = np.concatenate([[0], np.cumsum(self.kv)])
            old = self.b.PagedBatch(self.table.cuda(), torch.tensor(start, dtype=torch.int32).cuda(), torch.zeros(len(self.kv), dtype=torch.int32).cuda(),
                                    int(start[-1]), max(max(self.kv), 1))
            cat = lambda parts: torch.cat([p[:n] for p, n in zip(parts, self.kv)]).cuda()  # noqa: E731
            self.b.csd_paged_append(self.pool, old, cat(self.keys), cat(self.vals))
        new = self.batch()
        self.b.csd_paged_append(self.pool, new, self.packed([k[n:] for k, n in zip(self.keys, self.kv)]), self.packed([v[n:] for v, n in zip(self.vals, self.kv)]))
        return new


def trees(rows, seed, empty=()):
    """Masks of random trees [sum(rows)], a row's ancestors and itself; rows in `empty` see nothing of the block."""
    rng = np.random.default_rng(seed)
    out = []
    for n in rows:
        mine = []
        for r in range(n):
            mine.append((mine[int(rng.integers(0, r))] if r else 0) | (1 << r))
        out += mine
    for r in empty:
        out[r] = 0
    return out


def attention(q, k, v, kv, scale, masks=None, hide=()):
    """float64 q [r, H, D] over k, v [n, Hkv, D]; returns the output, sum_j p_j |v_j|, and max_j scale |q|.|k_j|.  hide: positions nobody sees."""
    r, H, D = q.shape
    group = H // k.shape[1]
    out, size, top = np.zeros((r, H, D)), np.zeros((r, H, D)), 0.0
    for i in range(r):
        sees = [j for j in range(len(k)) if (j < kv or (j <= kv + i if masks is None else (masks[i] >> (j - kv)) & 1)) and j not in hide]
        if not sees:
            continue
        for h in range(H):
            kk, vv = k[sees, h // group], v[sees, h // group]
            x = kk @ q[i, h] * scale
            p = np.exp(x - x.max())
            p /= p.sum()
            out[i, h], size[i, h] = p @ vv, p @ np.abs(vv)
            top = max(top, float((np.abs(kk) @ np.abs(q[i, h])).max()) * abs(scale))
    return out, size, top


def attention_bound(out, size, top, n, dim, dtype):
    """What rounding allows.  Scores: fp32 sums of dim products (three bf16 terms each at most), and exp of a difference of at most
    2 top in fp32; each weight is off by a factor of that, once in the numerator and once in the sum.  Products with V: at most 3 n / 8 + 64
    fp32 additions of at most `size`.  bf16 rows: the weights are rounded to bf16, and the output is."""
    step = 2.0 ** -23
    score = top * step * (3 * dim / 16 + 8) + 2 * top * 2 * step + 4 * step
    rel = 2 * score + (3 * n / 8 + 64) * step
    if dtype == torch.bfloat16:
        return size * (rel + 2 * 2.0 ** -8) * 1.01 + np.abs(out) * 2.0 ** -8
    return size * rel * 1.01 + np.abs(out) * 2.0 ** -24


def verify(p, q, tokens, u, n):
    """float64 laws [k+1, V], [k, V] or None: (accepted, tokens)."""
    k = len(tokens)
    mass = lambda x: np.where((x > 0) & np.isfinite(x), x, 0.0)  # noqa: E731
    out, left = [], None
    for i in range(n):
        x = tokens[i]
        ok = 0 <= x < p.shape[1]
        if ok:
            qx = q[i, x] if q is not None else 1.0
            ok = u[i] * qx < p[i, x]
        if not ok:
            if q is not None:
                left = np.maximum(mass(p[i]) - np.where(q[i] > 0, q[i], 0.0), 0.0)        # (an infinite entry of q leaves nothing)
            else:
                left = mass(p[i]).copy()
                if 0 <= x < p.shape[1]:
                    left[x] = 0.0
            if left.sum() == 0:
                left = mass(p[i])
            break
        out.append(x)
    if left is None:
        left = mass(p[len(out)])
    c = np.cumsum(left)
    out.append(int(np.searchsorted(c, u[k] * c[-1], side="right")) if c[-1] > 0 else 0)
    return len(out) - 1, out + [-1] * (k + 1 - len(out))
