"""Plain 64-bit reference of the paged cache (appending rows, attention) and builders of its inputs, for the tests."""
import math

import numpy as np
import torch

E4M3_MAX = 448.0


def rn_e4m3(x):
    """float64 array to the nearest e4m3 value, ties to even, saturating: three bits behind the leading one, steps of 2^-9
    below 2^-6."""
    x = np.asarray(x, dtype=np.float64)
    _, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.clip(np.round(x / step) * step, -E4M3_MAX, E4M3_MAX)


def need_scale(m):
    """The smallest power of two 2^e, e in -64 .. 120, with 448 * 2^e >= m (float)."""
    e = -64
    while e < 120 and math.ldexp(E4M3_MAX, e) < m:
        e += 1
    return math.ldexp(1.0, e)


def rotate(x, pos, inv_freq, rot, adjacent):
    """x [rows, heads, d] float64, pos [rows], inv_freq float32 [rot / 2]."""
    x = np.array(x, dtype=np.float64)
    if rot == 0:
        return x
    a = np.outer(np.asarray(pos, dtype=np.float64), np.asarray(inv_freq, dtype=np.float64))[:, None, :]
    i = np.arange(rot // 2)
    lo, hi = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
    x1, x2 = x[..., lo].copy(), x[..., hi].copy()
    x[..., lo] = x1 * np.cos(a) - x2 * np.sin(a)
    x[..., hi] = x2 * np.cos(a) + x1 * np.sin(a)
    return x


def attention(q, k, v, sees, scale):
    """q [Hq, d], k / v [n, Hkv, d] float64, over the first `sees` entries.  Returns out [Hq, d], lse [Hq], and what the
    error bounds need: sum_t p |v| [Hq, d] and max_t scale * sum |q k| [Hq]."""
    Hq, d = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    out, lse = np.zeros((Hq, d)), np.full(Hq, -np.inf)
    mass, size = np.zeros((Hq, d)), np.zeros(Hq)
    if sees <= 0:
        return out, lse, mass, size
    for h in range(Hq):
        kk, vv = k[:sees, h // G], v[:sees, h // G]
        x = scale * (kk @ q[h])
        m = x.max()
        p = np.exp(x - m)
        L = p.sum()
        out[h], lse[h] = (p / L) @ vv, m + math.log(L)
        mass[h], size[h] = (p / L) @ np.abs(vv), scale * (np.abs(kk) @ np.abs(q[h])).max()
    return out, lse, mass, size


class Pools:
    """A paged cache on the GPU with its contents mirrored in float64: every sequence's entries, pages dealt out at random,
    and poison (NaN) in every entry, page and scale that belongs to nobody."""

    def __init__(self, fmt, lens, room, page, Hkv, d, seed, v_exp=(-7, -4), spare=3):
        rng = np.random.default_rng(seed)
        self.fmt, self.page, self.Hkv, self.d = fmt, page, Hkv, d
        self.lens = list(lens)
        per = max(1, -(-max(max(room), 1) // page))
        need = [-(-max(r, 0) // page) for r in room]
        self.n_pages = sum(need) + spare
        order = rng.permutation(self.n_pages)
        table = np.full((len(lens), per), -1, dtype=np.int32)        # entries beyond a sequence's pages name no page
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.table_np = table
        shape = (self.n_pages, Hkv, page, d)
        if fmt == "bf16":
            self.k = torch.full(shape, float("nan"), dtype=torch.bfloat16)
            self.v = torch.full(shape, float("nan"), dtype=torch.bfloat16)
            self.ks = self.vs = None
        else:
            self.k = torch.full(shape, 0x7F, dtype=torch.uint8)
            self.v = torch.full(shape, 0x7F, dtype=torch.uint8)
            self.ks = torch.full(shape[:2], float("nan"))
            self.vs = torch.full(shape[:2], float("nan"))
        self.k64, self.v64 = [], []                                   # [len, Hkv, d] float64: what the entries stand for
        for b, n in enumerate(lens):
            both = []
            for name in ("k", "v"):
                pool, scales = getattr(self, name), getattr(self, name + "s")
                x = torch.from_numpy(rng.standard_normal((n, Hkv, d)))
                vals = torch.zeros_like(x)
                for p0 in range(0, n, page):
                    pid, m = int(table[b, p0 // page]), min(page, n - p0)
                    if fmt == "bf16":
                        y = x[p0:p0 + m].to(torch.bfloat16)
                        pool[pid, :, :m] = y.transpose(0, 1)
                        vals[p0:p0 + m] = y.double()
                    else:
                        lo, hi = (-7, -4) if name == "k" else v_exp
                        s = torch.exp2(torch.from_numpy(rng.integers(lo, hi + 1, Hkv)).double())
                        code = (x[p0:p0 + m] * 100.0).clamp(-448, 448).float().to(torch.float8_e4m3fn)
                        pool[pid, :, :m] = code.view(torch.uint8).transpose(0, 1)
                        scales[pid] = s.float()
                        vals[p0:p0 + m] = code.float().double() * s[None, :, None]
                both.append(vals.numpy())
            self.k64.append(both[0])
            self.v64.append(both[1])
        for name in ("k", "v", "ks", "vs"):
            t = getattr(self, name)
            setattr(self, name, None if t is None else t.cuda())
        self.table = torch.from_numpy(table).cuda()
        self.dev_lens = torch.tensor(self.lens, dtype=torch.int32, device="cuda")

    def cache(self):
        from paper_2502_01068_b200 import binding as B
        return B.make_paged_cache(self.k, self.v, self.table, self.ks, self.vs)

    def read(self, b, n):
        """Entries 0 .. n - 1 of sequence b as the pools hold them now: (k, v) [n, Hkv, d] float64."""
        got = []
        for pool, scales in ((self.k, self.ks), (self.v, self.vs)):
            x = (pool if self.fmt == "bf16" else pool.view(torch.float8_e4m3fn)).cpu()
            rows = []
            for p0 in range(0, n, self.page):
                pid, m = int(self.table_np[b, p0 // self.page]), min(self.page, n - p0)
                y = x[pid, :, :m].float().double()
                if scales is not None:
                    y = y * scales[pid].cpu().double()[:, None, None]
                rows.append(y.transpose(0, 1))
            got.append(torch.cat(rows).numpy() if rows else np.zeros((0, self.Hkv, self.d)))
        return got
