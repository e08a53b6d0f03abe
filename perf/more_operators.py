"""Cases of what a paged cache needs over a long run: attention over a prefix that several sequences share, the attention weight
that every cached entry draws, accumulated step by step, and the eviction of the entries that drew least.

Pages: K and V pools [n_pages, n_kv_heads, page_size, head_dim]; entry t of sequence b is row t % page_size of page
block_table[b][t // page_size].  In 8 bits (e4m3) the value of an entry is its code times a power of two that belongs to the
(page, KV head), K and V each with their own.

Prefix attention: a prefix is a row of a block table of its own.  Query token i of sequence b sees every entry of the prefix that
its group shares, and its own entries 0 .. lens[b] - (q_len - 1 - i) - 1.
Weights: [batch, n_kv_heads, stride]; an entry's weight becomes decay * weight + sum of exp(logit - lse) over the query rows of its
KV group that see it; the last q_len entries are the query tokens' own and start from zero.
Eviction: a sequence of more than `limit` entries keeps, for every KV head, the last `window` and the keep - window others of
largest weight (ties: the lowest slot).  Kept ones in slots below keep - window stay where they are, the others fill the freed
slots there in ascending order, the window follows in order.  An 8-bit page that receives entries takes the largest scale of
the pages its entries come from.
"""
import math

import torch

own = False          # set from outside: False computes the plain forms, True calls the library

E4M3_MAX = 448.0


# ---- cases ------------------------------------------------------------------------------------------------------------
def _prefix(name, **kw):
    c = dict(name=name, op="prefix", fmt="bf16", batch=8, groups=1, prefix=8192, shortest_prefix=0, length=256, shortest=64,
             q_len=1, page=64, hq=32, hkv=8, d=128)
    c.update(kw)
    return c


def _weights(name, **kw):
    c = dict(name=name, op="weights", fmt="bf16", batch=1, length=1024, shortest=0, q_len=1, page=64, hq=32, hkv=8, d=128,
             decay=1.0)
    c.update(kw)
    return c


def _evict(name, **kw):
    c = dict(name=name, op="evict", fmt="bf16", batch=1, length=2304, shortest=0, keep=2048, limit=2303, window=64, page=64,
             hkv=8, d=128)
    c.update(kw)
    return c


def listed():
    return [
        # two requests behind a short instruction, one small head (the smallest call)
        _prefix("prefix_2x512_bf16", batch=2, prefix=512, length=40, shortest=1, hq=4, hkv=1, d=64, page=16),
        # a full batch of requests about the same document
        _prefix("prefix_64x32768_bf16", batch=64, prefix=32768, length=512, shortest=64),
        # requests behind a system prompt, 8-bit pages
        _prefix("prefix_32x8192_e4m3", fmt="e4m3", batch=32, prefix=8192, length=384, shortest=16, page=128),
        # eight answers sampled for one 128K prompt
        _prefix("prefix_8x131072_e4m3", fmt="e4m3", prefix=131072, length=257, shortest=257, page=32),
        # four prompts of different lengths with a dozen requests each, four drafted tokens checked at once
        _prefix("prefix_4groups48_q4_bf16", batch=48, groups=4, prefix=11000, shortest_prefix=1500, length=700, shortest=5, q_len=4),
        # a short cache of one small head
        _weights("weights_1x257_bf16", length=257, hq=4, hkv=1, d=64, page=32),
        # a full batch of compressed requests, 16 bits, with forgetting
        _weights("weights_64x2048_bf16", batch=64, length=2048, shortest=1638, decay=0.98),
        # drafted tokens over requests of very different lengths, 8 bits
        _weights("weights_ragged16_q4_e4m3", fmt="e4m3", batch=16, length=40000, shortest=500, q_len=4),
        # one request's cache ran over its limit: 256 entries go
        _evict("evict_1x2304_bf16"),
        # the same for a whole batch, 8 bits, some of which are below the limit
        _evict("evict_64x2304_e4m3", fmt="e4m3", batch=64, shortest=2100, limit=2200, page=32),
        # an uncompressed 128K request is cut to 10 %
        _evict("evict_1x131072_bf16", length=131072, keep=13107, limit=13107, window=8),
        # four requests lose half, a long window of recent tokens stays
        _evict("evict_4x26214_e4m3", fmt="e4m3", batch=4, length=26214, shortest=20001, keep=13107, limit=20000, window=1024),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8, 8])
    page = rng.choice([16, 32, 64, 128])
    fmt = rng.choice(["bf16", "e4m3"])
    kind = rng.choice(["prefix", "weights", "evict"])
    if kind == "prefix":
        g = rng.choice([1, 3, 4, 4, 7, 8])
        c = _prefix("", fmt=fmt, page=page, hq=hkv * g, hkv=hkv, d=d, batch=_log_int(rng, 2, 64), q_len=rng.choice([1, 1, 1, 2, 4, 5]))
        c["groups"] = rng.choice([1, 1, 1, min(2, c["batch"]), min(5, c["batch"])])
        # entries of all prefixes together, by what is read and by what is computed
        read = 131072 * 8 // hkv // (1 if fmt == "e4m3" else 2) // c["groups"]
        rows = c["batch"] * c["q_len"] * c["hq"] // c["groups"]
        most = min(120000, read * 7 // 8, 60 * 32 * 32768 // (rows * c["groups"]))
        c["prefix"] = _log_int(rng, min(64, most), most)
        c["shortest_prefix"] = rng.choice([0, c["prefix"] // 4])
        c["length"] = _log_int(rng, 1, max(2, min(1000, 32768 // c["batch"])))
        c["shortest"] = rng.choice([0, 1, max(1, c["length"] // 4)])
    elif kind == "weights":
        g = rng.choice([1, 3, 4, 4, 7, 8])
        c = _weights("", fmt=fmt, page=page, hq=hkv * g, hkv=hkv, d=d, batch=_log_int(rng, 1, 64), q_len=rng.choice([1, 1, 1, 2, 4, 5]),
                     decay=rng.choice([1.0, 1.0, 0.9, 0.5]))
        cap = 131072 * 8 // (c["batch"] * hkv) // (2 if c["q_len"] > 1 else 1)
        c["length"] = _log_int(rng, 8, max(9, min(65536, cap)))
        c["shortest"] = rng.choice([0, 0, max(8, c["length"] // 8)])
    else:
        c = _evict("", fmt=fmt, page=page, hkv=hkv, d=d, batch=_log_int(rng, 1, 64))
        c["length"] = _log_int(rng, 64, max(65, min(131072, 131072 * 8 // (c["batch"] * hkv))))
        half, share, window, above = rng.random() < 0.5, rng.uniform(0.1, 0.98), rng.choice(["0", "1", "8", "1/16", "1/3", "all"]), rng.random() < 0.5
        while True:
            n = c["length"]
            keep = max(8, int(n * share))
            c.update(shortest=n // 2 if half else 0, keep=keep, limit=(keep + n) // 2 if above else keep,
                     window={"0": 0, "1": 1, "8": 8, "1/16": keep // 16, "1/3": keep // 3, "all": keep}[window])
            if work(c)["bytes"] <= 1.1e8:
                break
            c["length"] = max(64, n * 2 // 3)
    c.pop("name")
    return c


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _ints(g, lo, hi, shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda")


def _pool(g, c, n_pages):
    shape = (n_pages, c["hkv"], c["page"], c["d"])
    if c["fmt"] == "bf16":
        return _normal(g, shape), _normal(g, shape), None, None
    code = lambda: (torch.randn(shape, generator=g, device="cuda") * 100.0).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)  # noqa: E731
    scale = lambda: torch.exp2(_ints(g, -7, -5, shape[:2]).float())  # noqa: E731
    return code(), code(), scale(), scale()


def _tables(g, c, *lens):
    """A block table for each list of lengths, pages dealt out at random; some pages of the pool belong to nobody.  The last list
    is the sequences' own: the pool has room for the longest each of them may be, so that its size is the case's alone."""
    per_of = [[-(-n // c["page"]) for n in x] for x in lens]
    n_pages = sum(map(sum, per_of[:-1])) + c["batch"] * -(-c["length"] // c["page"]) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    tables, at = [], 0
    for need in per_of:
        table = torch.zeros((len(need), max(1, max(need))), dtype=torch.int32, device="cuda")
        for b, k in enumerate(need):
            table[b, :k] = order[at:at + k]
            at += k
        tables.append(table)
    return tables, n_pages


def _lengths(g, c):
    low = c["shortest"] or c["length"]
    lens = [int(x) for x in _ints(g, low, c["length"], (c["batch"],)).tolist()]
    lens[0] = c["length"]
    return lens


def _prefix_lengths(c):
    """Evenly from `prefix` down to `shortest_prefix`."""
    n, low = c["groups"], c["shortest_prefix"] or c["prefix"]
    return [c["prefix"] - (c["prefix"] - low) * i // max(1, n - 1) for i in range(n)]


def _cu_seqs(c):
    """Sequences of the groups: as even as it goes."""
    return [c["batch"] * i // c["groups"] for i in range(c["groups"] + 1)]


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = {"case": c}
    B = c["batch"]
    if c["op"] == "prefix":
        plens, lens = _prefix_lengths(c), _lengths(g, c)
        (s["ptable"], s["table"]), n_pages = _tables(g, c, plens, lens)
        s["cu"], s["plens_host"] = _cu_seqs(c), plens
        s["plens"] = torch.tensor(plens, dtype=torch.int32, device="cuda")
        s["cu_seqs"] = torch.tensor(s["cu"], dtype=torch.int32, device="cuda")
    else:
        lens = _lengths(g, c)
        (s["table"],), n_pages = _tables(g, c, lens)
    s["lens_host"] = lens
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"] = _pool(g, c, n_pages)
    stride = -(-c["length"] // 4) * 4
    if c["op"] != "evict":
        s["q"] = _normal(g, (B, c["q_len"], c["hq"], c["d"]))
    if c["op"] == "weights":
        s["lse"] = _lse(s)
        # what earlier steps left: most entries drew little
        s["weights"] = torch.randn((B, c["hkv"], stride), generator=g, device="cuda").mul_(1.5).exp_().mul_(0.01)
    if c["op"] == "evict":
        w = torch.randn((B, c["hkv"], stride), generator=g, device="cuda").mul_(1.5).exp_().mul_(0.01)
        # entries that never drew anything tie
        s["weights"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.02, torch.zeros_like(w), w)
        s["ids"] = torch.arange(stride, dtype=torch.int32, device="cuda").expand(B, c["hkv"], stride).contiguous()
        s["new_weights"], s["new_ids"] = torch.zeros_like(s["weights"]), torch.zeros_like(s["ids"])
        s["new_lens"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    if own:
        from paper_2502_01068_b200 import binding as F
        s["cache"] = F.make_paged_cache(s["k_pages"], s["v_pages"], s["table"], s["k_scales"], s["v_scales"])
        if c["op"] != "evict":
            s["query"] = F.make_query(n_q_heads=c["hq"], q_len=c["q_len"], max_len=max(lens), total_len=sum(lens))
        size = 256
        if c["op"] == "prefix":
            s["prefix"] = F.make_prefix(s["ptable"], s["plens"], max_len=max(plens), cu_seqs=s["cu_seqs"] if c["groups"] > 1 else None)
            s["out"] = torch.empty((B, c["q_len"], c["hq"], c["d"]), dtype=torch.bfloat16, device="cuda")
            s["lse"] = torch.empty((B, c["q_len"], c["hq"]), dtype=torch.float32, device="cuda")
            size = F.fastkv_prefix_attn_workspace_bytes(s["cache"], s["prefix"], s["query"])
        elif c["op"] == "evict":
            s["eviction"] = F.make_eviction(keep=c["keep"], limit=c["limit"], window=c["window"], max_len=max(lens))
            size = F.fastkv_paged_evict_workspace_bytes(s["cache"], s["eviction"])
        s["ws"] = torch.zeros(size, dtype=torch.uint8, device="cuda")
    return s


def _entries(pages, scales, table_row, n):
    """Entries 0 .. n - 1 of a block-table row in 32 bits: [n_kv_heads, n, d]."""
    P = pages.shape[2]
    ids = table_row[: -(-n // P)].long()
    x = pages[ids].float()
    if scales is not None:
        x = x * scales[ids][..., None, None]
    return x.transpose(0, 1).reshape(pages.shape[1], -1, pages.shape[3])[:, :n]


def _seen(n, q_len, device):
    """[q_len, n]: which of n own entries each query token sees."""
    t = torch.arange(n, device=device)
    return t[None, :] < (n - (q_len - 1 - torch.arange(q_len, device=device)))[:, None]


def _logits(s, b, k):
    """[n_kv_heads, q_len * group, n] over the entries k of sequence b, unmasked."""
    c = s["case"]
    q = s["q"][b].float().reshape(c["q_len"], c["hkv"], -1, c["d"]).transpose(0, 1).reshape(c["hkv"], -1, c["d"])
    return (q @ k.transpose(-1, -2)) * (1.0 / math.sqrt(c["d"]))


def _lse(s):
    """The log-sum-exp that the attention over the same cache hands out: fp32 [batch, q_len, n_q_heads]."""
    c = s["case"]
    T, G = c["q_len"], c["hq"] // c["hkv"]
    out = []
    for b, n in enumerate(s["lens_host"]):
        x = _logits(s, b, _entries(s["k_pages"], s["k_scales"], s["table"][b], n))
        x = x.reshape(c["hkv"], T, G, n).masked_fill(~_seen(n, T, x.device)[None, :, None, :], -math.inf)
        out.append(torch.logsumexp(x, dim=-1).transpose(0, 1).reshape(T, c["hq"]))
    return torch.stack(out)


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _part(logits, v):
    """Largest logit, sum of exponentials and weighted values of one stretch of entries."""
    if logits.shape[-1] == 0:
        shape = logits.shape[:-1]
        return logits.new_full(shape + (1,), -math.inf), logits.new_zeros(shape + (1,)), logits.new_zeros(shape + (v.shape[-1],))
    top = logits.amax(dim=-1, keepdim=True)
    p = torch.exp(logits - torch.where(top == -math.inf, torch.zeros_like(top), top))
    return top, p.sum(dim=-1, keepdim=True), p @ v


def _plain_prefix(s):
    c = s["case"]
    T, Hkv, d = c["q_len"], c["hkv"], c["d"]
    G = c["hq"] // Hkv
    outs, lses = [], []
    for i in range(c["groups"]):
        lo, hi = s["cu"][i], s["cu"][i + 1]
        if lo == hi:
            continue
        n = s["plens_host"][i]
        pk = _entries(s["k_pages"], s["k_scales"], s["ptable"][i], n)
        pv = _entries(s["v_pages"], s["v_scales"], s["ptable"][i], n)
        q = s["q"][lo:hi].float().reshape(hi - lo, T, Hkv, G, d).permute(2, 0, 1, 3, 4).reshape(Hkv, -1, d)
        pm, pl, po = _part((q @ pk.transpose(-1, -2)) * (1.0 / math.sqrt(d)), pv)
        apart = lambda x: x.reshape(Hkv, hi - lo, T * G, -1)  # noqa: E731
        pm, pl, po = apart(pm), apart(pl), apart(po)
        for b in range(lo, hi):
            m = s["lens_host"][b]
            k = _entries(s["k_pages"], s["k_scales"], s["table"][b], m)
            v = _entries(s["v_pages"], s["v_scales"], s["table"][b], m)
            x = _logits(s, b, k).reshape(Hkv, T, G, m).masked_fill(~_seen(m, T, k.device)[None, :, None, :], -math.inf)
            om, ol, oo = _part(x.reshape(Hkv, T * G, m), v)
            top = torch.maximum(pm[:, b - lo], om)
            a, e = torch.exp(pm[:, b - lo] - top), torch.exp(om - top)
            total = pl[:, b - lo] * a + ol * e
            back = lambda x: x.reshape(Hkv, T, G, -1).transpose(0, 1).reshape(T, c["hq"], -1)  # noqa: E731
            outs.append(back((po[:, b - lo] * a + oo * e) / total))
            lses.append(back(top + total.log())[..., 0])
    return {"out": torch.stack(outs).to(torch.bfloat16), "lse": torch.stack(lses)}


def _plain_weights(s):
    c = s["case"]
    T, G = c["q_len"], c["hq"] // c["hkv"]
    w = s["weights"]
    for b, n in enumerate(s["lens_host"]):
        x = _logits(s, b, _entries(s["k_pages"], s["k_scales"], s["table"][b], n)).reshape(c["hkv"], T, G, n)
        lse = s["lse"][b].reshape(T, c["hkv"], G).transpose(0, 1)[..., None]
        p = torch.exp(x - lse) * _seen(n, T, x.device)[None, :, None, :]
        drew = p.sum(dim=(1, 2))
        old = max(0, n - T)
        w[b, :, :old] = c["decay"] * w[b, :, :old] + drew[:, :old]
        w[b, :, old:n] = drew[:, old:]
    return {"weights": w}


def _origins(w, n, keep, window):
    """w [heads, n] -> [heads, keep]: the slot that each kept slot's entry comes from."""
    H, m, cand = w.shape[0], keep - window, n - window
    dev = w.device
    kept = torch.zeros((H, cand), dtype=torch.bool, device=dev)
    best = torch.sort(w[:, :cand], dim=1, descending=True, stable=True).indices[:, :m]
    kept.scatter_(1, best, True)
    slot = torch.arange(cand, device=dev).expand(H, cand)
    movers = torch.where(kept & (slot >= m), slot, torch.full_like(slot, cand)).sort(dim=1).values
    free = ~kept[:, :m]
    nth = (free.cumsum(dim=1) - 1).clamp(min=0)
    origin = torch.where(free, torch.gather(movers, 1, nth), slot[:, :m]) if m else slot[:, :0]
    return torch.cat([origin, torch.arange(cand, n, device=dev).expand(H, window)], dim=1)


def _move(pages, scales, table_row, origin):
    """Slot j of every head takes the entry of slot origin[head, j]; in 8 bits in the largest scale of the page's entries."""
    H, keep = origin.shape
    P, dev = pages.shape[2], origin.device
    heads = torch.arange(H, device=dev)[:, None]
    table = table_row.long()
    from_page, to = table[origin // P], torch.arange(keep, device=dev)
    rows = pages.view(torch.uint8)[from_page, heads, origin % P] if scales is not None else pages[from_page, heads, origin % P]
    to_page = table[to // P]
    if scales is not None:
        was = scales[from_page, heads]                                        # [heads, keep]
        n = -(-keep // P)
        padded = torch.zeros((H, n * P), device=dev)
        padded[:, :keep] = was
        new = padded.reshape(H, n, P).amax(dim=2)
        by = was / new.repeat_interleave(P, dim=1)[:, :keep]
        again = (rows.view(torch.float8_e4m3fn).float() * by[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
        pages.view(torch.uint8)[to_page[None], heads, (to % P)[None]] = again
        scales[table[:n][None], heads] = new
    else:
        pages[to_page[None], heads, (to % P)[None]] = rows


def _plain_evict(s):
    c = s["case"]
    for b, n in enumerate(s["lens_host"]):
        if n <= c["limit"]:
            s["new_weights"][b, :, :n], s["new_ids"][b, :, :n] = s["weights"][b, :, :n], s["ids"][b, :, :n]
            s["new_lens"][b] = n
            continue
        origin = _origins(s["weights"][b, :, :n], n, c["keep"], c["window"])
        _move(s["k_pages"], s["k_scales"], s["table"][b], origin)
        _move(s["v_pages"], s["v_scales"], s["table"][b], origin)
        s["new_weights"][b, :, : c["keep"]] = torch.gather(s["weights"][b], 1, origin)
        s["new_ids"][b, :, : c["keep"]] = torch.gather(s["ids"][b], 1, origin)
        s["new_lens"][b] = c["keep"]
    return _evicted(s)


def _evicted(s):
    out = {n: s[n] for n in ("k_pages", "v_pages", "new_weights", "new_ids", "new_lens")}
    if s["k_scales"] is not None:
        out["k_scales"], out["v_scales"] = s["k_scales"], s["v_scales"]
    return out


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"prefix": _plain_prefix, "weights": _plain_weights, "evict": _plain_evict}[c["op"]](s)
    from paper_2502_01068_b200 import binding as F
    if c["op"] == "prefix":
        F.fastkv_prefix_attn(s["cache"], s["prefix"], s["query"], s["lens"], s["q"], s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "weights":
        F.fastkv_paged_weights(s["cache"], s["query"], s["lens"], s["q"], s["lse"], c["decay"], s["weights"], s["ws"])
        return {"weights": s["weights"]}
    F.fastkv_paged_evict(s["cache"], s["eviction"], s["lens"], s["weights"], s["ids"], s["new_weights"], s["new_ids"], s["new_lens"],
                         s["ws"])
    return _evicted(s)


# ---- the same from the definition, in 64 bits ----------------------------------------------------------------------------
def _slots(s, name, table_row, head, n):
    """Values of entries 0 .. n - 1 of one KV head, [n, d] in 64 bits."""
    pages, scales = s[name + "_pages"], s[name + "_scales"]
    t = torch.arange(n, device="cuda")
    page = table_row.long()[t // pages.shape[2]]
    x = pages[page, head, t % pages.shape[2]].double()
    return x if scales is None else x * scales[page, head].double()[:, None]


def _exact_prefix(s):
    c = s["case"]
    T, Hkv, d = c["q_len"], c["hkv"], c["d"]
    G = c["hq"] // Hkv
    out = torch.zeros((c["batch"], T, c["hq"], d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((c["batch"], T, c["hq"]), dtype=torch.float64, device="cuda")
    for i in range(c["groups"]):
        n = s["plens_host"][i]
        for h in range(Hkv):
            pk, pv = (_slots(s, x, s["ptable"][i], h, n) for x in "kv")
            for b in range(s["cu"][i], s["cu"][i + 1]):
                m = s["lens_host"][b]
                k, v = (torch.cat([p, _slots(s, x, s["table"][b], h, m)]) for x, p in (("k", pk), ("v", pv)))
                for t in range(T):
                    sees = n + max(0, m - (T - 1 - t))
                    x = s["q"][b, t, h * G:(h + 1) * G].double() @ k[:sees].t() / math.sqrt(d)
                    lse[b, t, h * G:(h + 1) * G] = torch.logsumexp(x, dim=-1)
                    out[b, t, h * G:(h + 1) * G] = torch.softmax(x, dim=-1) @ v[:sees]
    return {"out": out, "lse": lse}


def _exact_weights(s):
    c = s["case"]
    T, Hkv = c["q_len"], c["hkv"]
    G = c["hq"] // Hkv
    w = s["weights"].double()
    for b, n in enumerate(s["lens_host"]):
        for h in range(Hkv):
            k = _slots(s, "k", s["table"][b], h, n)
            total = torch.zeros(n, dtype=torch.float64, device="cuda")
            for t in range(T):
                sees = max(0, n - (T - 1 - t))
                x = s["q"][b, t, h * G:(h + 1) * G].double() @ k[:sees].t() / math.sqrt(c["d"])
                total[:sees] += torch.exp(x - s["lse"][b, t, h * G:(h + 1) * G].double()[:, None]).sum(dim=0)
            first = max(0, n - T)
            total[:first] += float(torch.tensor(c["decay"], dtype=torch.float32)) * w[b, h, :first]
            w[b, h, :n] = total
    return {"weights": w}


def _exact_code(x):
    """x to the nearest e4m3 value, ties to even: 3 bits behind the leading one, steps of 2^-9 below 2^-6."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)
    return (torch.round(x / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_evict(s):
    c = s["case"]
    P = c["page"]
    old = {x: s[x + "_pages"].double() for x in "kv"}
    new = {x: old[x].clone() for x in "kv"}
    was = {x: None if s[x + "_scales"] is None else s[x + "_scales"].double() for x in "kv"}
    now = {x: None if was[x] is None else was[x].clone() for x in "kv"}
    weights, ids, lens = s["new_weights"].double(), s["new_ids"].clone(), []
    for b, n in enumerate(s["lens_host"]):
        lens.append(min(n, c["keep"]) if n > c["limit"] else n)
        for h in range(c["hkv"]):
            w = s["weights"][b, h, :n].double().tolist()
            order = list(range(n))
            if n > c["limit"]:
                m, cand = c["keep"] - c["window"], n - c["window"]
                best = set(sorted(range(cand), key=lambda t: (-w[t], t))[:m])
                movers = iter([t for t in range(m, cand) if t in best])
                order = [t if t in best else next(movers) for t in range(m)] + list(range(cand, n))
            at = torch.tensor(order, device="cuda", dtype=torch.long)
            weights[b, h, : len(order)] = s["weights"][b, h].double()[at]
            ids[b, h, : len(order)] = s["ids"][b, h][at]
            if n <= c["limit"]:
                continue
            table = s["table"][b].long()
            j = torch.arange(len(order), device="cuda")
            for x in "kv":
                rows = old[x][table[at // P], h, at % P]
                if was[x] is not None:
                    from_ = was[x][table[at // P], h]
                    top = torch.zeros(-(-len(order) // P), dtype=torch.float64, device="cuda").scatter_reduce_(0, j // P, from_, "amax")
                    now[x][table[: top.shape[0]], h] = top
                    rows = _exact_code(rows * (from_ / top[j // P])[:, None])
                new[x][table[j // P], h, j % P] = rows
    out = {"k_pages": new["k"], "v_pages": new["v"], "new_weights": weights, "new_ids": ids,
           "new_lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    if was["k"] is not None:
        out["k_scales"], out["v_scales"] = now["k"], now["v"]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"prefix": _exact_prefix, "weights": _exact_weights, "evict": _exact_evict}[case["op"]](s)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    c = case
    item = 2 if c["fmt"] == "bf16" else 1
    low = c["shortest"] or c["length"]
    entries = c["length"] + (c["batch"] - 1) * (low + c["length"]) / 2
    row = c["hkv"] * c["d"] * item                                          # a K (or V) row of all KV heads
    scales = lambda n: n / c["page"] * c["hkv"] * 4 if item == 1 else 0  # noqa: E731
    if c["op"] == "prefix":
        plens, cu = _prefix_lengths(c), _cu_seqs(c)
        shared = sum(plens)
        queries = c["batch"] * c["q_len"] * c["hq"]
        moved = 2 * ((shared + entries) * row + scales(shared + entries)) + queries * (4 * c["d"] + 4)
        pairs = sum(n * (cu[i + 1] - cu[i]) for i, n in enumerate(plens)) + entries
        return {"bytes": moved, "flops": 4.0 * pairs * c["q_len"] * c["hq"] * c["d"]}
    if c["op"] == "weights":
        moved = entries * (row + 8 * c["hkv"]) + scales(entries) + c["batch"] * c["q_len"] * c["hq"] * (2 * c["d"] + 4)
        return {"bytes": moved, "flops": 2.0 * entries * c["q_len"] * c["hq"] * c["d"]}
    moved = flops = 0.0
    for i in range(c["batch"]):
        n = c["length"] - (c["length"] - low) * i / max(1, c["batch"] - 1)
        if n <= c["limit"]:
            moved += n * c["hkv"] * 16                                       # weights and ids go through
            continue
        cand, m = n - c["window"], c["keep"] - c["window"]
        rows = m * (cand - m) / cand + c["window"]                           # as many as chance moves, and the window
        moved += 4 * rows * row + 4 * scales(rows) + c["hkv"] * (4 * cand + 12 * c["keep"])
        flops += cand * c["hkv"]
    return {"bytes": moved, "flops": flops}
