"""Cases of the paged-cache operators: appending keys and values (with the position rotation applied on the way, or
gathered by the selection's indices) to pages held in bf16 or in 8 bits, and the attention of new tokens over those pages.

Pages: K and V pools [n_pages, n_kv_heads, page_size, head_dim]; entry t of sequence b is row t % page_size of page
block_table[b][t // page_size].  In 8 bits (e4m3) the value of an entry is its code times a power of two that belongs to
the (page, KV head), K and V each with their own.
"""
import math

import torch

own = False          # set from outside: False computes the plain forms, True calls the library

E4M3_MAX = 448.0
SCALE_MIN_EXP, SCALE_MAX_EXP = -64, 120


# ---- cases ------------------------------------------------------------------------------------------------------------
def _append(name, **kw):
    c = dict(name=name, op="append", fmt="bf16", batch=1, new=1, ragged=False, cached=0, page=64, hq=32, hkv=8, d=128,
             rot=128, adjacent=False, source=0)
    c.update(kw)
    return c


def _attn(name, **kw):
    c = dict(name=name, op="attn", fmt="e4m3", batch=1, length=1024, shortest=0, q_len=1, page=64, hq=32, hkv=8, d=128)
    c.update(kw)
    return c


def listed():
    return [
        # one request's next token goes behind its kept entries (the smallest call of a decode step)
        _append("append_1x1_bf16", cached=13107),
        # a decode step of a full batch into an 8-bit cache, sequences of different lengths
        _append("append_64x1_e4m3", fmt="e4m3", batch=64, cached=1024),
        # a chunk of a prompt, behind the tokens that are there already
        _append("append_8192_bf16", new=8192, cached=1638),
        # the rows that the selection kept of a 128K prompt go into 8-bit pages
        _append("append_kept_13107_e4m3", fmt="e4m3", new=13107, source=131072, rot=0, hq=0),
        # prompts of different lengths in one call, 8-bit pages of 128 entries
        _append("append_ragged8_e4m3", fmt="e4m3", batch=8, new=8192, ragged=True, cached=300, page=128),
        # a short cache of one small head (the smallest attention call)
        _attn("attn_1x257_e4m3", length=257, hq=4, hkv=1, d=64, page=32),
        # one request's next token over 10 % of a 128K prompt
        _attn("attn_1x13107_e4m3", length=13107),
        # the same over the 20 % budget in 16 bits
        _attn("attn_1x26214_bf16", fmt="bf16", length=26214, page=16),
        # a batch of uncompressed requests of very different lengths
        _attn("attn_ragged8_e4m3", batch=8, length=65536, shortest=4096),
        # a full batch of compressed requests, 16 bits
        _attn("attn_64x2048_bf16", fmt="bf16", batch=64, length=2048, shortest=1638),
        # four drafted tokens per request are checked at once
        _attn("attn_32x1638_q4_e4m3", batch=32, length=1638, shortest=819, q_len=4, page=128),
        # one uncompressed 128K request
        _attn("attn_1x131072_e4m3", length=131072),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8, 8])
    page = rng.choice([16, 32, 64, 128])
    fmt = rng.choice(["bf16", "e4m3"])
    if rng.random() < 0.5:
        g = rng.choice([1, 2, 4, 4, 8])
        c = _append("", fmt=fmt, page=page, hq=hkv * g, hkv=hkv, d=d, cached=rng.choice([0, _log_int(rng, 1, 8192)]),
                    rot=rng.choice([d, d, d // 2]), adjacent=rng.random() < 0.3)
        kind = rng.random()
        if kind < 0.4:                               # a decode step: one to a few new tokens per sequence
            c.update(batch=_log_int(rng, 1, 128), new=rng.choice([1, 1, 1, 2, 5]), cached=_log_int(rng, 1, 1024))
        elif kind < 0.8:                             # prompts, or chunks of them
            c.update(batch=rng.choice([1, 1, 2, 5]), new=_log_int(rng, 9, 8192 * 4 // max(4, g)), ragged=rng.random() < 0.5)
        else:                                        # what the selection kept
            n = _log_int(rng, 16, 13107)
            c.update(new=n, source=min(131072, n * rng.choice([5, 10])), cached=0, rot=0, hq=0)
    else:
        g = rng.choice([1, 3, 4, 4, 7, 8])
        c = _attn("", fmt=fmt, page=page, hq=hkv * g, hkv=hkv, d=d, batch=_log_int(rng, 1, 64), q_len=rng.choice([1, 1, 1, 2, 3, 8]))
        cap = 400000 * 8 // (c["batch"] * hkv) // (1 if fmt == "e4m3" else 2) // (2 if c["q_len"] > 1 else 1)
        c["length"] = _log_int(rng, 1, max(2, min(131072, cap)))
        c["shortest"] = rng.choice([0, 0, c["length"] // 8])
    c.pop("name")
    return c


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _keys(g, shape):
    """Keys as models produce them: a few channels of every head are several times larger than the others."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    gain = torch.ones(shape[-2:], device="cuda")
    gain[:, :: max(1, shape[-1] // 4)] = 4.0
    return (x * gain).to(torch.bfloat16)


def _ints(g, lo, hi, shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda")


def _pool(g, c, n_pages):
    shape = (n_pages, c["hkv"], c["page"], c["d"])
    if c["fmt"] == "bf16":
        return _normal(g, shape), _normal(g, shape), None, None
    code = lambda: (torch.randn(shape, generator=g, device="cuda") * 100.0).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)  # noqa: E731
    scale = lambda: torch.exp2(_ints(g, -7, -5, shape[:2]).float())  # noqa: E731
    return code(), code(), scale(), scale()


def _table(g, c, lens):
    """Pages dealt out at random; some pages of the pool belong to nobody."""
    per = -(-max(lens) // c["page"])
    n_pages = sum(-(-n // c["page"]) for n in lens) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((c["batch"], per), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(lens):
        k = -(-n // c["page"])
        table[b, :k] = order[at:at + k]
        at += k
    return table, n_pages


def _new_lengths(c):
    """New rows per sequence; ragged: spread evenly from an eighth of `new` up to `new`."""
    B, n = c["batch"], c["new"]
    if not c["ragged"] or B == 1:
        return [n] * B
    return [max(1, n - (n - n // 8) * b // (B - 1)) for b in range(B)]


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = {"case": c}
    B = c["batch"]
    if c["op"] == "append":
        new = _new_lengths(c)
        cached = [int(x) for x in _ints(g, c["cached"] // 2, c["cached"], (B,)).tolist()]
        total = sum(new)
        s["new"], s["total"] = new, total
        # room for the longest that may be cached, so that the pools' size is the case's alone
        s["table"], n_pages = _table(g, c, [c["cached"] + n for n in new])
        s["lens"] = torch.tensor(cached, dtype=torch.int32, device="cuda")
        s["new_lens"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        s["cu_new"] = torch.tensor([sum(new[:i]) for i in range(B + 1)], dtype=torch.int32, device="cuda")
        s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"] = _pool(g, c, n_pages)
        rows = c["source"] or total
        s["k"], s["v"] = _keys(g, (rows, c["hkv"], c["d"])), _normal(g, (rows, c["hkv"], c["d"]))
        s["idx"] = None
        if c["source"]:
            pick = torch.rand((c["hkv"], c["source"]), generator=g, device="cuda").topk(total, dim=1).indices
            s["idx"] = pick.sort(dim=1).values.to(torch.int32)
        s["q"] = _normal(g, (total, c["hq"], c["d"])) if c["hq"] else None
        s["q_out"] = torch.zeros_like(s["q"]) if c["hq"] else None
        s["pos"] = s["inv_freq"] = None
        if c["rot"]:
            # the prompt was longer than what the cache kept of it, so positions run ahead of the slots
            first = _ints(g, 0, 120000, (B,)).tolist()
            s["pos"] = torch.cat([torch.arange(f, f + n, device="cuda") for f, n in zip(first, new)]).to(torch.int32)
            s["inv_freq"] = (500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])).float().cuda()
        if own:
            from paper_2502_01068_b200 import binding as F
            s["cache"] = F.make_paged_cache(s["k_pages"], s["v_pages"], s["table"], s["k_scales"], s["v_scales"])
            s["rows"] = F.make_new_rows(batch=B, total=total, max_new=max(new), cu_new=s["cu_new"] if c["ragged"] else None,
                                        n_q_heads=c["hq"], n_kv_heads=c["hkv"], head_dim=c["d"], rot_dim=c["rot"],
                                        rot_pairs=F.ROT_ADJACENT if c["adjacent"] else F.ROT_HALVES, total_src=c["source"])
            s["ws"] = torch.zeros(256, dtype=torch.uint8, device="cuda")
        return s
    low = c["shortest"] or c["length"]
    lens = [int(x) for x in _ints(g, low, c["length"], (B,)).tolist()]
    lens[0] = c["length"]
    s["table"], n_pages = _table(g, c, lens)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"] = _pool(g, c, n_pages)
    s["q"] = _normal(g, (B, c["q_len"], c["hq"], c["d"]))
    if own:
        from paper_2502_01068_b200 import binding as F
        s["cache"] = F.make_paged_cache(s["k_pages"], s["v_pages"], s["table"], s["k_scales"], s["v_scales"])
        s["query"] = F.make_query(n_q_heads=c["hq"], q_len=c["q_len"], max_len=max(lens), total_len=sum(lens))
        s["out"] = torch.empty((B, c["q_len"], c["hq"], c["d"]), dtype=torch.float32, device="cuda")
        s["lse"] = torch.empty((B, c["q_len"], c["hq"]), dtype=torch.float32, device="cuda")
        s["ws"] = torch.zeros(F.fastkv_paged_attn_workspace_bytes(s["cache"], s["query"]), dtype=torch.uint8, device="cuda")
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _rotate(x, pos, inv_freq, rot, adjacent):
    """x [rows, heads, d] in 32 bits; the angles of far positions need 64."""
    angle = pos.double()[:, None] * inv_freq.double()[None, :]
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    if adjacent:
        x1, x2 = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        x1, x2 = x[..., : rot // 2], x[..., rot // 2: rot]
    y1, y2 = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    y = torch.stack([y1, y2], dim=-1).flatten(-2) if adjacent else torch.cat([y1, y2], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _need(m):
    """The smallest 2^e with 448 * 2^e >= m, e within its range (m: largest absolute values, >= 0)."""
    frac, e = torch.frexp(m)                                      # m = frac * 2^e, frac in [0.5, 1)
    e = torch.where(frac > 0.875, e - 8, e - 9)                   # 448 = 0.875 * 2^9
    e = torch.where(m > 0, e, torch.full_like(e, SCALE_MIN_EXP)).clamp(SCALE_MIN_EXP, SCALE_MAX_EXP)
    return torch.ldexp(torch.ones_like(m), e)


def _write_pages_e4m3(pages, scales, rows, at_page, at_row, touched, where, old_rows):
    """rows [n, heads, d] go to row at_row of the touched page `where` says; old_rows [touched, page]: entries that stay."""
    T, H, P, d = touched.shape[0], pages.shape[1], pages.shape[2], pages.shape[3]
    top = torch.zeros((T, H), dtype=torch.float32, device=rows.device)
    top.scatter_reduce_(0, where[:, None].expand(-1, H), rows.abs().amax(dim=-1), "amax")
    before = scales[touched]
    scale = torch.where(old_rows.any(dim=1)[:, None], torch.maximum(before, _need(top)), _need(top))
    code = pages[touched].float()
    again = (code * (before / scale)[:, :, None, None]).clamp(-E4M3_MAX, E4M3_MAX)
    code = torch.where(old_rows[:, None, :, None], again, code).to(torch.float8_e4m3fn)
    # whole pages go back: byte by byte where an entry was neither there nor is new
    block = torch.where(old_rows[:, None, :, None], code.view(torch.uint8), pages[touched].view(torch.uint8))
    fresh = (rows / scale[where][:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    block[where, :, at_row] = fresh.view(torch.uint8)
    pages.view(torch.uint8)[touched] = block
    scales[touched] = scale


def _plain_append(s):
    c, dev = s["case"], s["lens"].device
    P, total, lens = c["page"], s["total"], s["lens"].long()
    counts = (s["cu_new"][1:] - s["cu_new"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(c["batch"], device=dev), counts, output_size=total)
    slot = lens[seq] + torch.arange(total, device=dev) - s["cu_new"].long()[seq]
    page = s["table"][seq, slot // P].long()
    row = slot % P
    if s["idx"] is not None:
        heads = torch.arange(c["hkv"], device=dev)[None, :]
        src = s["idx"].long().t()
        k, v = s["k"][src, heads].float(), s["v"][src, heads].float()
    else:
        k, v = s["k"].float(), s["v"].float()
    out = {}
    if c["rot"]:
        k = _rotate(k, s["pos"], s["inv_freq"], c["rot"], c["adjacent"])
    if s["q"] is not None:
        q = s["q"].float()
        q = _rotate(q, s["pos"], s["inv_freq"], c["rot"], c["adjacent"]) if c["rot"] else q
        out["q"] = q.to(torch.bfloat16)
    if c["fmt"] == "bf16":
        s["k_pages"][page, :, row] = k.to(torch.bfloat16)
        s["v_pages"][page, :, row] = v.to(torch.bfloat16)
    else:
        # pages that get a row, each once, and which of their entries were there before
        per = s["table"].shape[1]
        flat = torch.zeros(c["batch"] * per, dtype=torch.bool, device=dev)
        flat[seq * per + slot // P] = True
        slots = flat.nonzero()[:, 0]
        place = torch.zeros(c["batch"] * per, dtype=torch.long, device=dev)
        place[slots] = torch.arange(slots.shape[0], device=dev)
        where = place[seq * per + slot // P]
        touched = s["table"].reshape(-1)[slots].long()
        first = (slots % per) * P
        old_rows = first[:, None] + torch.arange(P, device=dev)[None, :] < lens[slots // per][:, None]
        _write_pages_e4m3(s["k_pages"], s["k_scales"], k, page, row, touched, where, old_rows)
        _write_pages_e4m3(s["v_pages"], s["v_scales"], v, page, row, touched, where, old_rows)
        out["k_scales"], out["v_scales"] = s["k_scales"], s["v_scales"]
    out["k_pages"], out["v_pages"] = s["k_pages"], s["v_pages"]
    out["lens"] = s["lens"] + counts.int()
    return out


def _plain_attn(s):
    c = s["case"]
    B, T, Hq, Hkv, d, P = c["batch"], c["q_len"], c["hq"], c["hkv"], c["d"], c["page"]
    G, S, dev = Hq // Hkv, s["table"].shape[1] * c["page"], s["lens"].device

    def gather(pages, scales):
        x = pages[s["table"].long()].float()                       # [B, pages, Hkv, P, d]
        if scales is not None:
            x = x * scales[s["table"].long()][..., None, None]
        return x.transpose(1, 2).reshape(B, Hkv, S, d)

    t = torch.arange(S, device=dev)
    sees = t[None, None, :] < (s["lens"][:, None, None] - (T - 1 - torch.arange(T, device=dev))[None, :, None])   # [B, T, S]
    q = s["q"].float().reshape(B, T, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, d)
    logits = (q @ gather(s["k_pages"], s["k_scales"]).transpose(-1, -2)) * (1.0 / math.sqrt(d))
    mask = sees[:, None, :, None, :].expand(B, Hkv, T, G, S).reshape(B, Hkv, T * G, S)
    logits = logits.masked_fill(~mask, -math.inf)
    top = logits.amax(dim=-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(logits - top)
    total = p.sum(dim=-1, keepdim=True)
    v = gather(s["v_pages"], s["v_scales"])
    v = torch.where((t[None, :] < s["lens"][:, None])[:, None, :, None], v, torch.zeros_like(v))
    out = torch.where(total > 0, (p @ v) / total, torch.zeros_like(q))
    lse = (top + total.log())[..., 0]
    back = lambda x: x.reshape(B, Hkv, T, G, -1).permute(0, 2, 1, 3, 4)  # noqa: E731
    return {"out": back(out).reshape(B, T, Hq, d), "lse": back(lse).reshape(B, T, Hq)}


def run(state):
    s, c = state, state["case"]
    if not own:
        return _plain_append(s) if c["op"] == "append" else _plain_attn(s)
    from paper_2502_01068_b200 import binding as F
    if c["op"] == "append":
        F.fastkv_paged_append(s["cache"], s["rows"], s["lens"], s["q"], s["k"], s["v"], s["pos"], s["inv_freq"], s["idx"],
                              s["q_out"], s["new_lens"], s["ws"])
        out = {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "lens": s["new_lens"]}
        if s["q"] is not None:
            out["q"] = s["q_out"]
        if c["fmt"] == "e4m3":
            out["k_scales"], out["v_scales"] = s["k_scales"], s["v_scales"]
        return out
    F.fastkv_paged_attn(s["cache"], s["query"], s["lens"], s["q"], s["out"], s["lse"], s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


# ---- the same from the definition, in 64 bits ----------------------------------------------------------------------------
def _exact_turn(x, pos, freq, rot, adjacent):
    """Each pair as a complex number times e^(i pos f)."""
    x = x.double().clone()
    if not rot:
        return x
    a = torch.outer(pos.double(), freq.double())[:, None, :]
    turn = torch.polar(torch.ones_like(a), a)
    i = torch.arange(rot // 2, device=x.device)
    lo, hi = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
    z = torch.complex(x[..., lo], x[..., hi]) * turn
    x[..., lo], x[..., hi] = z.real, z.imag
    return x


def _exact_code(x):
    """x to the nearest e4m3 value, ties to even: 3 bits behind the leading one, steps of 2^-9 below 2^-6."""
    _, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), (e - 1).clamp(min=-6) - 3)
    return (torch.round(x / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _exact_append(s):
    c = s["case"]
    P, out = c["page"], {}
    pools = {"k": s["k_pages"].double(), "v": s["v_pages"].double()}
    scales = {n: (s[n + "_scales"].double() if s[n + "_scales"] is not None else None) for n in "kv"}
    at = 0
    for b, n in enumerate(s["new"]):
        have = int(s["lens"][b])
        first, last = have // P, (have + n - 1) // P
        ids = s["table"][b, first:last + 1].long()
        for name in "kv":
            if s["idx"] is not None:
                fresh = torch.stack([s[name][s["idx"][h].long(), h] for h in range(c["hkv"])], dim=1).double()
            else:
                fresh = s[name][at:at + n].double()
            if name == "k" and c["rot"]:
                fresh = _exact_turn(fresh, s["pos"][at:at + n], s["inv_freq"], c["rot"], c["adjacent"])
            # the run of touched pages as one stretch of slots [heads, slots, d]
            run_ = pools[name][ids].transpose(0, 1).reshape(c["hkv"], -1, c["d"])
            lo = have - first * P
            if scales[name] is None:
                run_[:, lo:lo + n] = fresh.transpose(0, 1)
            else:
                is_new = torch.zeros(run_.shape[1], dtype=torch.bool, device=run_.device)
                is_new[lo:lo + n] = True
                y = torch.zeros_like(run_)
                y[:, lo:lo + n] = fresh.transpose(0, 1)
                m = y.abs().reshape(c["hkv"], -1, P * c["d"]).amax(dim=-1)             # [heads, pages]
                e = torch.ceil(torch.log2(m.clamp(min=2.0 ** -80) / E4M3_MAX))
                e = torch.where(torch.exp2(e - 1) * E4M3_MAX >= m, e - 1, e)
                e = torch.where(torch.exp2(e) * E4M3_MAX < m, e + 1, e).clamp(SCALE_MIN_EXP, SCALE_MAX_EXP)
                want = torch.exp2(e)
                was = scales[name][ids].t()
                if lo > 0:
                    want[:, 0] = torch.maximum(want[:, 0], was[:, 0])
                per_slot = lambda z: z.repeat_interleave(P, dim=1)[..., None]  # noqa: E731
                old = (torch.arange(run_.shape[1], device=run_.device) < lo)[None, :, None]
                run_ = torch.where(old, _exact_code(run_ * per_slot(was) / per_slot(want)), run_)
                run_ = torch.where(is_new[None, :, None], _exact_code(y / per_slot(want)), run_)
                scales[name][ids] = want.t()
            pools[name][ids] = run_.reshape(c["hkv"], -1, P, c["d"]).transpose(0, 1)
        at += n
    if s["q"] is not None:
        out["q"] = _exact_turn(s["q"], s["pos"], s["inv_freq"], c["rot"], c["adjacent"]) if c["rot"] else s["q"].double()
    if c["fmt"] == "e4m3":
        out["k_scales"], out["v_scales"] = scales["k"], scales["v"]
    out["k_pages"], out["v_pages"] = pools["k"], pools["v"]
    out["lens"] = s["lens"] + torch.tensor(s["new"], dtype=torch.int32, device="cuda")
    return out


def _exact_attn(s):
    c = s["case"]
    T, Hkv, d, P = c["q_len"], c["hkv"], c["d"], c["page"]
    G = c["hq"] // Hkv
    outs, lses = [], []
    for b in range(c["batch"]):
        n = int(s["lens"][b])
        ids = s["table"][b, : -(-n // P)].long()
        o = torch.zeros((T, Hkv, G, d), dtype=torch.float64, device="cuda")
        l = torch.full((T, Hkv, G), -math.inf, dtype=torch.float64, device="cuda")
        for h in range(Hkv):
            k, v = s["k_pages"][ids, h].double(), s["v_pages"][ids, h].double()
            if s["k_scales"] is not None:
                k = k * s["k_scales"][ids, h].double()[:, None, None]
                v = v * s["v_scales"][ids, h].double()[:, None, None]
            k, v = k.reshape(-1, d), v.reshape(-1, d)
            for i in range(T):
                m = n - (T - 1 - i)
                if m <= 0:
                    continue
                x = s["q"][b, i, h * G:(h + 1) * G].double() @ k[:m].t() / math.sqrt(d)
                l[i, h] = torch.logsumexp(x, dim=-1)
                o[i, h] = torch.softmax(x, dim=-1) @ v[:m]
        outs.append(o.reshape(T, c["hq"], d))
        lses.append(l.reshape(T, c["hq"]))
    return {"out": torch.stack(outs), "lse": torch.stack(lses)}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(s) if case["op"] == "append" else _exact_attn(s)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    c = case
    item = 2 if c["fmt"] == "bf16" else 1
    if c["op"] == "append":
        rows = sum(_new_lengths(c))
        kv = rows * 2 * c["hkv"] * c["d"]
        q = rows * c["hq"] * c["d"]
        moved = kv * (2 + item) + q * 4 + (rows * 4 if c["rot"] else 0) + (4 * rows * c["hkv"] if c["source"] else 0)
        turned = rows * (c["hq"] + c["hkv"]) * c["rot"] * 3
        return {"bytes": moved, "flops": turned}
    low = c["shortest"] or c["length"]
    entries = c["length"] + (c["batch"] - 1) * (low + c["length"]) / 2
    moved = entries * c["hkv"] * 2 * c["d"] * item + (entries / c["page"] * c["hkv"] * 8 if item == 1 else 0)
    moved += c["batch"] * c["q_len"] * c["hq"] * (c["d"] * 2 + c["d"] * 4 + 4)
    return {"bytes": moved, "flops": 4.0 * entries * c["hq"] * c["q_len"] * c["d"]}
