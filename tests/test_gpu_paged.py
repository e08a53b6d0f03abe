"""The paged cache on a B200: appending rows (rotation, bf16 and 8-bit pages, kept rows by index) and the attention over the
pages, against the 64-bit reference; then the two in use together behind a selection.

Every entry, page and scale that belongs to nobody holds NaN, and block-table entries beyond a sequence's pages name no page:
a read that strays shows up in the output or in the status word.

Bounds.  A rounding to bf16 is off by at most 2^-8 of the value, one to e4m3 by 2^-4 of it (2^-10 of the scale where codes are
subnormal).  A rotated value has two fp32 products and a sum, with cos and sin rounded to fp32: off by at most
3 * 2^-24 (|x1| + |x2|) <= 2^-20 max|row|.  Attention: a logit is a sum of d exact products, accumulated in fp32 with at most
d / 16 + 8 roundings of 2^-23 of sum |q k| (a step of 16 products may lose one unit of its largest partial sum); the weights
p are off by twice the largest logit error, 2^-20 for the exponentials, their two-term rounding and the merges; the sums over
n entries by one rounding of 2^-23 for each 16 entries, all of it relative to sum p |v|."""
import math

import numpy as np
import pytest
import torch

from paper_2502_01068_b200 import binding as B
from paper_2502_01068_b200 import workloads as W
from tests.paged_reference import Pools, attention, need_scale, rn_e4m3, rotate

pytestmark = pytest.mark.gpu


def bf16_rows(rng, shape, gain=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * gain).to(torch.bfloat16)


def workspace(nbytes=256):
    """A header of zeros, and behind it what no call may read before it has written it: NaN in every word."""
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
    ws[:256] = 0
    return ws


def inv_freq(rot, base=500000.0):
    return torch.from_numpy((base ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)) if rot else None


def check_append(pools, before, lens, news, k64, v64, rotated):
    """pools: after the call; before: (k, v, ks, vs) copies from before it; k64 / v64: the new rows in 64 bits, per sequence."""
    P, Hkv, d = pools.page, pools.Hkv, pools.d
    for name, old_pool, old_scales, rows, old64 in (("k", before[0], before[2], k64, pools.k64), ("v", before[1], before[3], v64, pools.v64)):
        pool = getattr(pools, name).cpu()
        scales = None if old_scales is None else getattr(pools, name + "s").cpu()
        loose = rotated and name == "k"
        want_bits = old_pool.view(torch.uint8).clone() if pools.fmt == "e4m3" else old_pool.view(torch.int16).clone()
        want_scales = None if old_scales is None else old_scales.clone()
        for b, (n0, n) in enumerate(zip(lens, news)):
            for pg in range(n0 // P, -(-(n0 + n) // P) if n else n0 // P):
                pid = int(pools.table_np[b, pg])
                lo, hi = max(n0, pg * P), min(n0 + n, (pg + 1) * P)
                if hi <= lo:
                    continue
                new = rows[b][lo - n0:hi - n0]                        # [m, Hkv, d]
                n_old = max(0, min(P, n0 - pg * P))
                if pools.fmt == "bf16":
                    got = pool[pid, :, lo - pg * P:hi - pg * P].float().double().numpy().transpose(1, 0, 2)
                    slack = 2.0 ** -20 * np.abs(new).max(axis=-1, keepdims=True) if loose else 0.0
                    assert np.all(np.abs(got - new) <= 2.0 ** -8 * (np.abs(new) + slack) + slack), (name, b, pg)
                    if not loose:
                        ref = torch.from_numpy(new).to(torch.bfloat16).transpose(0, 1)
                        assert torch.equal(pool[pid, :, lo - pg * P:hi - pg * P].view(torch.int16), ref.contiguous().view(torch.int16))
                    want_bits[pid, :, lo - pg * P:hi - pg * P] = pool.view(torch.int16)[pid, :, lo - pg * P:hi - pg * P]
                    continue
                for h in range(Hkv):
                    s_old = float(old_scales[pid, h]) if n_old else 0.0
                    top = float(np.abs(new[:, h]).max())
                    s = float(scales[pid, h])
                    ok = {max(s_old, need_scale(top))}
                    if loose:
                        ok |= {max(s_old, need_scale(top * (1 - 2.0 ** -20))), max(s_old, need_scale(top * (1 + 2.0 ** -20)))}
                    assert s in ok, (name, b, pg, h, s, ok)
                    want_scales[pid, h] = s
                    got = pool[pid, h, lo - pg * P:hi - pg * P].view(torch.float8_e4m3fn).float().double().numpy() * s
                    ref = rn_e4m3(new[:, h] / s) * s
                    if loose:
                        slack = 2.0 ** -20 * np.abs(new[:, h]).max(axis=-1, keepdims=True)
                        assert np.all(np.abs(got - new[:, h]) <= 2.0 ** -4 * (np.abs(new[:, h]) + slack) + slack + s * 2.0 ** -10)
                        assert np.mean(got != ref) < 1e-3              # a value next to a rounding border may fall either way
                    else:
                        np.testing.assert_array_equal(got, ref)
                    want_bits[pid, h, lo - pg * P:hi - pg * P] = pool[pid, h, lo - pg * P:hi - pg * P]
                    if n_old:
                        ref = rn_e4m3(old64[b][pg * P:pg * P + n_old, h] / s)
                        got = pool[pid, h, :n_old].view(torch.float8_e4m3fn).float().double().numpy()
                        np.testing.assert_array_equal(got, ref)
                        want_bits[pid, h, :n_old] = pool[pid, h, :n_old]
        now = pool.view(torch.uint8) if pools.fmt == "e4m3" else pool.view(torch.int16)
        assert torch.equal(now, want_bits), "%s: an entry that the call does not own changed" % name
        if scales is not None:
            assert torch.equal(scales.view(torch.int32), want_scales.view(torch.int32))


def run_append(fmt, lens, news, page, Hq, Hkv, d, rot=0, adjacent=False, uniform=False, gain=1.0, packed=False, seed=0, first_pos=0):
    rng = np.random.default_rng(seed)
    pools = Pools(fmt, lens, [a + b for a, b in zip(lens, news)], page, Hkv, d, seed + 1)
    before = [None if t is None else t.cpu().clone() for t in (pools.k, pools.v, pools.ks, pools.vs)]
    total, Bn = sum(news), len(news)
    if packed:                                                         # q, k and v side by side, as one projection leaves them
        qkv = bf16_rows(rng, (total, Hq + 2 * Hkv, d), gain).cuda()
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        st = (Hq + 2 * Hkv) * d
    else:
        q, k, v = (bf16_rows(rng, (total, H, d), gain).cuda() for H in (Hq, Hkv, Hkv))
        st = None
    pos = torch.from_numpy(first_pos + rng.integers(0, 131072, total).astype(np.int32)) if rot else None
    cu = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    rows = B.make_new_rows(batch=Bn, total=total, max_new=max(news), cu_new=None if uniform else torch.from_numpy(cu).cuda(),
                           n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, rot_dim=rot,
                           rot_pairs=B.ROT_ADJACENT if adjacent else B.ROT_HALVES, q_stride_tok=st, k_stride_tok=st, v_stride_tok=st)
    q_out = torch.full((total, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda") if Hq else None
    new_lens = torch.full((Bn,), -1, dtype=torch.int32, device="cuda")
    ws = workspace()
    f = inv_freq(rot)
    B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, q if Hq else None, k, v, pos.cuda() if rot else None,
                          f.cuda() if rot else None, None, q_out, new_lens, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    assert new_lens.cpu().tolist() == [a + b for a, b in zip(lens, news)]
    x64 = lambda t: t.cpu().float().double().numpy()  # noqa: E731
    k64 = rotate(x64(k), pos, f, rot, adjacent)
    split = lambda x: [x[cu[b]:cu[b + 1]] for b in range(Bn)]  # noqa: E731
    check_append(pools, before, lens, news, split(k64), split(x64(v)), rot > 0)
    if Hq:
        ref = rotate(x64(q), pos, f, rot, adjacent)
        slack = 2.0 ** -20 * np.abs(ref).max(axis=-1, keepdims=True)
        assert np.all(np.abs(x64(q_out) - ref) <= 2.0 ** -8 * (np.abs(ref) + slack) + slack)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens,news,page", [
    ([0], [1], 16), ([15], [1], 16), ([16], [1], 16), ([31, 0, 64, 7], [1, 1, 1, 1], 32),       # single tokens
    ([13, 0, 40], [5, 0, 8], 16), ([63, 64, 1], [2, 8, 3], 64),                                # a few, across a page's end, none
    ([0], [200], 64), ([37], [171], 128), ([5, 130, 0], [300, 9, 77], 32), ([100], [64], 16),  # chunks of prompts
    ([120, 3], [17, 260], 128)])
@pytest.mark.parametrize("Hq,Hkv,d,rot,adjacent", [(8, 2, 128, 128, False), (3, 1, 64, 64, True), (8, 8, 128, 64, False), (0, 3, 64, 0, False)])
def test_append_against_the_reference(fmt, lens, news, page, Hq, Hkv, d, rot, adjacent):
    run_append(fmt, lens, news, page, Hq, Hkv, d, rot, adjacent, uniform=len(set(news)) == 1, seed=page + d + sum(news))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("news", [[1, 1, 1], [40, 3, 90]])
def test_append_from_a_packed_projection_and_far_positions(fmt, news):
    """q, k and v are slices of one tensor; positions up to 2^31 - 1 (the angle needs 64 bits)."""
    run_append(fmt, [10, 0, 33], news, 32, 8, 2, 128, 128, False, packed=True, seed=3, first_pos=2 ** 31 - 131072 - 1)


@pytest.mark.parametrize("news", [[1, 1], [70, 9]])
def test_append_larger_rows_re_encode_the_page(news):
    """New rows a thousand times larger than what the page holds: its scale grows and most old codes become subnormal or zero."""
    run_append("e4m3", [9, 50], news, 64, 0, 2, 128, gain=3000.0, seed=11)
    run_append("e4m3", [9, 50], news, 64, 0, 2, 64, gain=1e-6, seed=12)      # and far smaller ones: the old scale stays


def test_append_extreme_values():
    """Zeros, the largest bf16 values, tiny ones and infinities; a NaN stays a NaN of its own element."""
    Hkv, d, P = 1, 64, 16
    pools = Pools("e4m3", [0] * 5, [1] * 5, P, Hkv, d, 5)
    big = float(torch.finfo(torch.bfloat16).max)
    x = torch.zeros(5, Hkv, d)
    x[1] = torch.where(torch.arange(d) % 2 == 0, big, -big / 3)
    x[2] = 1e-38
    x[3, 0, 0], x[3, 0, 1] = float("inf"), 1.0
    x[4], x[4, 0, 5] = 2.0, float("nan")
    x = x.to(torch.bfloat16)
    rows = B.make_new_rows(batch=5, total=5, n_kv_heads=Hkv, head_dim=d)
    ws = workspace()
    B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, None, x.cuda(), x.cuda(), None, None, None, None, None, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    got = [pools.read(b, 1)[0][0, 0] for b in range(5)]
    ref = x.float().double().numpy()[:, 0]
    assert np.all(got[0] == 0.0)
    np.testing.assert_array_equal(got[1], rn_e4m3(ref[1] / need_scale(np.abs(ref[1]).max())) * need_scale(np.abs(ref[1]).max()))
    np.testing.assert_array_equal(got[2], np.zeros(d))                       # 1e-38 lies below the smallest step
    assert got[3][0] == 448.0 * 2.0 ** 120 and np.all(got[3][1:] == 0.0)     # an infinity saturates the block's largest scale
    assert np.isnan(got[4][5]) and np.all(np.delete(got[4], 5) == 2.0)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hkv,d,page", [(8, 128, 64), (2, 64, 16), (3, 128, 128)])
def test_append_kept_rows_equals_compact_then_append(fmt, Hkv, d, page):
    """What the selection kept goes straight into pages: the same bytes as compacting first and appending the compact rows (whose
    heads lie far apart: a token stride smaller than the head stride)."""
    rng = np.random.default_rng(d + page)
    src_lens, kept = [400, 150, 911], [80, 150, 300]
    cu_src = np.concatenate([[0], np.cumsum(src_lens)]).astype(np.int32)
    cu_k = np.concatenate([[0], np.cumsum(kept)]).astype(np.int32)
    k, v = bf16_rows(rng, (sum(src_lens), Hkv, d)).cuda(), bf16_rows(rng, (sum(src_lens), Hkv, d)).cuda()
    idx = np.concatenate([np.stack([np.sort(rng.permutation(n)[:m]) for _ in range(Hkv)]) for n, m in zip(src_lens, kept)], axis=1)
    idx = torch.from_numpy(idx.astype(np.int32)).cuda()
    d_src, d_k = torch.from_numpy(cu_src).cuda(), torch.from_numpy(cu_k).cuda()
    got = []
    for way in ("gather", "compact"):
        pools = Pools(fmt, [0, 0, 0], kept, page, Hkv, d, 77)
        ws = workspace()
        if way == "gather":
            rows = B.make_new_rows(batch=3, total=sum(kept), max_new=max(kept), cu_new=d_k, n_kv_heads=Hkv, head_dim=d,
                                   total_src=sum(src_lens), cu_src=d_src)
            B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, None, k, v, None, None, idx, None, None, ws)
        else:
            shape = B.make_shape(total_len=sum(src_lens), n_q_heads=Hkv, n_kv_heads=Hkv, head_dim=d, batch=3, max_len=911,
                                 cu_seqlens=d_src)
            ko = torch.zeros((Hkv, sum(kept), d), dtype=torch.int16, device="cuda")
            vo = torch.zeros_like(ko)
            B.fastkv_compact(shape, idx, B.make_budget(0, cu_k=d_k, total=sum(kept)), None, None, k, v, None, None, ko, vo, None, None, ws)
            rows = B.make_new_rows(batch=3, total=sum(kept), max_new=max(kept), cu_new=d_k, n_kv_heads=Hkv, head_dim=d,
                                   k_stride_tok=d, k_stride_head=sum(kept) * d, v_stride_tok=d, v_stride_head=sum(kept) * d)
            B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, None, ko, vo, None, None, None, None, None, ws)
        assert B.fastkv_device_status(ws) == (0, 0)
        got.append([t.cpu().view(torch.uint8) for t in (pools.k, pools.v, pools.ks, pools.vs) if t is not None])
    assert all(torch.equal(a, b) for a, b in zip(*got))
    x = pools.read(1, kept[1])[1]                                            # and they are the rows that were asked for
    ref = v.cpu().float().double().numpy()[400:][idx[:, 80:230].cpu().numpy().T, np.arange(Hkv)[None, :]]
    tol = 2.0 ** -8 if fmt == "bf16" else 2.0 ** -4
    assert np.all(np.abs(x - ref) <= tol * np.abs(ref) + (0.0 if fmt == "bf16" else 2.0 ** -10 * need_scale(np.abs(ref).max())))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("kept", [5, 100])
def test_append_kept_rows_of_a_head_major_source(fmt, kept):
    """Keys and values that are stored head by head, [n_kv_heads, rows, head_dim]: the rows that idx names, exactly."""
    rng = np.random.default_rng(kept)
    Hkv, d, L = 4, 128, 777
    k, v = bf16_rows(rng, (Hkv, L, d)), bf16_rows(rng, (Hkv, L, d))
    idx = np.stack([np.sort(rng.permutation(L)[:kept]) for _ in range(Hkv)]).astype(np.int32)
    pools = Pools(fmt, [0], [kept], 32, Hkv, d, 3)
    before = [None if t is None else t.cpu().clone() for t in (pools.k, pools.v, pools.ks, pools.vs)]
    rows = B.make_new_rows(batch=1, total=kept, n_kv_heads=Hkv, head_dim=d, total_src=L, k_stride_tok=d, k_stride_head=L * d,
                           v_stride_tok=d, v_stride_head=L * d)
    ws = workspace()
    B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, None, k.cuda(), v.cuda(), None, None, torch.from_numpy(idx).cuda(), None, None, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    pick = lambda x: x.double().numpy()[np.arange(Hkv)[:, None], idx].transpose(1, 0, 2)  # noqa: E731
    check_append(pools, before, [0], [kept], [pick(k)], [pick(v)], False)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1, 40])
def test_append_reports_what_it_cannot_write(fmt, n):
    """A page id outside the pool, rows beyond the block table's room, an index outside its sequence: reported, and nothing but
    the good rows is written."""
    Hkv, d, P = 2, 64, 16
    rng = np.random.default_rng(4)
    k = bf16_rows(rng, (2 * n, Hkv, d)).cuda()
    rows = B.make_new_rows(batch=2, total=2 * n, n_kv_heads=Hkv, head_dim=d)
    for bad in (-1, 10 ** 6):
        pools = Pools(fmt, [5, 3], [5 + n, 3 + n], P, Hkv, d, 9)
        pools.table[0, :] = bad
        before = pools.k.cpu().clone()
        ws = workspace()
        new_lens = torch.zeros(2, dtype=torch.int32, device="cuda")
        B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, None, k, k, None, None, None, None, new_lens, ws)
        assert B.fastkv_device_status(ws)[0] == B.ERR_DEVICE_INDEX
        own = [int(x) for x in pools.table_np[1] if x >= 0]
        others = [i for i in range(pools.n_pages) if i not in own]
        assert torch.equal(pools.k.cpu().view(torch.uint8)[others], before.view(torch.uint8)[others])
        assert np.isfinite(pools.read(1, 3 + n)[0]).all()
    pools = Pools(fmt, [5, 3], [5 + n, 3 + n], P, Hkv, d, 9)
    room = pools.table.shape[1] * P
    lens = torch.tensor([room, 3], dtype=torch.int32, device="cuda")         # sequence 0 is full
    ws, new_lens = workspace(), torch.zeros(2, dtype=torch.int32, device="cuda")
    B.fastkv_paged_append(pools.cache(), rows, lens, None, k, k, None, None, None, None, new_lens, ws)
    assert B.fastkv_device_status(ws)[0] == B.ERR_DEVICE_INDEX
    assert new_lens.tolist() == [room, 3 + n]
    pools = Pools(fmt, [5, 3], [5 + n, 3 + n], P, Hkv, d, 9)
    idx = torch.zeros((Hkv, 2 * n), dtype=torch.int32, device="cuda")
    idx[1, 0], idx[0, n] = n, -1
    cu = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
    r2 = B.make_new_rows(batch=2, total=2 * n, n_kv_heads=Hkv, head_dim=d, total_src=2 * n, cu_src=cu)
    ws = workspace()
    B.fastkv_paged_append(pools.cache(), r2, pools.dev_lens, None, k, k, None, None, idx, None, None, ws)
    assert B.fastkv_device_status(ws)[0] == B.ERR_DEVICE_INDEX
    assert np.isfinite(pools.read(0, 5 + n)[0][:, 0]).all() and np.isfinite(pools.read(1, 3 + n)[0][:, 1]).all()
    assert np.isnan(pools.read(0, 6)[0][5, 1]).all() and np.isnan(pools.read(1, 4)[0][3, 0]).all()      # the skipped rows


def test_queries_may_be_rotated_in_place():
    rng = np.random.default_rng(8)
    outs = []
    for place in (False, True):
        pools = Pools("e4m3", [3, 9], [10, 30], 16, 2, 128, 1)
        rng = np.random.default_rng(8)
        q, k = bf16_rows(rng, (8, 8, 128)).cuda(), bf16_rows(rng, (8, 2, 128)).cuda()
        pos = torch.arange(1000, 1008, dtype=torch.int32, device="cuda")
        rows = B.make_new_rows(batch=2, total=8, n_q_heads=8, n_kv_heads=2, head_dim=128, rot_dim=128)
        q_out = q if place else torch.zeros_like(q)
        ws = workspace()
        B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, q, k, k, pos, inv_freq(128).cuda(), None, q_out, None, ws)
        assert B.fastkv_device_status(ws) == (0, 0)
        outs.append(q_out.cpu())
    assert torch.equal(outs[0], outs[1])


# ---- attention --------------------------------------------------------------------------------------------------------------
def check_attention(pools, lens, q, out, lse, scale, sequences=None):
    d = pools.d
    T = q.shape[1]
    for b in (range(len(lens)) if sequences is None else sequences):
        for i in range(T):
            sees = lens[b] - (T - 1 - i)
            ref, ref_lse, mass, size = attention(q[b, i], pools.k64[b], pools.v64[b], sees, scale)
            delta = (d / 16 + 8) * 2.0 ** -23 * size[:, None] + 2.0 ** -23 * np.abs(np.where(np.isfinite(ref_lse), ref_lse, 0.0))[:, None]
            tol = (2 * delta + 2.0 ** -20 + (max(sees, 0) / 16 + 16) * 2.0 ** -23) * mass + 1e-30
            err = np.abs(out[b, i] - ref)
            assert np.all(err <= tol), (b, i, float((err / tol).max()), float(err.max()))
            if sees <= 0:
                assert np.all(out[b, i] == 0.0) and np.all(np.isneginf(lse[b, i]))
            else:
                t_lse = delta[:, 0] + 2.0 ** -20 + (sees / 16 + 16) * 2.0 ** -23 + 2.0 ** -22 * np.abs(ref_lse)
                assert np.all(np.abs(lse[b, i] - ref_lse) <= t_lse), (b, i, np.abs(lse[b, i] - ref_lse).max())


def run_attention(fmt, lens, page, Hq, Hkv, d, T=1, scale=0.0, seed=0, v_exp=(-7, -4), max_len=None, gain=1.0, total_len=0, check=True, sequences=None):
    rng = np.random.default_rng(seed)
    pools = Pools(fmt, lens, lens, page, Hkv, d, seed + 1, v_exp=v_exp)
    q = bf16_rows(rng, (len(lens), T, Hq, d), gain)
    query = B.make_query(n_q_heads=Hq, q_len=T, max_len=max(lens) if max_len is None else max_len, total_len=total_len, softmax_scale=scale)
    cache = pools.cache()
    ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
    out = torch.full((len(lens), T, Hq, d), 7.0, device="cuda")
    lse = torch.full((len(lens), T, Hq), 7.0, device="cuda")
    B.fastkv_paged_attn(cache, query, pools.dev_lens, q.cuda(), out, lse, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    out, lse = out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    if check:
        check_attention(pools, lens, q.float().double().numpy(), out, lse, scale or d ** -0.5, sequences)
    return out, lse


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,d", [(32, 8, 128), (4, 1, 64), (8, 8, 128), (16, 2, 64), (6, 3, 128)])
@pytest.mark.parametrize("lens,page", [([1], 16), ([17], 16), ([129], 128), ([1000, 5, 16, 0, 333], 32), ([4097], 64)])
def test_attention_against_the_reference(fmt, Hq, Hkv, d, lens, page):
    run_attention(fmt, lens, page, Hq, Hkv, d, seed=Hq + d + sum(lens))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("T", [2, 3, 5, 9])
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 128), (8, 1, 64), (3, 3, 128), (28, 4, 128)])
def test_attention_of_several_query_tokens(fmt, T, Hq, Hkv, d):
    """Rows of a group in one, two and more tiles; sequences shorter than q_len have queries that see nothing."""
    run_attention(fmt, [300, 1, 33, 0, 16, 4], 16, Hq, Hkv, d, T=T, seed=T)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("max_len,total", [(130, 0), (40000, 0), (40000, 1000), (900000, 1000)])
def test_attention_of_a_whole_stretch_of_query_tokens(fmt, max_len, total):
    """As many query tokens as entries, more than entries, and fewer; every tile of rows has its own masks."""
    run_attention(fmt, [130, 330, 64, 0], 32, 6, 2, 64, T=130, seed=4, max_len=max_len, total_len=total)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_attention_masks_what_is_not_finite(fmt):
    """A query token does not see the entries of the tokens behind it, whatever they hold: its outputs are those of a cache
    without them.  Where it does see a NaN in V, that element is NaN; an infinity leaves it NaN or infinite; a NaN in K makes
    the whole row NaN, and none of it spreads to the other sequences, heads or rows."""
    T, Hq, Hkv, d, lens = 4, 8, 2, 128, [700, 66, 5]
    pools = Pools(fmt, lens, lens, 32, Hkv, d, 3)
    pools.k64, pools.v64 = [x.copy() for x in pools.k64], [x.copy() for x in pools.v64]
    bad_code = {"nan": 0x7F, "inf": 0xFF}

    def spoil(name, b, t, h, col, what):
        pid, row = int(pools.table_np[b, t // 32]), t % 32
        if fmt == "bf16":
            getattr(pools, name)[pid, h, row, col] = float(what)
        else:
            getattr(pools, name)[pid, h, row, col] = bad_code[what]

    spoil("v", 0, 699, 1, 77, "nan")             # the last token's own entry: seen by token 3 alone
    spoil("v", 0, 697, 0, 5, "inf")              # by tokens 1, 2 and 3
    spoil("v", 1, 65, 1, 0, "inf")
    spoil("v", 1, 64, 1, 127, "nan")             # by tokens 2 and 3; 63 and 64 lie in different pages
    spoil("k", 1, 65, 0, 9, "nan")
    spoil("v", 2, 3, 0, 64, "nan")
    spoil("k", 2, 2, 1, 3, "nan")                # by tokens 1, 2 and 3
    q = bf16_rows(np.random.default_rng(8), (len(lens), T, Hq, d))
    cache = pools.cache()
    for longest, total in ((66, 0), (700, 0), (20000, 771), (200000, 771)):       # whole, split in two ways, dealt out
        query = B.make_query(n_q_heads=Hq, q_len=T, max_len=longest, total_len=total)
        ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
        out, lse = (torch.full(s, 7.0, device="cuda") for s in ((len(lens), T, Hq, d), (len(lens), T, Hq)))
        B.fastkv_paged_attn(cache, query, pools.dev_lens, q.cuda(), out, lse, ws)
        assert B.fastkv_device_status(ws) == (0, 0)
        out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
        wild = np.zeros(out.shape, dtype=bool)
        lost = np.zeros(lse.shape, dtype=bool)
        wild[0, 3, 4:, 77] = wild[0, 1:, :4, 5] = wild[1, 3, 4:, 0] = wild[1, 2:, 4:, 127] = wild[2, 2:, :4, 64] = True
        lost[1, 3, :4] = lost[2, 1:, 4:] = True
        assert np.array_equal(np.isnan(lse), lost)
        assert np.array_equal(~np.isfinite(out), wild | lost[..., None])
        for b, n in enumerate(lens):
            for i in range(T):
                want, want_lse, mass, size = attention(q[b, i].double().numpy(), pools.k64[b], pools.v64[b], n - (T - 1 - i), d ** -0.5)
                good = ~(wild[b, i] | lost[b, i][:, None])
                delta = (d / 16 + 8) * 2.0 ** -23 * size[:, None] + 2.0 ** -23 * np.abs(want_lse)[:, None]
                tol = (2 * delta + 2.0 ** -20 + (n / 16 + 16) * 2.0 ** -23) * mass + 1e-30
                assert np.all((np.abs(out[b, i] - want) <= tol)[good])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_a_length_below_zero_is_reported_however_the_batch_is_dealt(fmt):
    lens = [20000, 40, 3000, 90]
    pools = Pools(fmt, lens, lens, 32, 2, 64, 5)
    q = bf16_rows(np.random.default_rng(5), (4, 1, 8, 64))
    cache = pools.cache()
    for longest, total in ((20000, sum(lens)), (20000, 4 * 20000), (200000, sum(lens))):
        query = B.make_query(n_q_heads=8, max_len=longest, total_len=total)
        ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
        out, lse = torch.full((4, 1, 8, 64), 7.0, device="cuda"), torch.full((4, 1, 8), 7.0, device="cuda")
        pools.dev_lens[1] = -3
        B.fastkv_paged_attn(cache, query, pools.dev_lens, q.cuda(), out, lse, ws)
        assert B.fastkv_device_status(ws) == (B.ERR_DEVICE_INDEX, 41)
        check_attention(pools, [20000, 0, 3000, 90], q.double().numpy(), out.cpu().double().numpy(), lse.cpu().double().numpy(), 64 ** -0.5)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_attention_of_batches_larger_than_the_machine(fmt):
    rng = np.random.default_rng(2)
    lens = [int(x) for x in rng.integers(0, 300, 70)]
    run_attention(fmt, lens, 32, 8, 4, 64, seed=3, total_len=sum(lens), sequences=range(0, 70, 9))
    run_attention(fmt, lens, 32, 8, 4, 64, T=4, seed=4, sequences=range(0, 70, 9))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_attention_of_very_different_lengths(fmt):
    lens = [9000, 3, 700, 0, 64, 2500]
    run_attention(fmt, lens, 64, 8, 2, 128, seed=5, total_len=sum(lens))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("scale,gain", [(4.0, 1.0), (0.05, 1.0), (0.0, 1000.0), (0.0, 1e-30)])
def test_attention_with_peaked_and_flat_softmax(fmt, scale, gain):
    run_attention(fmt, [500, 77], 16, 8, 2, 128, scale=scale, gain=gain, seed=6)


def test_attention_when_the_pages_scales_lie_far_apart():
    """V's scale is an addend of the exponent: pages from 2^-64 to 2^100 in one sequence."""
    for v_exp in ((-64, -60), (95, 100), (-64, 100)):
        run_attention("e4m3", [600, 40], 16, 8, 2, 128, seed=7, v_exp=v_exp)
        run_attention("e4m3", [600, 40], 16, 4, 2, 64, T=3, seed=8, v_exp=v_exp)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_what_the_host_knows_of_lengths_changes_nothing(fmt):
    """max_len and total_len only size the launch: a bound that is too large, or too small, gives the same results."""
    for guess, total in ((2000, 0), (100000, 10), (1, 1), (700, 5000)):
        run_attention(fmt, [1999, 20, 0], 64, 8, 2, 128, seed=9, max_len=guess, total_len=total)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens", [[0, 0, 0], [40, 0, 1], [70, 333, 64, 1], [130] * 20])
@pytest.mark.parametrize("T", [1, 5])
@pytest.mark.parametrize("longest", [40000, 400000])
def test_batches_far_shorter_than_the_host_thinks(fmt, lens, T, longest):
    """Dealt out evenly, there are fewer chunks than CTAs: some of them get none, and whoever joins the pieces must know it."""
    run_attention(fmt, lens, 16, 8, 2, 64, T=T, seed=9, max_len=longest, total_len=50000)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(128, 16), (128, 64), (64, 16), (64, 128)])
def test_attention_with_the_pools_in_either_order_or_far_apart(fmt, d, page):
    """K and V boxes arrive by one copy where the pools allow it: K below V, V below K, and (forced) a copy each."""
    rng = np.random.default_rng(12)
    lens = [333, 0, 17]
    q = bf16_rows(rng, (3, 1, 8, d))
    query = B.make_query(n_q_heads=8, max_len=333)
    results = []
    for way in ("k below v", "v below k", "apart"):
        pools = Pools(fmt, lens, lens, page, 2, d, 13)
        both = torch.empty((2,) + tuple(pools.k.shape), dtype=pools.k.dtype, device="cuda")
        k, v = (both[1], both[0]) if way == "v below k" else (both[0], both[1])
        k.copy_(pools.k)
        v.copy_(pools.v)
        cache = B.make_paged_cache(k, v, pools.table, pools.ks, pools.vs)
        ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
        out, lse = torch.zeros((3, 1, 8, d), device="cuda"), torch.zeros((3, 1, 8), device="cuda")
        B.fastkv_debug_set("paged_two_maps", int(way == "apart"))
        try:
            B.fastkv_paged_attn(cache, query, pools.dev_lens, q.cuda(), out, lse, ws)
        finally:
            B.fastkv_debug_set("paged_two_maps", 0)
        assert B.fastkv_device_status(ws) == (0, 0)
        check_attention(pools, lens, q.double().numpy(), out.cpu().double().numpy(), lse.cpu().double().numpy(), d ** -0.5)
        results.append((out.cpu(), lse.cpu()))
    for out, lse in results[1:]:
        assert torch.equal(out, results[0][0]) and torch.equal(lse, results[0][1])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_attention_reports_bad_pages_and_lengths(fmt):
    pools = Pools(fmt, [100, 60], [100, 60], 16, 2, 64, 1)
    q = bf16_rows(np.random.default_rng(0), (2, 1, 4, 64))
    query = B.make_query(n_q_heads=4, max_len=100)
    for what in ("page", "length", "negative"):
        table, lens = pools.table.clone(), pools.dev_lens.clone()
        if what == "page":
            table[0, 3] = pools.n_pages
        else:
            lens[0] = 10 ** 6 if what == "length" else -5
            table[0] = torch.where(table[0] < 0, 0, table[0])
        cache = B.make_paged_cache(pools.k, pools.v, table, pools.ks, pools.vs)
        ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
        out, lse = torch.zeros((2, 1, 4, 64), device="cuda"), torch.zeros((2, 1, 4), device="cuda")
        B.fastkv_paged_attn(cache, query, lens, q.cuda(), out, lse, ws)
        assert B.fastkv_device_status(ws)[0] == B.ERR_DEVICE_INDEX
        check_attention(pools, [100, 60], q.float().double().numpy(), out.cpu().numpy().astype(np.float64),
                        lse.cpu().numpy().astype(np.float64), 64 ** -0.5, sequences=[1])
        if what == "negative":
            assert torch.all(out[0] == 0) and torch.all(lse[0] == -math.inf)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_pools_beyond_32_bit_offsets(fmt):
    """Pages at the far end of a pool of more than 2^32 bytes: an append there, then the attention over it."""
    Hkv, d, P = 8, 128, 128
    item = 2 if fmt == "bf16" else 1
    n_pages = (2 ** 32 + 2 ** 28) // (Hkv * d * P * item)
    dtype = torch.bfloat16 if fmt == "bf16" else torch.uint8
    k, v = torch.zeros((n_pages, Hkv, P, d), dtype=dtype, device="cuda"), torch.zeros((n_pages, Hkv, P, d), dtype=dtype, device="cuda")
    ks = torch.ones((n_pages, Hkv), device="cuda") if fmt == "e4m3" else None
    vs = torch.ones((n_pages, Hkv), device="cuda") if fmt == "e4m3" else None
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device="cuda")
    cache = B.make_paged_cache(k, v, table, ks, vs)
    n = 300
    rng = np.random.default_rng(1)
    kn, vn = bf16_rows(rng, (n, Hkv, d)), bf16_rows(rng, (n, Hkv, d))
    lens, new_lens = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = workspace()
    B.fastkv_paged_append(cache, B.make_new_rows(batch=1, total=n, n_kv_heads=Hkv, head_dim=d), lens, None, kn.cuda(), vn.cuda(), None, None, None, None, new_lens, ws)
    assert B.fastkv_device_status(ws) == (0, 0)

    class Read:
        pass
    r = Read()
    r.d, r.k64, r.v64 = d, [], []
    for pool, sc, dst in ((k, ks, r.k64), (v, vs, r.v64)):
        x = pool[table[0].long()]
        x = x.float().double() if fmt == "bf16" else x.view(torch.float8_e4m3fn).float().double() * sc[table[0].long()].double()[:, :, None, None]
        dst.append(x.permute(0, 2, 1, 3).reshape(-1, Hkv, d)[:n].cpu().numpy())
    tol = 2.0 ** -8 if fmt == "bf16" else 2.0 ** -4
    assert np.all(np.abs(r.k64[0] - kn.double().numpy()) <= tol * np.abs(kn.double().numpy()) + 2.0 ** -10 * 2.0 ** -6)
    q = bf16_rows(rng, (1, 1, 32, d))
    query = B.make_query(n_q_heads=32, max_len=n)
    ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
    out, lse = torch.zeros((1, 1, 32, d), device="cuda"), torch.zeros((1, 1, 32), device="cuda")
    B.fastkv_paged_attn(cache, query, new_lens, q.cuda(), out, lse, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    check_attention(r, [n], q.float().double().numpy(), out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64), d ** -0.5)


def test_a_cache_on_another_device_is_refused():
    pools = Pools("bf16", [5], [6], 16, 1, 64, 1)
    cache = pools.cache()
    cache._index = torch.cuda.current_device() + 1
    with pytest.raises(ValueError):
        B.fastkv_paged_attn(cache, B.make_query(n_q_heads=1, max_len=5), pools.dev_lens, pools.k, pools.k, None, workspace())
    with pytest.raises(ValueError):
        B.fastkv_paged_append(cache, B.make_new_rows(batch=1, total=1, n_kv_heads=1, head_dim=64), pools.dev_lens, None, pools.k, pools.k,
                              None, None, None, None, None, workspace())


# ---- waits that run out -----------------------------------------------------------------------------------------------------
@pytest.fixture
def short_waits():
    """A poll limit of about 2 ms, and copies withheld as the test asks; the defaults afterwards."""
    def withhold(n):
        B.fastkv_debug_set("wait_limit_cycles", 4_000_000)
        B.fastkv_debug_set("paged_skip_copy", n)

    yield withhold
    B.fastkv_debug_set("wait_limit_cycles", 0)
    B.fastkv_debug_set("paged_skip_copy", 0)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("lens,n", [([3000], 1), ([3000], 2), ([90], 1), ([20000, 40, 3000], 3), ([20000, 40, 3000], 1),
                                    ([60000, 40, 3000], 2)])
def test_an_attention_whose_data_never_comes_gives_up(fmt, lens, n, short_waits):
    pools = Pools(fmt, lens, lens, 32, 2, 128, 5)
    q = bf16_rows(np.random.default_rng(5), (len(lens), 1, 8, 128))
    cache, query = pools.cache(), B.make_query(n_q_heads=8, max_len=max(lens), total_len=sum(lens))
    ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
    out, lse = torch.zeros((len(lens), 1, 8, 128), device="cuda"), torch.zeros((len(lens), 1, 8), device="cuda")
    short_waits(n)
    B.fastkv_paged_attn(cache, query, pools.dev_lens, q.cuda(), out, lse, ws)
    status, site = B.fastkv_device_status(ws)
    if n == 1 or max(lens) > 10000:                        # a short sequence's split may have no n-th chunk to withhold
        assert status == B.ERR_DEVICE_TIMEOUT
    assert (site in (39, 43)) if status == B.ERR_DEVICE_TIMEOUT else (status, site) == (0, 0)
    B.fastkv_debug_set("paged_skip_copy", 0)
    ws[:256] = 0
    B.fastkv_paged_attn(cache, query, pools.dev_lens, q.cuda(), out, lse, ws)          # and the next call is right
    assert B.fastkv_device_status(ws) == (0, 0)
    check_attention(pools, lens, q.double().numpy(), out.cpu().double().numpy(), lse.cpu().double().numpy(), 128 ** -0.5)


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("n", [1, 2, 7])
def test_an_append_whose_rows_never_come_gives_up(gather, n, short_waits):
    rng = np.random.default_rng(6)
    Hkv, d, new = 4, 128, 100
    k = bf16_rows(rng, (new, Hkv, d)).cuda()
    idx = torch.arange(new, dtype=torch.int32, device="cuda").expand(Hkv, new).contiguous() if gather else None
    rows = B.make_new_rows(batch=1, total=new, n_kv_heads=Hkv, head_dim=d, total_src=new if gather else 0)
    for withheld in (n, 0):
        pools = Pools("e4m3", [0], [new], 64, Hkv, d, 7)
        before = [t.cpu().clone() for t in (pools.k, pools.v, pools.ks, pools.vs)]
        ws = workspace()
        short_waits(withheld)
        B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, None, k, k, None, None, idx, None, None, ws)
        if withheld:
            status, site = B.fastkv_device_status(ws)
            # gathered rows come by copies that nobody waits for but the lane that asked; of tiled ones, the heads are split over
            # blocks, so that a block may have no n-th one
            assert (status, site) in ([] if n == 1 and not gather else [(0, 0)]) + ([] if gather else [(B.ERR_DEVICE_TIMEOUT, 42)])
        if not withheld or gather:
            assert B.fastkv_device_status(ws) == (0, 0)
            x = k.cpu().double().numpy()
            check_append(pools, before, [0], [new], [x], [x], False)


# ---- together -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_decoding_behind_a_selection(fmt):
    """score -> select -> the kept rows into pages -> a few decode steps (append the new token, attend), the steps replayed from
    one captured graph on a side stream; every step's output against the reference over what the pages then hold."""
    L, Hq, Hkv, d, kept, P, steps = 1500, 8, 2, 128, 150, 32, 5
    wl = W.Workload(name="paged", cfg=71, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, hidden_dim=64, window=8, pool_kernel=7,
                    pool_mode=W.POOL_AVG, seq_lens=[L], k_kv=[kept], k_tsp=None)
    x = W.make_layer(wl, with_hidden=False)
    t = lambda a: torch.from_numpy(a.view(np.int16)).cuda()  # noqa: E731
    shape = B.make_shape(total_len=L, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d)
    ws = torch.empty(B.fastkv_workspace_bytes(shape), dtype=torch.uint8, device="cuda")
    s_kv = torch.empty((Hkv, L), device="cuda")
    idx = torch.empty((Hkv, kept), dtype=torch.int32, device="cuda")
    k, v = t(x.k), t(x.v)
    B.fastkv_score(shape, t(x.q_win), k, s_kv, None, ws)
    B.fastkv_select_kv(shape, s_kv, B.make_budget(kept), idx, ws)
    pools = Pools(fmt, [0], [kept + steps], P, Hkv, d, 5)
    cache = pools.cache()
    lens, nxt = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.fastkv_paged_append(cache, B.make_new_rows(batch=1, total=kept, n_kv_heads=Hkv, head_dim=d, total_src=L), lens, None, k, v,
                          None, None, idx, None, nxt, ws)
    assert B.fastkv_device_status(ws) == (0, 0) and nxt.tolist() == [kept]
    got_k = pools.read(0, kept)[0]
    ref = W.bf16_bits_to_f32(x.k).astype(np.float64)[idx.cpu().numpy().T, np.arange(Hkv)[None]]
    assert np.all(np.abs(got_k - ref) <= (2.0 ** -8 if fmt == "bf16" else 2.0 ** -4) * np.abs(ref) + 2.0 ** -10 * need_scale(np.abs(ref).max()))
    lens.copy_(nxt)
    rows = B.make_new_rows(batch=1, total=1, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, rot_dim=d)
    query = B.make_query(n_q_heads=Hq, max_len=kept + steps)
    wa = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
    f = inv_freq(d).cuda()
    q, kn, vn = (torch.zeros((1, H, d), dtype=torch.bfloat16, device="cuda") for H in (Hq, Hkv, Hkv))
    pos = torch.full((1,), L, dtype=torch.int32, device="cuda")
    q_rot = torch.zeros_like(q)
    out, lse = torch.zeros((1, 1, Hq, d), device="cuda"), torch.zeros((1, 1, Hq), device="cuda")

    def step(s):
        B.fastkv_paged_append(cache, rows, lens, q, kn, vn, pos, f, None, q_rot, nxt, wa, s)
        B.fastkv_paged_attn(cache, query, nxt, q_rot, out, lse, wa, s)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(side)                                     # first call: one-time kernel attributes are set here
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream())
    rng = np.random.default_rng(3)
    for n in range(steps):
        fresh = [bf16_rows(rng, (1, H, d)) for H in (Hq, Hkv, Hkv)]
        for dst, src in zip((q, kn, vn), fresh):
            dst.copy_(src)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert B.fastkv_device_status(wa) == (0, 0) and nxt.tolist() == [kept + n + 1]
        pools.k64[0], pools.v64[0] = pools.read(0, kept + n + 1)
        new_k = rotate(fresh[1].double().numpy(), [L + n], inv_freq(d).numpy(), d, False)
        tol = 2.0 ** -8 if fmt == "bf16" else 2.0 ** -4
        assert np.all(np.abs(pools.k64[0][-1] - new_k[0]) <= tol * np.abs(new_k[0]) + 2.0 ** -9 * need_scale(8.0))
        check_attention(pools, [kept + n + 1], q_rot.cpu().double().numpy()[None], out.cpu().numpy().astype(np.float64),
                        lse.cpu().numpy().astype(np.float64), d ** -0.5)
        lens.copy_(nxt)
        pos.add_(1)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_sequences_may_share_pages_for_reading(fmt):
    """Three sequences whose first pages are the same ones, each with pages of its own behind them."""
    P, Hkv, d, lens = 32, 2, 128, [200, 170, 96]
    pools = Pools(fmt, lens, lens, P, Hkv, d, 3)
    for b in (1, 2):
        pools.table_np[b, :3] = pools.table_np[0, :3]
        for x in (pools.k64, pools.v64):
            x[b][:96] = x[0][:96]
    pools.table = torch.from_numpy(pools.table_np).cuda()
    q = bf16_rows(np.random.default_rng(8), (3, 2, 8, d))
    cache, query = pools.cache(), B.make_query(n_q_heads=8, q_len=2, max_len=200)
    ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
    out, lse = torch.zeros((3, 2, 8, d), device="cuda"), torch.zeros((3, 2, 8), device="cuda")
    B.fastkv_paged_attn(cache, query, pools.dev_lens, q.cuda(), out, lse, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    check_attention(pools, lens, q.double().numpy(), out.cpu().double().numpy(), lse.cpu().double().numpy(), d ** -0.5)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [5, 70])
def test_a_kept_row_may_be_named_twice(fmt, n):
    rng = np.random.default_rng(n)
    Hkv, d, src = 2, 64, 40
    k, v = (bf16_rows(rng, (src, Hkv, d)).cuda() for _ in range(2))
    idx = torch.from_numpy(rng.integers(0, src, (Hkv, n)).astype(np.int32)).cuda()
    idx[:, 1] = idx[:, 0]
    pools = Pools(fmt, [3], [3 + n], 16, Hkv, d, 2)
    before = [None if t is None else t.cpu().clone() for t in (pools.k, pools.v, pools.ks, pools.vs)]
    ws = workspace()
    B.fastkv_paged_append(pools.cache(), B.make_new_rows(batch=1, total=n, n_kv_heads=Hkv, head_dim=d, total_src=src), pools.dev_lens,
                          None, k, v, None, None, idx, None, None, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    at = idx.cpu().numpy().T
    take = lambda x: x.cpu().double().numpy()[at, np.arange(Hkv)[None]]  # noqa: E731
    check_append(pools, before, [3], [n], [take(k)], [take(v)], False)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("longest,total", [(96, 0), (200000, 1000)])
def test_an_append_behind_an_attention_waits_for_it(fmt, longest, total):
    """The entries that an attention call reads are written over by the append behind it, call after call: each attention sees
    the entries that were there when it was called.  Dealt out evenly, 37 sequences of 8 heads are one pair for every CTA, and
    the kernel behind the main one has nothing to merge."""
    n, Hkv, d, P = 37, 8, 64, 32
    pools = Pools(fmt, [96] * n, [96] * n, P, Hkv, d, 8)
    rng = np.random.default_rng(8)
    q = bf16_rows(rng, (n, 1, 2 * Hkv, d))
    cache, query = pools.cache(), B.make_query(n_q_heads=2 * Hkv, max_len=longest, total_len=total)
    ws, wa = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query)), workspace()
    first = [bf16_rows(rng, (n * 32, Hkv, d)).cuda() for _ in range(2)]
    rows = B.make_new_rows(batch=n, total=n * 32, max_new=32, n_kv_heads=Hkv, head_dim=d)
    at64 = torch.full((n,), 64, dtype=torch.int32, device="cuda")
    outs = [torch.zeros((n, 1, 2 * Hkv, d), device="cuda") for _ in range(8)]
    qd = q.cuda()
    for k, out in enumerate(outs):                                      # the last page of every sequence holds one set, the other, ...
        src = first[0] if k % 2 == 0 else first[1]
        B.fastkv_paged_append(cache, rows, at64, None, src, src, None, None, None, None, None, wa)
        B.fastkv_paged_attn(cache, query, pools.dev_lens, qd, out, None, ws)
    assert B.fastkv_device_status(ws) == (0, 0) and B.fastkv_device_status(wa) == (0, 0)
    for k in (2, 4, 6):
        assert torch.equal(outs[k], outs[0]) and torch.equal(outs[k + 1], outs[1])
    assert not torch.equal(outs[0], outs[1])


def test_graphs_may_share_a_workspace():
    """Graphs of attention calls of different shapes over one workspace, replayed by turns: each gives what it gave alone."""
    made, need = [], 0
    for lens, Hq, seed in (([5000], 8, 1), ([20000, 40, 3000, 90], 16, 2), ([60000, 40, 3000], 8, 3)):
        pools = Pools("e4m3", lens, lens, 32, 2, 128, seed)
        q = bf16_rows(np.random.default_rng(seed), (len(lens), 1, Hq, 128)).cuda()
        cache, query = pools.cache(), B.make_query(n_q_heads=Hq, max_len=max(lens), total_len=sum(lens))
        need = max(need, B.fastkv_paged_attn_workspace_bytes(cache, query))
        made.append((pools, q, cache, query, torch.zeros((len(lens), 1, Hq, 128), device="cuda")))
    ws = workspace(need)
    alone, graphs = [], []
    for pools, q, cache, query, out in made:
        B.fastkv_paged_attn(cache, query, pools.dev_lens, q, out, None, ws)
        alone.append(out.cpu())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.fastkv_paged_attn(cache, query, pools.dev_lens, q, out, None, ws)
        graphs.append(graph)
    for _ in range(10):
        for (_, _, _, _, out), graph in zip(made, graphs):
            out.zero_()
            graph.replay()
    torch.cuda.synchronize()
    assert B.fastkv_device_status(ws) == (0, 0)
    for (_, _, _, _, out), ref in zip(made, alone):
        assert torch.equal(out.cpu(), ref)


def test_calls_on_two_streams_do_not_meet():
    """Two caches with their own workspaces, their calls interleaved on two streams: the same results as one after the other."""
    made = []
    for seed in (1, 2):
        pools = Pools("e4m3", [700, 90], [701, 91], 16, 2, 128, seed)
        rng = np.random.default_rng(seed)
        q, k, v = (bf16_rows(rng, (2, H, 128)).cuda() for H in (8, 2, 2))
        made.append((pools, q, k, v))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    res = []
    for mode in ("apart", "together"):
        outs = []
        for (pools, q, k, v), s in zip(made, streams):
            s = s if mode == "together" else torch.cuda.current_stream()
            cache, query = pools.cache(), B.make_query(n_q_heads=8, max_len=701)
            with torch.cuda.stream(s):
                ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
                nl = torch.zeros(2, dtype=torch.int32, device="cuda")
                out, lse = torch.zeros((2, 1, 8, 128), device="cuda"), torch.zeros((2, 1, 8), device="cuda")
                for _ in range(20):
                    B.fastkv_paged_append(cache, B.make_new_rows(batch=2, total=2, n_kv_heads=2, head_dim=128), pools.dev_lens, None, k, v,
                                          None, None, None, None, nl, ws)
                    B.fastkv_paged_attn(cache, query, nl, q, out, lse, ws)
            outs.append((out, lse, ws))
        torch.cuda.synchronize()
        res.append([(o.cpu(), l.cpu()) for o, l, w in outs])
        assert all(B.fastkv_device_status(w) == (0, 0) for _, _, w in outs)
    for (a, la), (b, lb) in zip(*res):
        assert torch.equal(a, b) and torch.equal(la, lb)
