"""Appends so large that every block goes round its pipelines: lane groups that walk more heads than they have slots for (row role),
blocks that walk more heads of a page than they have slots for (page role, copies tiled or gathered), non-empty pages whose
entries have to be encoded again on the way.  Against the 64-bit reference; then the same with a copy withheld at every place."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2502_01068_b200 import binding as B
from tests import test_gpu_paged as T
from tests.paged_reference import Pools, need_scale, rn_e4m3
from tests.test_gpu_paged import bf16_rows, check_append, run_append, short_waits, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,Hq,d,rot,adjacent", [(2500, 32, 128, 128, False), (2500, 32, 128, 64, True), (3600, 32, 64, 64, False)])
def test_row_role_walks_more_heads_than_it_has_slots(new, Hq, d, rot, adjacent):
    """2500 tokens of 48 heads: a lane group takes 12 of them."""
    run_append("bf16", [37, 5], [new, 63], 32, Hq, 8, d, rot, adjacent, seed=new + rot)


def run_kept(fmt, lens, news, page, Hkv, d, seed, gain=1.0):
    rng = np.random.default_rng(seed)
    pools = Pools(fmt, lens, [a + b for a, b in zip(lens, news)], page, Hkv, d, seed + 1)
    before = [None if t is None else t.cpu().clone() for t in (pools.k, pools.v, pools.ks, pools.vs)]
    src = [2 * n + 3 for n in news]
    cu_src, cu = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (src, news))
    k, v = (bf16_rows(rng, (sum(src), Hkv, d), gain) for _ in range(2))
    idx = np.concatenate([np.stack([np.sort(rng.permutation(n)[:m]) for _ in range(Hkv)]) for n, m in zip(src, news)], axis=1)
    rows = B.make_new_rows(batch=len(news), total=sum(news), max_new=max(news), cu_new=torch.from_numpy(cu).cuda(), n_kv_heads=Hkv,
                           head_dim=d, total_src=sum(src), cu_src=torch.from_numpy(cu_src).cuda())
    ws = workspace()
    B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, None, k.cuda(), v.cuda(), None, None,
                          torch.from_numpy(idx.astype(np.int32)).cuda(), None, None, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    at = [cu_src[b] + idx[:, cu[b]:cu[b + 1]].T for b in range(len(news))]
    take = lambda x: [x.double().numpy()[a, np.arange(Hkv)[None]] for a in at]  # noqa: E731
    check_append(pools, before, lens, news, take(k), take(v), False)


def test_row_role_walks_more_heads_than_it_has_slots_gathered():
    """9000 kept rows: a lane group takes all 16 heads of K and V."""
    run_kept("bf16", [0, 21], [8800, 200], 32, 8, 128, 31)


# batches of so many pages that a block walks all heads of its page: (page, head_dim, KV heads, sequences, rows)
WALKS = [(16, 128, 8, 40, 100), (16, 64, 16, 40, 100), (32, 128, 8, 40, 230), (64, 128, 8, 60, 200), (64, 64, 8, 60, 200), (128, 128, 8, 50, 200)]


def lens_of(n, page):
    return [int(x) for x in np.random.default_rng(n + page).integers(0, page, n)]


def check_turned(pools, before, lens, news, k64, v64, rotated):
    """check_append for some ten million rotated values in 8-bit pages, of which a few lie next to a border between two codes.  A
    rotated value is off by at most 2^-20 max |row| before it is rounded, and rounding is monotonic: its code lies between those
    of the two ends.  V exactly as check_append has it."""
    P = pools.page
    scales = pools.ks.cpu().double().numpy()
    codes = pools.k.cpu().view(torch.float8_e4m3fn).float().double().numpy()
    raw, was = pools.k.cpu(), before[0].view(torch.uint8)
    old_scales = before[2].double().numpy()
    mine = torch.zeros(raw.shape[0], P, dtype=torch.bool)               # entries that the call may write
    for b, (n0, n) in enumerate(zip(lens, news)):
        for pg in range(n0 // P, (n0 + n - 1) // P + 1) if n else ():
            pid, first, lo, hi = int(pools.table_np[b, pg]), pg * P, max(n0, pg * P), min(n0 + n, pg * P + P)
            new = k64[b][lo - n0:hi - n0].transpose(1, 0, 2)             # [Hkv, m, d]
            slack = 2.0 ** -20 * np.abs(new).max(axis=-1, keepdims=True)
            n_old = max(0, n0 - first)
            s, top = scales[pid], np.abs(new).max(axis=(1, 2))
            for h in range(pools.Hkv):
                floor = old_scales[pid, h] if n_old else 0.0
                assert s[h] in [max(floor, need_scale(top[h] * x)) for x in (1 - 2.0 ** -20, 1 + 2.0 ** -20)]
            got, by = codes[pid, :, lo - first:hi - first], s[:, None, None]
            assert np.all(rn_e4m3((new - slack) / by) <= got) and np.all(got <= rn_e4m3((new + slack) / by)), (b, pg)
            if n_old:
                assert np.array_equal(codes[pid, :, :n_old], rn_e4m3(pools.k64[b][first:first + n_old].transpose(1, 0, 2) / by))
            mine[pid, :n_old], mine[pid, lo - first:hi - first] = True, True
    assert torch.equal(raw.transpose(1, 2)[~mine], was.transpose(1, 2)[~mine])
    touched = mine.any(dim=1).numpy()
    assert np.array_equal(scales[~touched], old_scales[~touched], equal_nan=True)
    both = SimpleNamespace(page=P, Hkv=pools.Hkv, d=pools.d, fmt=pools.fmt, table_np=pools.table_np, k=pools.v, v=pools.v, ks=pools.vs, vs=pools.vs,
                           k64=pools.v64, v64=pools.v64)
    check_append(both, [before[1], before[1], before[3], before[3]], lens, news, v64, v64, False)


@pytest.mark.parametrize("page,d,Hkv,n,new", WALKS)
@pytest.mark.parametrize("rot,adjacent", [(0, False), (1, False), (1, True)])
def test_page_role_walks_more_heads_than_it_has_slots(page, d, Hkv, n, new, rot, adjacent, monkeypatch):
    if rot:
        monkeypatch.setattr(T, "check_append", check_turned)
    news = [new - (i % 7) for i in range(n)]
    run_append("e4m3", lens_of(n, page), news, page, 2 * Hkv if adjacent else 0, Hkv, d, rot * d, adjacent, gain=8.0, seed=page + d)


@pytest.mark.parametrize("page,d,Hkv,n,new", WALKS)
def test_page_role_walks_more_heads_than_it_has_slots_gathered(page, d, Hkv, n, new):
    run_kept("e4m3", lens_of(n, page), [new - (i % 7) for i in range(n)], page, Hkv, d, page + d, gain=8.0)


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("withheld", [1, 2, 3, 6, 7, 12, 15, 16, 17])
def test_a_copy_that_never_comes_leaves_heads_whole(gather, withheld, short_waits):  # noqa: F811
    """A block of the page role takes 16 heads of its page, two a round.  The heads of the rounds before the copy that is withheld
    are appended, the others are as they were, entries and scale: no head is left between the two.  Gathered rows have no copy
    that could be withheld, and a seventeenth is none's."""
    page, Hkv, d, n, new = 64, 8, 128, 60, 200
    lens = lens_of(n, page)
    rng = np.random.default_rng(40)
    k = bf16_rows(rng, (n * new, Hkv, d), 8.0).cuda()
    idx = torch.arange(new, dtype=torch.int32, device="cuda").repeat(n).expand(Hkv, n * new).contiguous() if gather else None
    cu = torch.arange(n + 1, dtype=torch.int32, device="cuda") * new
    rows = B.make_new_rows(batch=n, total=n * new, n_kv_heads=Hkv, head_dim=d, total_src=n * new if gather else 0, cu_src=cu if gather else None)
    kept = []
    for skip in (0, withheld):
        pools = Pools("e4m3", lens, [a + new for a in lens], page, Hkv, d, 41)
        before = [t.cpu().clone().view(torch.uint8) for t in (pools.k, pools.v, pools.ks, pools.vs)]
        ws = workspace()
        short_waits(skip)
        B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, None, k, k, None, None, idx, None, None, ws)
        status = B.fastkv_device_status(ws)
        assert status == ((0, 0) if gather or skip in (0, 17) else (B.ERR_DEVICE_TIMEOUT, 42))
        kept.append([t.cpu().view(torch.uint8) for t in (pools.k, pools.v, pools.ks, pools.vs)])
    good, got = kept
    done = 2 * Hkv if gather or withheld == 17 else (withheld - 1) // 2 * 2          # heads of K, then of V, that are through
    for name, first in ((0, 0), (1, Hkv)):
        for h in range(Hkv):
            want = good if first + h < done else before
            assert torch.equal(got[name][:, h], want[name][:, h]), (name, h)
            assert torch.equal(got[2 + name].view(pools.n_pages, Hkv, 4)[:, h], want[2 + name].view(pools.n_pages, Hkv, 4)[:, h]), (name, h)
