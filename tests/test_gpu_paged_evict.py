"""Eviction from the paged cache by accumulated weight against the rule itself: which entries stay, where they go, in which scale, and
that nothing else is touched."""
import numpy as np
import pytest
import torch

from paper_2502_01068_b200 import binding as B
from tests.paged_reference import Pools, rn_e4m3

pytestmark = pytest.mark.gpu


def origins(w, n, keep, window):
    """Slot that each kept slot's entry comes from, by the rule (NaN ranks lowest)."""
    m, cand = keep - window, n - window
    rank = [(-(-np.inf if np.isnan(x) else float(x)), not np.isnan(x), t) for t, x in enumerate(w[:cand])]
    best = set(sorted(range(cand), key=lambda t: (rank[t][0], not rank[t][1], t))[:m])
    movers = iter(t for t in range(m, cand) if t in best)
    return [t if t in best else next(movers) for t in range(m)] + list(range(cand, n))


def raw(pools):
    return [None if t is None else t.cpu().clone() for t in (pools.k, pools.v, pools.ks, pools.vs)]


def run(fmt, lens, keep, window, page, Hkv, d, seed=0, limit=None, weights=None, room=None, max_len=None, with_ids=True, pools=None):
    rng = np.random.default_rng(seed)
    limit = keep if limit is None else limit
    pools = pools or Pools(fmt, lens, room or lens, page, Hkv, d, seed + 1)
    stride = max(max(lens), 1) + 3
    w = np.exp(rng.standard_normal((len(lens), Hkv, stride))).astype(np.float32) if weights is None else weights(rng, (len(lens), Hkv, stride))
    ids = rng.integers(0, 1 << 30, w.shape).astype(np.int32)
    before = raw(pools)
    ev = B.make_eviction(keep=keep, limit=limit, window=window, max_len=max_len or max(max(lens), 1))
    cache = pools.cache()
    ws = torch.zeros(B.fastkv_paged_evict_workspace_bytes(cache, ev), dtype=torch.uint8, device="cuda")
    new_w, new_ids = torch.full(w.shape, -1.0, device="cuda"), torch.full(w.shape, -1, dtype=torch.int32, device="cuda")
    new_lens = torch.full((len(lens),), -7, dtype=torch.int32, device="cuda")
    B.fastkv_paged_evict(cache, ev, pools.dev_lens, torch.from_numpy(w).cuda(), torch.from_numpy(ids).cuda() if with_ids else None, new_w,
                         new_ids if with_ids else None, new_lens, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    after = raw(pools)
    item = lambda t: t.view(torch.int16).numpy() if fmt == "bf16" else t.view(torch.uint8).numpy()  # noqa: E731
    want = [item(t).copy() for t in before[:2]]
    want_s = [None if t is None else t.numpy().copy() for t in before[2:]]
    got_w, got_ids = new_w.cpu().numpy(), new_ids.cpu().numpy()
    for b, n in enumerate(lens):
        for g in range(Hkv):
            o = origins(w[b, g], n, keep, window) if n > limit else list(range(n))
            assert np.array_equal(got_w[b, g, :len(o)].view(np.int32), w[b, g, o].view(np.int32)) and np.all(got_w[b, g, len(o):] == -1)
            if with_ids:
                assert np.array_equal(got_ids[b, g, :len(o)], ids[b, g, o])
            assert np.all(got_ids[b, g, len(o) if with_ids else 0:] == -1)
            if n <= limit:
                continue
            at = np.array(o, dtype=np.int64)
            pages, src = pools.table_np[b, np.arange(len(o)) // page], pools.table_np[b, at // page]
            for x in range(2):
                rows = item(before[x])[src, g, at % page]
                if fmt == "e4m3":
                    was = before[2 + x].numpy()[src, g].astype(np.float64)
                    now = np.array([was[i // page * page:(i // page + 1) * page].max() for i in range(len(o))])
                    values = before[x].view(torch.float8_e4m3fn).float().numpy().astype(np.float64)[src, g, at % page]
                    codes = rn_e4m3(values * (was / now)[:, None])
                    rows = np.where((was == now)[:, None], rows, torch.from_numpy(codes).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
                    want_s[x][pages, g] = now
                want[x][pages, g, np.arange(len(o)) % page] = rows
    assert new_lens.tolist() == [keep if n > limit else n for n in lens]
    for x in range(2):
        bad = np.argwhere(item(after[x]) != want[x])
        assert len(bad) == 0, ("kv"[x], len(bad), bad[:4], [np.argwhere(pools.table_np == q).tolist() for q in sorted(set(bad[:, 0]))[:3]])
        if fmt == "e4m3":
            assert np.array_equal(after[2 + x].numpy(), want_s[x], equal_nan=True)
    return pools


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("keep,window", [(100, 8), (130, 0), (333, 333), (257, 100), (1, 0), (1, 1), (128, 16)])
def test_against_the_rule(fmt, d, page, keep, window):
    run(fmt, [700, keep + 1, keep, 3, 512], keep, window, page, 3, d, seed=keep + page)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,keep,window", [(1025, 1024, 64), (4200, 2100, 300), (9000, 8000, 3000), (20000, 1500, 128), (40000, 30000, 20000)])
def test_lengths_of_every_ranking_variant(fmt, n, keep, window):
    run(fmt, [n, n // 2], keep, window, 64, 2, 64, seed=n)


def test_candidates_beyond_the_registers():
    run("e4m3", [140000], 5000, 100, 128, 1, 64, seed=1)


@pytest.mark.parametrize("page", [16, 128])
def test_ties_zeros_and_values_at_the_ends(page):
    """Few distinct weights, -0 and 0, infinities, subnormals and NaN: equal ones stay by slot, NaN goes first."""
    def few(rng, shape):
        w = rng.choice(np.array([0.0, -0.0, 1.0, 1.0, np.inf, -np.inf, -3.0, 1e-42, np.nan], dtype=np.float32), shape)
        return w
    for seed in range(4):
        run("bf16", [500, 300, 90], 80, 10, page, 2, 64, seed=seed, weights=few)
    run("e4m3", [500, 300], 80, 10, page, 2, 64, weights=lambda rng, s: np.zeros(s, dtype=np.float32))
    run("bf16", [500, 300], 80, 10, page, 2, 64, weights=lambda rng, s: np.full(s, np.nan, dtype=np.float32))


def test_order_of_the_weights():
    """All that stay come last, and all that stay come first."""
    up = lambda rng, s: np.broadcast_to(np.arange(s[-1], dtype=np.float32), s).copy()  # noqa: E731
    for w in (up, lambda rng, s: -up(rng, s)):
        run("bf16", [1000], 300, 20, 32, 2, 64, weights=w)
        run("e4m3", [1000], 300, 20, 32, 2, 64, weights=w)


def test_limit_room_and_no_ids():
    run("bf16", [200, 201, 150], 100, 8, 16, 2, 64, limit=200, room=[300, 300, 300], with_ids=False)
    run("e4m3", [64], 64, 8, 16, 1, 64, limit=64)                       # nothing over the limit
    run("bf16", [0, 5], 3, 1, 16, 1, 64)


def test_a_batch_with_small_clusters():
    lens = [int(x) for x in np.random.default_rng(2).integers(200, 600, 96)]
    run("e4m3", lens, 256, 32, 32, 4, 64, limit=300, seed=5)


def test_sequences_it_cannot_take_are_left_and_reported():
    pools = Pools("bf16", [100, 100, 100], [112, 112, 112], 16, 1, 64, 1)
    before = raw(pools)
    lens = torch.tensor([-5, 113, 100], dtype=torch.int32, device="cuda")
    w, new_w = torch.rand(3, 1, 112, device="cuda"), torch.full((3, 1, 112), -1.0, device="cuda")
    new_lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    for max_len, taken in ((100, True), (99, False)):
        ev = B.make_eviction(keep=50, window=8, max_len=max_len)
        ws = torch.zeros(B.fastkv_paged_evict_workspace_bytes(pools.cache(), ev), dtype=torch.uint8, device="cuda")
        pools.k, pools.v = before[0].cuda(), before[1].cuda()
        B.fastkv_paged_evict(pools.cache(), ev, lens, w, None, new_w, None, new_lens, ws)
        assert B.fastkv_device_status(ws) == (B.ERR_DEVICE_INDEX, 47)
        assert new_lens.tolist() == [-5, 113, 50 if taken else 100]
        for b in (0, 1) if taken else (0, 1, 2):
            ids = torch.from_numpy(pools.table_np[b]).long()
            assert torch.equal(pools.k.cpu()[ids].view(torch.int16), before[0][ids].view(torch.int16))
        assert (new_w[:2] == -1).all()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_pages_outside_the_pool_are_reported(fmt):
    pools = Pools(fmt, [200], [200], 16, 2, 64, 1)
    good = pools.table.clone()
    ev = B.make_eviction(keep=100, window=30, max_len=200)
    for at in (1, 5, 9, 12):
        pools.table = good.clone()
        pools.table[0, at] = -1 if at % 2 else 10 ** 6
        ws = torch.zeros(B.fastkv_paged_evict_workspace_bytes(pools.cache(), ev), dtype=torch.uint8, device="cuda")
        w, new_w = torch.rand(1, 2, 200, device="cuda"), torch.zeros(1, 2, 200, device="cuda")
        B.fastkv_paged_evict(pools.cache(), ev, pools.dev_lens, w, None, new_w, None, None, ws)
        assert B.fastkv_device_status(ws) == (B.ERR_DEVICE_INDEX, 46)


def test_again_after_more_entries_and_from_a_graph():
    """Evict, append, evict: the new lengths of one call are the lengths of the next; the captured call does the same."""
    outs = []
    for captured in (False, True):
        pools = Pools("e4m3", [300, 180], [300, 300], 32, 2, 64, 7)
        cache, ev = pools.cache(), B.make_eviction(keep=150, window=16, max_len=300, limit=200)
        ws = torch.zeros(B.fastkv_paged_evict_workspace_bytes(cache, ev), dtype=torch.uint8, device="cuda")
        gen = torch.Generator(device="cuda").manual_seed(3)
        w = torch.rand(2, 2, 300, device="cuda", generator=gen)
        w2, l2 = torch.zeros_like(w), torch.zeros(2, dtype=torch.int32, device="cuda")
        w3, l3 = torch.zeros_like(w), torch.zeros(2, dtype=torch.int32, device="cuda")
        k = torch.randn(2 * 60, 2, 64, device="cuda", generator=gen).to(torch.bfloat16)
        rows = B.make_new_rows(batch=2, total=120, n_kv_heads=2, head_dim=64)
        l4 = torch.zeros(2, dtype=torch.int32, device="cuda")

        def step():
            B.fastkv_paged_evict(cache, ev, pools.dev_lens, w, None, w2, None, l2, ws)
            B.fastkv_paged_append(cache, rows, l2, None, k, k, None, None, None, None, l4, ws)
            B.fastkv_paged_evict(cache, ev, l4, w2, None, w3, None, l3, ws)
        if captured:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            graph.replay()
        else:
            step()
        assert B.fastkv_device_status(ws) == (0, 0)
        assert l2.tolist() == [150, 180] and l4.tolist() == [210, 240] and l3.tolist() == [150, 150]
        outs.append([t.clone() for t in (pools.k, pools.v, pools.ks, w2, w3)])
    for a, b in zip(*outs):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,keep,window", [([9000, 8000], 7000, 7000), ([9000], 7001, 6500), ([3000] * 30, 2500, 2500), ([700] * 40, 600, 599), ([12000], 11990, 11985)])
def test_windows_of_several_rounds(fmt, d, lens, keep, window):
    """Nothing but the window moves, or next to nothing: rounds of as many rows as shared memory holds, sources that overlap with what is
    written (by 10 slots of a page, or by none), ends inside a round and a page."""
    run(fmt, lens, keep, window, 32, 2, d, seed=keep)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,keep,window", [(16, 100, 30), (16, 96, 0), (32, 120, 120), (64, 140, 9)])
def test_rows_of_pages_outside_the_pool_stay_where_they_are(fmt, page, keep, window):
    """Every row whose page and whose source's page exist moves by the rule; nothing else is written: not page 0, not the page that the table
    named before, not the rows whose source is not to be had.  The other sequence is cut as ever."""
    lens, Hkv, d = [200, 190], 2, 64
    for at in range(-(-200 // page)):
        for bad in (-1, 10 ** 6):
            pools = Pools(fmt, lens, lens, page, Hkv, d, at + 1)
            table = pools.table_np.copy()
            table[0, at] = bad
            pools.table = torch.from_numpy(table).cuda()
            before = raw(pools)
            rng = np.random.default_rng(at)
            w = np.exp(rng.standard_normal((2, Hkv, 200))).astype(np.float32)
            ev = B.make_eviction(keep=keep, window=window, max_len=200)
            ws = torch.zeros(B.fastkv_paged_evict_workspace_bytes(pools.cache(), ev), dtype=torch.uint8, device="cuda")
            new_w, new_lens = torch.zeros(w.shape, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
            B.fastkv_paged_evict(pools.cache(), ev, pools.dev_lens, torch.from_numpy(w).cuda(), None, new_w, None, new_lens, ws)
            status = B.fastkv_device_status(ws)
            after = raw(pools)
            item = lambda t: t.view(torch.int16).numpy() if fmt == "bf16" else t.view(torch.uint8).numpy()  # noqa: E731
            want = [item(t).copy() for t in before[:2]]
            want_s = [None if t is None else t.numpy().copy() for t in before[2:]]
            touched = False
            for b, n in enumerate(lens):
                for g in range(Hkv):
                    o = np.array(origins(w[b, g], n, keep, window))
                    assert np.array_equal(new_w.cpu().numpy()[b, g, :keep], w[b, g, o])
                    to, src = table[b, np.arange(keep) // page], table[b, o // page]
                    moves = (to >= 0) & (to < pools.n_pages) & (src >= 0) & (src < pools.n_pages)
                    touched = touched or not moves[o != np.arange(keep)].all()
                    j = np.flatnonzero(moves)
                    for x in range(2):
                        rows = item(before[x])[src[j], g, o[j] % page]
                        if fmt == "e4m3":
                            was = before[2 + x].numpy()[src[j], g].astype(np.float64)
                            now = np.array([was[j // page == i // page].max() for i in j])
                            values = before[x].view(torch.float8_e4m3fn).float().numpy().astype(np.float64)[src[j], g, o[j] % page]
                            codes = torch.from_numpy(rn_e4m3(values * (was / now)[:, None])).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
                            rows = np.where((was == now)[:, None], rows, codes)
                            want_s[x][to[j], g] = now
                        want[x][to[j], g, j % page] = rows
            for x in range(2):
                assert np.array_equal(item(after[x]), want[x]), (at, bad, "kv"[x], np.argwhere(item(after[x]) != want[x])[:4])
                if fmt == "e4m3":
                    assert np.array_equal(after[2 + x].numpy(), want_s[x], equal_nan=True)
            assert new_lens.tolist() == [keep, keep]
            assert not touched or status == (B.ERR_DEVICE_INDEX, 46)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_pages_and_rows_beyond_32_bits(fmt):
    """The same entries in the last pages of pools of more than 2^32 elements, weights in rows of 2^30, and a bound beyond everything: the same."""
    lens = [300, 170]
    small = Pools(fmt, lens, lens, 16, 2, 128, 3)
    far = Pools(fmt, lens, lens, 16, 2, 128, 3)
    n, last = (1 << 32) // (2 * 16 * 128) + far.n_pages, far.n_pages
    for name in ("k", "v", "ks", "vs"):
        x = getattr(far, name)
        if x is not None:
            y = torch.empty((n, *x.shape[1:]), dtype=x.dtype, device="cuda")
            y[n - last:] = x
            setattr(far, name, y)
    far.table += torch.where(far.table >= 0, n - last, 0).to(torch.int32)
    first = torch.rand(2, 2, 300, device="cuda")
    got = []
    for pools, stride, max_len in ((small, 300, 300), (far, 1 << 30, 2 ** 31 - 1)):
        w, new_w = torch.empty(2, 2, stride, device="cuda"), torch.empty(2, 2, stride, device="cuda")
        w[:, :, :300] = first
        ev, new_lens = B.make_eviction(keep=120, window=20, max_len=max_len), torch.zeros(2, dtype=torch.int32, device="cuda")
        ws = torch.zeros(B.fastkv_paged_evict_workspace_bytes(pools.cache(), ev), dtype=torch.uint8, device="cuda")
        B.fastkv_paged_evict(pools.cache(), ev, pools.dev_lens, w, None, new_w, None, new_lens, ws)
        assert B.fastkv_device_status(ws) == (0, 0) and new_lens.tolist() == [120, 120]
        got.append([new_w[:, :, :120].clone()] + [x[-last:].clone() for x in (pools.k, pools.v, pools.ks, pools.vs) if x is not None])
        del w, new_w
    for a, b in zip(*got):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
