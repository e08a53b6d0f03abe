"""Attention over shared prefixes and the sequences' own entries against the 64-bit formula."""
import math

import numpy as np
import pytest
import torch

from paper_2502_01068_b200 import binding as B
from tests.paged_reference import Pools, attention

pytestmark = pytest.mark.gpu


class Shared:
    """Prefixes and sequences in one pool: rows 0 .. n - 1 of the pools' table are the prefixes'."""

    def __init__(self, fmt, plens, lens, page, Hkv, d, seed, cu=None):
        self.pools = Pools(fmt, list(plens) + list(lens), list(plens) + list(lens), page, Hkv, d, seed)
        n = len(plens)
        self.n, self.plens, self.lens, self.cu = n, list(plens), list(lens), cu
        self.ptable, self.table = self.pools.table[:n].contiguous(), self.pools.table[n:].contiguous()
        self.dev_plens, self.dev_lens = self.pools.dev_lens[:n].contiguous(), self.pools.dev_lens[n:].contiguous()
        self.dev_cu = None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda")

    def cache(self):
        p = self.pools
        return B.make_paged_cache(p.k, p.v, self.table, p.ks, p.vs)

    def prefix(self, max_len=None):
        return B.make_prefix(self.ptable, self.dev_plens, max_len=max_len or max(1, max(self.plens)), cu_seqs=self.dev_cu)

    def prefix_of(self, b):
        if self.cu is None:
            return 0
        return next((i for i in range(self.n) if self.cu[i] <= b < self.cu[i + 1]), None)

    def entries(self, b):
        i, p = self.prefix_of(b), self.pools
        k, v = p.k64[self.n + b], p.v64[self.n + b]
        if i is None:
            return 0, k, v
        return self.plens[i], np.concatenate([p.k64[i], k]), np.concatenate([p.v64[i], v])


def call(sh, q, scale=0.0, lse=True, max_len=None, own_max=None, total_len=None, stream=None, ws=None):
    Bn, T, Hq, d = q.shape
    cache, prefix = sh.cache(), sh.prefix(max_len)
    query = B.make_query(n_q_heads=Hq, q_len=T, max_len=own_max or max(1, max(sh.lens)), total_len=sum(sh.lens) if total_len is None else total_len,
                         softmax_scale=scale)
    if ws is None:
        # what a workspace holds is anything but its header
        ws = torch.full((B.fastkv_prefix_attn_workspace_bytes(cache, prefix, query),), 0xFF, dtype=torch.uint8, device="cuda")
        ws[:256] = 0
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    l = torch.full((Bn, T, Hq), float("nan"), device="cuda") if lse else None
    B.fastkv_prefix_attn(cache, prefix, query, sh.dev_lens, q, out, l, ws, stream)
    return out, l, ws


def check(sh, q, out, lse, scale=0.0, rows=None):
    """A weight is rounded to bf16 (2^-8 of it) and so is the output; a logit is off by at most d 2^-23 of sum scale |q k|, which moves
    weights and their sum; exponentials, sums and the merge add 2^-20.  8-bit entries: an element of q below 2^-9 of its row's largest is off by
    at most 2^-17 of that, which moves a logit of the prefix by at most scale 2^-17 max |q| sum |k|."""
    Bn, T, Hq, d = q.shape
    by = scale or 1.0 / math.sqrt(d)
    q64, o64 = q.double().cpu().numpy(), out.double().cpu().numpy()
    l64 = None if lse is None else lse.double().cpu().numpy()
    for b, i in rows or [(b, i) for b in range(Bn) for i in range(T)]:
        n, k, v = sh.entries(b)
        sees = n + max(0, sh.lens[b] - (T - 1 - i))
        want, want_lse, mass, size = attention(q64[b, i], k, v, sees, by)
        rel = d * 2.0 ** -23 * size + 2.0 ** -20
        if sh.pools.fmt == "e4m3" and n > 0:
            rel = rel + by * 2.0 ** -17 * np.abs(q64[b, i]).max(axis=-1) * np.repeat(np.abs(k[:n]).sum(axis=-1).max(axis=0), Hq // sh.pools.Hkv)
        slack = 2.0 ** -8 * (mass + np.abs(want)) * 1.01 + 2 * rel[:, None] * mass
        bad = ~(np.abs(o64[b, i] - want) <= slack)
        assert not bad.any(), (b, i, np.argwhere(bad)[:4], o64[b, i][bad][:4], want[bad][:4])
        if l64 is not None:
            for h in range(Hq):
                if sees == 0:
                    assert l64[b, i, h] == -np.inf
                else:
                    assert abs(l64[b, i, h] - want_lse[h]) <= rel[h] + 2.0 ** -21 * (abs(want_lse[h]) + 1), (b, i, h, l64[b, i, h], want_lse[h])


def run(fmt, plens, lens, page, Hq, Hkv, d, T=1, cu=None, seed=0, scale=0.0, gain=1.0, rows=None, **kw):
    sh = Shared(fmt, plens, lens, page, Hkv, d, seed, cu)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q = (torch.randn(len(lens), T, Hq, d, device="cuda", generator=gen) * gain).to(torch.bfloat16)
    out, lse, ws = call(sh, q, scale, **kw)
    assert B.fastkv_device_status(ws) == (0, 0)
    check(sh, q, out, lse, scale, rows)
    return sh, q, out, lse


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 127, 128, 129, 300, 1000, 0])
def test_lengths_of_the_prefix(fmt, d, n):
    run(fmt, [n], [5, 1, 40], 16, 4, 1, d, seed=n)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv,T", [(8, 8, 1), (6, 2, 2), (14, 2, 1), (8, 1, 5), (12, 4, 3)])
def test_against_the_formula(fmt, page, Hq, Hkv, T):
    run(fmt, [777], [3, 90, 17, 1], page, Hq, Hkv, 128, T, seed=page + T)
    run(fmt, [500], [30, 9], page, Hq, Hkv, 64, T, seed=page + T)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch,Hq,Hkv,T", [(32, 4, 1, 1), (33, 4, 1, 1), (64, 4, 1, 1), (65, 4, 1, 1), (40, 8, 2, 2), (70, 3, 1, 3), (300, 1, 1, 1), (3, 64, 1, 2),
                                            (2, 128, 1, 1), (2, 100, 1, 2)])
def test_row_tiles(fmt, batch, Hq, Hkv, T):
    """One tile, two, pairs of them with a ragged last one; heads that do not divide a tile."""
    run(fmt, [1500], [1 + (7 * b) % 23 for b in range(batch)], 32, Hq, Hkv, 128, T, seed=batch, rows=[(b, b % T) for b in range(0, batch, max(1, batch // 12))] + [(batch - 1, T - 1)])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_several_prefixes(fmt, d):
    """Prefixes of all lengths, one that nobody uses, one of length 0, sequences before the first and behind the last."""
    run(fmt, [400, 77, 1300, 0, 128], [4, 30, 1, 9, 60, 2, 7, 8, 33, 5, 12], 16, 8, 2, d, T=2, cu=[1, 4, 4, 7, 8, 10], seed=3)
    run(fmt, [90, 4000], [4] * 80, 64, 4, 1, d, cu=[0, 70, 80], seed=4, rows=[(0, 0), (31, 0), (32, 0), (69, 0), (70, 0), (79, 0)])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_many_prefixes(fmt):
    rng = np.random.default_rng(2)
    cu = np.concatenate([[0], np.cumsum(rng.integers(0, 4, 200))]).tolist()
    run(fmt, [int(x) for x in rng.integers(0, 300, 200)], [int(x) for x in rng.integers(0, 20, cu[-1])], 16, 2, 1, 64, cu=cu, seed=5,
        rows=[(b, 0) for b in range(0, cu[-1], 9)])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_long_prefix_on_every_sm(fmt):
    run(fmt, [40000], [100, 3, 800, 64], 64, 16, 4, 128, seed=6)
    run(fmt, [20000], [9] * 70, 128, 4, 1, 128, seed=7, rows=[(0, 0), (63, 0), (64, 0), (69, 0)])


def test_nothing_to_see():
    """No prefix and no entries of one's own, query tokens ahead of the cache, a prefix alone."""
    sh, q, out, lse = run("bf16", [0], [0, 3, 1], 16, 4, 2, 64, T=3, seed=1)
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    run("e4m3", [200], [0, 0], 16, 4, 2, 64, T=2, seed=1, total_len=1)


def test_scale_and_sharp_rows():
    """Logits of a hundred: the reference moves, earlier sums and outputs are rescaled."""
    for fmt in ("bf16", "e4m3"):
        run(fmt, [3000], [50] * 3, 32, 8, 2, 128, scale=0.5, gain=3.0, seed=8)
        run(fmt, [3000], [50] * 40, 32, 8, 2, 128, scale=0.5, gain=3.0, seed=9, rows=[(0, 0), (20, 0), (39, 0)])


def test_bounds_that_are_off():
    run("bf16", [900], [70, 3], 16, 4, 2, 64, max_len=10, own_max=1, total_len=1, seed=2)
    run("e4m3", [900], [70, 3], 16, 4, 2, 64, max_len=10 ** 6, own_max=10 ** 6, total_len=0, seed=2, lse=False)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,batch", [(64, 2), (128, 2), (128, 40)])
def test_nan_and_infinities_where_they_are_seen(fmt, d, batch):
    """The pools' other entries, those behind the prefix in its last page among them, are NaN in every test; here one entry of the
    prefix, too: its sequences' rows get it, and no other's."""
    sh = Shared(fmt, [200, 333], [9] * batch, 32, 2, d, 3, cu=[0, batch // 2, batch])
    pid = int(sh.pools.table_np[0, 70 // 32])
    for pool in (sh.pools.k, sh.pools.v):
        x = pool if fmt == "bf16" else pool.view(torch.float8_e4m3fn)
        x[pid, 0, 70 % 32, 5] = float("nan")
    q = torch.randn(batch, 1, 8, d, device="cuda").to(torch.bfloat16)
    out, lse, ws = call(sh, q)
    assert B.fastkv_device_status(ws) == (0, 0)
    half = batch // 2
    assert torch.isnan(out[:half, :, :4]).all() and torch.isnan(lse[:half, :, :4]).all()
    check(sh, q, out, lse, rows=[(half, 0), (batch - 1, 0)])
    assert not torch.isnan(out[:half, :, 4:]).any() and not torch.isnan(lse[:half, :, 4:]).any()


def test_entries_that_weigh_nothing():
    """Logits of -infinity in the whole prefix: only the own entries count; in all entries: like a query that sees none."""
    sh = Shared("bf16", [300], [20, 20], 16, 1, 64, 3)
    q = torch.ones(2, 1, 2, 64, device="cuda").to(torch.bfloat16)
    for row in range(19):
        sh.pools.k[int(sh.pools.table_np[0, row])][0, :] = -math.inf
    out, lse, ws = call(sh, q)
    n, k, v = sh.entries(0)
    want, want_lse, _, _ = attention(q[0, 0].double().cpu().numpy(), k[n:], v[n:], 20, 0.125)
    assert np.allclose(lse[0, 0].double().cpu().numpy(), want_lse, rtol=1e-5) and np.allclose(out[0, 0].double().cpu().numpy(), want, rtol=2.0 ** -8, atol=1e-5)
    sh.pools.k[sh.table[0].long()] = -math.inf
    out, lse, ws = call(sh, q)
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()


def test_reports():
    sh = Shared("bf16", [300, 90], [20, 20], 16, 1, 64, 3, cu=[0, 1, 2])
    q = torch.randn(2, 1, 2, 64, device="cuda").to(torch.bfloat16)
    good = sh.ptable.clone()
    for bad in (-1, 10 ** 6):
        sh.ptable = good.clone()
        sh.ptable[0, 3] = bad
        assert B.fastkv_device_status(call(sh, q)[2]) == (B.ERR_DEVICE_INDEX, 58)
    sh.ptable = good
    for n in (-1, 16 * good.shape[1] + 1):
        sh.dev_plens[0] = n
        assert B.fastkv_device_status(call(sh, q)[2]) == (B.ERR_DEVICE_INDEX, 59)
    sh.dev_plens[0] = 300
    for cu in ([0, 2, 1], [-1, 1, 2], [0, 1, 3], [5, 1, 0]):
        sh.dev_cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
        assert B.fastkv_device_status(call(sh, q)[2]) == (B.ERR_DEVICE_INDEX, 60)
    sh.dev_cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    out, lse, ws = call(sh, q)
    assert B.fastkv_device_status(ws) == (0, 0)
    check(sh, q, out, lse)


def test_groups_that_overlap_have_no_room():
    """A cu_seqs that goes back and forth would name every sequence many times over."""
    n = 64
    sh = Shared("bf16", [150] * n, [3] * 8, 16, 1, 64, 3, cu=[0, 8] * (n // 2) + [8])
    q = torch.randn(8, 1, 128, 64, device="cuda").to(torch.bfloat16)
    out, lse, ws = call(sh, q)
    assert B.fastkv_device_status(ws) == (B.ERR_DEVICE_INDEX, 60)


def test_same_bits_twice_on_a_stream_and_from_a_graph():
    for fmt in ("bf16", "e4m3"):
        sh = Shared(fmt, [5000, 333], [40, 9, 300, 5], 32, 2, 128, 1, cu=[0, 3, 4])
        q = torch.randn(4, 2, 8, 128, device="cuda").to(torch.bfloat16)
        a, la, ws = call(sh, q)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            b, lb, _ = call(sh, q, stream=side, ws=ws)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c, lc, _ = call(sh, q, ws=ws)
            e, le, _ = call(sh, q, ws=ws)                  # two calls share a workspace in one graph
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in ((a, b), (a, c), (a, e)):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))
        assert torch.equal(la, lb) and torch.equal(la, lc) and torch.equal(la, le)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch", [2, 140])
def test_a_wait_that_runs_out(fmt, batch):
    """A completion that is never signalled: the waits for it run out, the kernel ends, and the next call is whole.  (Of few rows the second
    chunk is the other tile's.)"""
    sh = Shared(fmt, [30000, 600], [9] * batch, 32, 2, 128, 3, cu=[0, batch // 2, batch])
    q = torch.randn(batch, 1, 8, 128, device="cuda").to(torch.bfloat16)
    for n in (1, 2, 3):
        B.fastkv_debug_set("wait_limit_cycles", 2_000_000)
        B.fastkv_debug_set("prefix_skip_commit", n)
        try:
            _, _, ws = call(sh, q)
            status, site = B.fastkv_device_status(ws)
        finally:
            B.fastkv_debug_set("wait_limit_cycles", 0)
            B.fastkv_debug_set("prefix_skip_commit", 0)
        if n == 2 and batch == 2:
            assert (status, site) == (0, 0)
        else:
            assert status == B.ERR_DEVICE_TIMEOUT and 48 <= site <= 57
        out, lse, ws = call(sh, q)
        assert B.fastkv_device_status(ws) == (0, 0)
        check(sh, q, out, lse, rows=[(0, 0), (batch - 1, 0)])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch,T", [(60, 4), (40, 4), (50, 2), (32, 1)])
def test_merge_by_one_to_eight_warps(fmt, batch, T):
    """Rows for every number of warps that share a row's pieces out, over prefixes of very different lengths: CTAs that end inside what a
    unit counts for besides its chunks, units of one chunk, a prefix without entries and one without sequences."""
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(T, 60, batch)]
    cu = [1, 6, 7, 7 + batch // 6, batch // 2, batch // 2, batch - 2]
    rows = [(b, int(rng.integers(T))) for b in sorted({0, 1, 5, 6, 7, batch // 2 - 1, batch // 2, batch - 3, batch - 1})]
    run(fmt, [3000, 1, 5000, 0, 129, 2000], lens, 16, 32, 8, 128, T, cu=cu, seed=batch, rows=rows)
    run(fmt, [3000, 1, 5000, 0, 129, 2000], lens, 32, 16, 8, 64, T, cu=cu, seed=batch, rows=rows)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_one_prefix_for_some_of_the_sequences(fmt):
    run(fmt, [700], [9, 3, 30, 1, 17], 16, 8, 2, 128, 2, cu=[1, 4])
    run(fmt, [40000], [9, 3, 30, 1, 17], 64, 8, 2, 128, 1, cu=[2, 5])
    run(fmt, [700], [9, 3], 16, 8, 2, 64, 1, cu=[1, 1])


@pytest.mark.parametrize("batch", [3, 60])
def test_nan_and_infinite_keys_of_every_column(batch):
    """Two row tiles share an SM (or one has it): whichever way a weight's exponential is taken, a NaN key reaches every output, a key whose
    logits are -infinity none, one of +infinity makes its row NaN."""
    for col in (0, 1, 2, 3, 5, 6, 7, 62, 63, 64, 100, 127, 130):
        sh = Shared("bf16", [131], [2] * batch, 16, 1, 64, col)
        q = torch.ones(batch, 1, 4, 64, device="cuda", dtype=torch.bfloat16)
        page, row = sh.ptable[0, col // 16].long(), col % 16
        keep = sh.pools.k[page, 0, row].clone()
        for value in (float("nan"), -math.inf, math.inf):
            sh.pools.k[page, 0, row] = keep
            sh.pools.k[page, 0, row, 0] = value
            out, lse, ws = call(sh, q)
            assert B.fastkv_device_status(ws) == (0, 0)
            if value == -math.inf:
                without = sh.pools.k64[0].copy()
                without[col, 0] = -1e6                    # (weighs nothing either)
                k = np.concatenate([without, sh.pools.k64[1]])
                v = np.concatenate([sh.pools.v64[0], sh.pools.v64[1]])
                want, want_lse, mass, size = attention(q[0, 0].double().cpu().numpy(), np.delete(k, col, 0), np.delete(v, col, 0), 132, 0.125)
                rel = 64 * 2.0 ** -23 * size + 2.0 ** -20
                got = out[0, 0].double().cpu().numpy()
                assert np.all(np.abs(got - want) <= 2.0 ** -8 * (mass + np.abs(want)) * 1.01 + 2 * rel[:, None] * mass)
                assert np.all(np.abs(lse[0, 0].double().cpu().numpy() - want_lse) <= rel + 2.0 ** -21 * (np.abs(want_lse) + 1))
            else:
                assert torch.isnan(out).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_merge_by_sixteen_and_more_warps(fmt, d):
    """Few rows and a piece of them on every SM: 16 warps share them out, or 32."""
    run(fmt, [20000], [5] * (40 if d == 128 else 80), 64, 8, 2, d, seed=1, rows=[(0, 0), (7, 0), (8, 0), (31, 0), (39, 0)])
    run(fmt, [20000], [5, 1, 300], 64, 7, 1, d, T=2, seed=2)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch", [3, 50])
def test_values_next_to_the_end_of_the_range(fmt, batch):
    """V up to 2^125: a weight is never above 1 and a row's largest starts at 2^-16 or below, so the running output of 2000 entries, which is
    not divided by their sum yet, stays finite."""
    sh = Shared(fmt, [2000], [4] * batch, 32, 2, 128, 5)
    if fmt == "bf16":
        sh.pools.v *= 2.0 ** 122
    else:
        sh.pools.vs *= 2.0 ** 119
    sh.pools.v64 = [x * 2.0 ** (122 if fmt == "bf16" else 119) for x in sh.pools.v64]
    q = (torch.randn(batch, 1, 8, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) * 0.25).to(torch.bfloat16)
    out, lse, ws = call(sh, q)
    assert B.fastkv_device_status(ws) == (0, 0) and torch.isfinite(out).all()
    check(sh, q, out, lse, rows=[(b, 0) for b in range(0, batch, 7)])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,T,longest", [(1, 1, 128), (4, 25, 128), (4, 1, 700), (4, 60, 700)])
def test_shares_of_many_short_segments(fmt, d, G, T, longest):
    """Hundreds of prefixes of a chunk each, or of a few: a CTA's share is a row of short segments, many of which leave one of its two row tiles
    without chunks, and ends in one of them.  Again and again, with memory busy on another stream: the same bits."""
    rng = np.random.default_rng(longest + T)
    n = 400
    sh = Shared(fmt, [int(x) for x in rng.integers(1, longest + 1, n)], [int(x) for x in rng.integers(T, T + 9, n)], 16, 8, d, 3, list(range(n + 1)))
    q = torch.randn(n, T, 8 * G, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).to(torch.bfloat16)
    first, lse, ws = call(sh, q)
    assert B.fastkv_device_status(ws) == (0, 0)
    check(sh, q, first, lse, rows=[(b, b % T) for b in range(0, n, 13)] + [(n - 1, T - 1)])
    side, a, b = torch.cuda.Stream(), torch.zeros(1 << 28, dtype=torch.uint8, device="cuda"), torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(40):
            b.copy_(a)
    for _ in range(10):
        out, l, ws = call(sh, q)
        assert B.fastkv_device_status(ws) == (0, 0)
        assert torch.equal(out.view(torch.int16), first.view(torch.int16)) and torch.equal(l, lse)
    torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch,n,heavy", [(3, 128, 3), (50, 128, 3), (3, 128, 64), (50, 300, 30), (2, 16000, 15900), (70, 16000, 15900)])
def test_values_at_the_end_of_the_range_and_logits_that_rise(fmt, batch, n, heavy):
    """The last entries' logits are 2^15 times the first ones' in weight, which is below what moves a row's reference, and all values of the
    prefix are the largest of bf16 (8 bits: 224 * 2^120): their sum before the division has to stay finite."""
    d, scale = 64, math.log(2.0)
    sh = Shared(fmt, [n], [4] * batch, 16, 1, d, 5)
    p = sh.pools
    top = float(torch.finfo(torch.bfloat16).max) if fmt == "bf16" else 224.0 * 2.0 ** 120
    pages = sh.ptable[0].long()
    k, v = torch.zeros(n, d), torch.full((n, d), top if fmt == "bf16" else 224.0)
    k[n - heavy:, 0] = 15.0
    v[1::2, ::3] *= -1
    for page0 in range(0, n, 16):
        m, page = min(16, n - page0), pages[page0 // 16]
        for pool, x in ((p.k, k), (p.v, v)):
            pool[page, 0, :m] = (x[page0:page0 + m].to(torch.bfloat16) if fmt == "bf16" else x[page0:page0 + m].to(torch.float8_e4m3fn).view(torch.uint8)).cuda()
    if fmt == "e4m3":
        p.ks[pages], p.vs[pages] = 1.0, 2.0 ** 120
    p.k64[0], p.v64[0] = k[:, None].double().numpy(), (v[:, None].double() * (1.0 if fmt == "bf16" else 2.0 ** 120)).numpy()
    q = torch.zeros(batch, 1, 4, d, device="cuda", dtype=torch.bfloat16)
    q[..., 0] = 1.0
    out, lse, ws = call(sh, q, scale)
    assert B.fastkv_device_status(ws) == (0, 0) and torch.isfinite(out).all()
    check(sh, q, out, lse, scale, rows=[(b, 0) for b in range(0, batch, 7)])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch", [3, 70])
def test_own_values_at_the_end_of_the_range(fmt, batch):
    """One's own entry weighs 2^16 times an entry of the prefix, and all values are next to the end of the range: so is the sum of both parts."""
    n, d, scale = 16000, 64, math.log(2.0)
    sh = Shared(fmt, [n], [1] * batch, 16, 1, d, 5)
    p, top = sh.pools, float(torch.finfo(torch.bfloat16).max) if fmt == "bf16" else 224.0 * 2.0 ** 120
    if fmt == "bf16":
        p.v = torch.where(torch.isnan(p.v), p.v, torch.full_like(p.v, top))
        p.k = torch.where(torch.isnan(p.k), p.k, torch.zeros_like(p.k))
    else:
        p.v = torch.where(p.v == 0x7F, p.v, torch.full_like(p.v, 0x76))                   # 224
        p.k = torch.where(p.k == 0x7F, p.k, torch.zeros_like(p.k))
        p.vs, p.ks = torch.full_like(p.vs, 2.0 ** 120), torch.ones_like(p.ks)
    p.k[sh.table[:, 0].long(), 0, 0, 0] = 16.0 if fmt == "bf16" else 0x58                 # (16)
    p.v64 = [np.full_like(x, top) for x in p.v64]
    p.k64 = [np.zeros_like(p.k64[0])] + [np.full_like(x, 16.0) * (np.arange(d) == 0) for x in p.k64[1:]]
    q = torch.ones(batch, 1, 4, d, device="cuda", dtype=torch.bfloat16)
    out, lse, ws = call(sh, q, scale)
    assert B.fastkv_device_status(ws) == (0, 0) and torch.isfinite(out).all()
    check(sh, q, out, lse, scale, rows=[(b, 0) for b in range(0, batch, 29)])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,Hq,cu", [(64, 128, None), (4, 8, [0, 8, 0, 8, 2]), (3, 8, [8, 0, 8, 4]), (64, 8, None), (5, 4, [-3, 20, 1, 7, 3, 100])])
def test_groups_that_overlap_stay_in_their_buffers(fmt, n, Hq, cu):
    """Whatever cu_seqs says: nothing is written behind the workspace, the outputs and the lse, or in front of them, and sequences are all
    there is to write to."""
    sh = Shared(fmt, [150] * n, [3] * 8, 16, 1, 64, 3, cu=cu or [0, 8] * (n // 2) + [8])
    cache, prefix, query = sh.cache(), sh.prefix(), B.make_query(n_q_heads=Hq, max_len=3, total_len=24)
    q = torch.randn(8, 1, Hq, 64, device="cuda").to(torch.bfloat16)
    size, edge = B.fastkv_prefix_attn_workspace_bytes(cache, prefix, query), 4096

    def guarded(nbytes):
        x = torch.full((nbytes + 2 * edge,), 0x5A, dtype=torch.uint8, device="cuda")
        return x, x[edge:edge + nbytes]
    (all_ws, ws), (all_out, out), (all_lse, lse) = guarded(size), guarded(8 * Hq * 64 * 2), guarded(8 * Hq * 4)
    ws[:256] = 0
    pools = [x.clone() for x in (sh.pools.k, sh.pools.v)]
    B.fastkv_prefix_attn(cache, prefix, query, sh.dev_lens, q, out.view(torch.bfloat16), lse.view(torch.float32), ws)
    assert B.fastkv_device_status(ws) == (B.ERR_DEVICE_INDEX, 60)
    for x in (all_ws, all_out, all_lse):
        assert (x[:edge] == 0x5A).all() and (x[-edge:] == 0x5A).all()
    for x, y in zip(pools, (sh.pools.k, sh.pools.v)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch,Hq,Hkv,T,lens", [(2, 8, 2, 300, [300, 512]), (3, 5, 1, 129, [700, 64, 0]), (1, 32, 8, 512, [512]), (4, 4, 4, 65, [65, 66, 64, 1])])
def test_many_query_tokens(fmt, batch, Hq, Hkv, T, lens):
    """A prompt's chunk behind the prefix: hundreds of query tokens, some ahead of what their sequence holds."""
    rows = [(b, i) for b in range(batch) for i in sorted({0, 1, T // 2, T - 65, T - 2, T - 1})]
    run(fmt, [900], lens, 32, Hq, Hkv, 128, T, seed=T, rows=rows)
    run(fmt, [130, 257], lens, 16, Hq, Hkv, 64, T, seed=T, cu=[0, batch // 2, batch], rows=rows)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_the_most_prefixes(fmt):
    rng = np.random.default_rng(3)
    cu = [1] + (1 + np.cumsum(rng.integers(0, 3, 1024))).tolist()
    run(fmt, [int(x) for x in rng.integers(0, 200, 1024)], [int(x) for x in rng.integers(0, 20, cu[-1] + 1)], 32, 4, 2, 64, cu=cu, seed=5,
        rows=[(b, 0) for b in range(0, cu[-1] + 1, 31)] + [(cu[-1], 0)])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_pages_beyond_32_bits(fmt):
    """The same entries in the last pages of pools of more than 2^32 elements: the same bits."""
    sh = Shared(fmt, [300, 70], [20, 9, 40], 16, 2, 128, 3, cu=[0, 2, 3])
    q = torch.randn(3, 2, 8, 128, device="cuda").to(torch.bfloat16)
    want, want_lse, _ = call(sh, q)
    p = sh.pools
    n = (1 << 32) // (2 * 16 * 128) + p.n_pages
    for name in ("k", "v", "ks", "vs"):
        x = getattr(p, name)
        if x is not None:
            far = torch.empty((n, *x.shape[1:]), dtype=x.dtype, device="cuda")
            far[n - p.n_pages:] = x
            setattr(p, name, far)
    for table in (sh.ptable, sh.table):
        table += torch.where(table >= 0, n - p.n_pages, 0).to(torch.int32)
    out, lse, ws = call(sh, q)
    assert B.fastkv_device_status(ws) == (0, 0)
    assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("batch", [3, 50])
def test_queries_that_are_not_finite_keep_to_themselves(fmt, batch):
    """A NaN in one head's query, an infinity in another's: their own outputs are NaN (keys of either sign meet them), all others as ever."""
    sh = Shared(fmt, [400], [9] * batch, 16, 2, 128, 3)
    q = torch.randn(batch, 2, 8, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
    want, want_lse, _ = call(sh, q)
    bad = q.clone()
    bad[1, 0, 2, 7], bad[1, 1, 5, 127], bad[batch - 1, 1, 0, 0] = float("nan"), math.inf, -math.inf
    out, lse, ws = call(sh, bad)
    assert B.fastkv_device_status(ws) == (0, 0)
    hit = torch.zeros(batch, 2, 8, dtype=torch.bool, device="cuda")
    hit[1, 0, 2] = hit[1, 1, 5] = hit[batch - 1, 1, 0] = True
    assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
    assert torch.equal(out[~hit].view(torch.int16), want[~hit].view(torch.int16)) and torch.equal(lse[~hit], want_lse[~hit])
