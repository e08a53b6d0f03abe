"""Accumulated attention weights of paged entries against the 64-bit formula."""
import math

import numpy as np
import pytest
import torch

from paper_2502_01068_b200 import binding as B
from tests.paged_reference import Pools

pytestmark = pytest.mark.gpu


def reference(pools, q, lse, lens, old, decay, scale):
    """(weights, bound on the error): q [B, T, Hq, d] float64, lse [B, T, Hq] as given, old [B, Hkv, stride].

    A logit is off by at most d 2^-23 of sum scale |q k| (d products summed in fp32, cut off or rounded), its difference to lse and
    the exponent's scaling by 2^-23 of their size, the exponential by 2^-21; the sums and the decay by one rounding each."""
    want, slack = old.copy(), np.zeros_like(old)
    Bn, T, Hq, d = q.shape
    G = Hq // pools.Hkv
    for b in range(Bn):
        n = lens[b]
        k = pools.k64[b][:n]
        for g in range(pools.Hkv):
            w, e = np.zeros(n), np.zeros(n)
            for i in range(T):
                sees = max(0, n - (T - 1 - i))
                for h in range(g * G, (g + 1) * G):
                    if lse[b, i, h] == -np.inf:
                        continue
                    x = scale * (k[:sees, g] @ q[b, i, h])
                    size = scale * (np.abs(k[:sees, g]) @ np.abs(q[b, i, h]))
                    p = np.exp(x - lse[b, i, h])
                    w[:sees] += p
                    e[:sees] += p * (d * 2.0 ** -23 * size + 2.0 ** -22 * (np.abs(x) + abs(lse[b, i, h])) + 2.0 ** -21)
            first = max(0, n - T)
            w[:first] += decay * old[b, g, :first]
            want[b, g, :n] = w
            slack[b, g, :n] = e + (T * G + 4) * 2.0 ** -24 * w + 2.0 ** -120
    return want, slack


def lse_of(pools, q, lens, scale):
    Bn, T, Hq, d = q.shape
    G = Hq // pools.Hkv
    out = np.full((Bn, T, Hq), -np.inf)
    for b in range(Bn):
        for i in range(T):
            sees = lens[b] - (T - 1 - i)
            for h in range(Hq):
                if sees > 0:
                    x = scale * (pools.k64[b][:sees, h // G] @ q[b, i, h])
                    out[b, i, h] = x.max() + math.log(np.exp(x - x.max()).sum())
    return out.astype(np.float32)


def workspace():
    return torch.zeros(256, dtype=torch.uint8, device="cuda")


def run(fmt, lens, page, Hq, Hkv, d, T=1, decay=1.0, seed=0, stride=None, scale=0.0, gain=1.0, total_len=None):
    rng = np.random.default_rng(seed)
    pools = Pools(fmt, lens, lens, page, Hkv, d, seed + 1)
    q = torch.from_numpy(rng.standard_normal((len(lens), T, Hq, d)) * gain).to(torch.bfloat16)
    q64 = q.double().numpy()
    by = scale or 1.0 / math.sqrt(d)
    lse = lse_of(pools, q64, lens, by)
    stride = stride or max(max(lens), 1) + 5
    old = np.exp(rng.standard_normal((len(lens), Hkv, stride))).astype(np.float32)
    for b, n in enumerate(lens):                          # what may not be read: NaN
        old[b, :, max(0, n - T):] = np.nan
    w = torch.from_numpy(old).cuda()
    ws = workspace()
    query = B.make_query(n_q_heads=Hq, q_len=T, max_len=max(max(lens), 1), total_len=sum(lens) if total_len is None else total_len,
                         softmax_scale=scale)
    B.fastkv_paged_weights(pools.cache(), query, pools.dev_lens, q.cuda(), torch.from_numpy(lse).cuda(), decay, w, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    want, slack = reference(pools, q64, lse.astype(np.float64), lens, old.astype(np.float64), float(np.float32(decay)), by)
    got = w.cpu().double().numpy()
    for b, n in enumerate(lens):
        assert np.array_equal(got[b, :, n:], old[b, :, n:].astype(np.float64), equal_nan=True), "rows behind the end"
        bad = ~(np.abs(got[b, :, :n] - want[b, :, :n]) <= slack[b, :, :n])
        assert not bad.any(), (b, np.argwhere(bad)[:5], got[b, :, :n][bad][:5], want[b, :, :n][bad][:5])
    return got


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv,T", [(4, 1, 1), (6, 2, 1), (8, 8, 3), (32, 4, 2), (14, 2, 5)])
def test_against_the_formula(fmt, d, page, Hq, Hkv, T):
    run(fmt, [1, 257, 16, 700, 33], page, Hq, Hkv, d, T, decay=0.75, seed=page + T)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [0, 1, 15, 127, 128, 129, 255, 511, 512, 513, 1500])
def test_lengths(fmt, n):
    run(fmt, [n], 16, 4, 1, 128, seed=n)
    run(fmt, [3, n, 0, 40], 32, 4, 2, 64, T=2, seed=n)


def test_many_sequences_and_a_bound_that_is_off():
    lens = [int(x) for x in np.random.default_rng(5).integers(0, 90, 300)]
    run("bf16", lens, 16, 2, 2, 64, seed=9)
    run("e4m3", lens, 16, 2, 1, 128, seed=9, total_len=1)


def test_query_tokens_ahead_of_the_cache():
    """More query tokens than entries: the first ones see nothing, their lse is -infinity and they draw nothing."""
    run("bf16", [2, 1, 0, 5], 16, 4, 2, 64, T=4, seed=3)


def test_scale_and_sharp_rows():
    run("bf16", [300], 16, 8, 2, 128, scale=0.5, gain=4.0, seed=4)
    run("e4m3", [300], 16, 8, 2, 128, scale=0.25, gain=4.0, seed=4)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_what_a_query_does_not_see_never_reaches_a_weight(fmt):
    """The last token's key is NaN: the first query token's row has no part of it."""
    pools = Pools(fmt, [40], [40], 16, 1, 64, 1)
    pid = int(pools.table_np[0, 39 // 16])
    (pools.k if fmt == "bf16" else pools.k.view(torch.float8_e4m3fn))[pid, :, 39 % 16] = float("nan")
    q = torch.randn(1, 2, 2, 64, device="cuda").to(torch.bfloat16)
    lse = torch.tensor([[[0.0, 0.0], [0.0, -math.inf]]], device="cuda")
    w, ws = torch.zeros(1, 1, 40, device="cuda"), workspace()
    B.fastkv_paged_weights(pools.cache(), B.make_query(n_q_heads=2, q_len=2, max_len=40), pools.dev_lens, q, lse, 1.0, w, ws)
    x = w[0, 0].cpu()
    assert torch.isfinite(x[:39]).all() and torch.isnan(x[39])


def test_reports_and_keeps_to_its_rows():
    pools = Pools("bf16", [100, 50], [100, 50], 16, 1, 64, 1)
    pools.table[0, 1] = 10 ** 6
    lens = torch.tensor([1000, 50], dtype=torch.int32, device="cuda")           # beyond the table's room of 112
    q = torch.randn(2, 1, 2, 64, device="cuda").to(torch.bfloat16)
    w, ws = torch.full((2, 1, 60), 7.0, device="cuda"), workspace()
    B.fastkv_paged_weights(pools.cache(), B.make_query(n_q_heads=2, max_len=112), lens, q, torch.zeros(2, 1, 2, device="cuda"), 1.0, w, ws)
    assert B.fastkv_device_status(ws)[0] == B.ERR_DEVICE_INDEX
    assert (w[1, 0, 50:] == 7.0).all() and not (w[1, 0, :50] == 7.0).any()


def test_same_bits_twice_on_a_stream_and_from_a_graph():
    pools = Pools("e4m3", [900, 40, 333], [900, 40, 333], 32, 2, 128, 1)
    q = torch.randn(3, 2, 8, 128, device="cuda").to(torch.bfloat16)
    lse = torch.full((3, 2, 8), 4.0, device="cuda")
    query = B.make_query(n_q_heads=8, q_len=2, max_len=900, total_len=1273)
    first = torch.rand(3, 2, 900, device="cuda")
    cache, ws = pools.cache(), workspace()
    a = first.clone()
    B.fastkv_paged_weights(cache, query, pools.dev_lens, q, lse, 0.5, a, ws)
    b, side = first.clone(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.fastkv_paged_weights(cache, query, pools.dev_lens, q, lse, 0.5, b, ws)
    torch.cuda.current_stream().wait_stream(side)
    c = first.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.fastkv_paged_weights(cache, query, pools.dev_lens, q, lse, 0.5, c, ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("pairs", [1, 2, 4])
@pytest.mark.parametrize("Hq,Hkv,T", [(4, 2, 1), (6, 2, 5), (6, 2, 9)])
def test_steps_of_a_unit(fmt, d, pairs, Hq, Hkv, T):
    """One, two and four pairs of steps a unit (the bound on the lengths decides), with ends in every step of them; rows of one tile of
    eight, two and more."""
    lens = [1, 31, 32, 33, 65, 127, 128, 129, 255, 257, 0, 511, 513, 700, 1023, 1500, 2049]
    run(fmt, lens, 16, Hq, Hkv, d, T, decay=0.5, seed=T, total_len={1: 10 ** 4, 2: 3 * 1776 * 256 // Hkv, 4: 10 ** 8}[pairs] * (2 if d == 64 else 1))


def test_a_bound_beyond_everything():
    run("bf16", [300, 20], 16, 4, 2, 64, seed=1, total_len=2 ** 63 - 1)
    run("e4m3", [300, 20], 16, 4, 2, 128, seed=1, total_len=2 ** 62)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,T", [(2, 2, 1), (4, 1, 1), (8, 2, 1), (10, 2, 1), (8, 1, 1), (8, 2, 3), (4, 1, 4), (7, 1, 3)])
def test_infinite_and_nan_keys(fmt, d, Hq, Hkv, T):
    """Entries with one infinite element (bf16; NaN in both formats): logits of -infinity draw 0, those of +infinity infinity, NaN gives NaN, where
    every row sees the step and where the last entries cut it; rows 1 to 21, tiles of eight with and without padding.  Nothing else changes."""
    rng = np.random.default_rng(d + Hq + T)
    n, by = 700, 1.0 / math.sqrt(d)
    values = [float("nan")] if fmt == "e4m3" else [-math.inf, math.inf, float("nan")]
    slots = [0, 17, 100, 255, 256, 511, 600, 697, 698, 699]
    for signs in (1.0, None):                             # all queries meet them with one sign, or with either
        for value in values:
            pools = Pools(fmt, [n], [n], 16, Hkv, d, 5)
            k64 = pools.k64[0].copy()
            for t in slots:
                page = int(pools.table_np[0, t // 16])
                (pools.k if fmt == "bf16" else pools.k.view(torch.float8_e4m3fn))[page, :, t % 16, 3] = value
                k64[t, :, 3] = value
            q = rng.standard_normal((1, T, Hq, d))
            q[..., 3] = 1.0 if signs else np.sign(q[..., 3])
            q = torch.from_numpy(q).to(torch.bfloat16)
            q64 = q.double().numpy()
            lse = lse_of(pools, q64, [n], by)             # of the entries without them
            old = np.exp(rng.standard_normal((1, Hkv, n))).astype(np.float32)
            w, ws = torch.from_numpy(old).cuda(), workspace()
            B.fastkv_paged_weights(pools.cache(), B.make_query(n_q_heads=Hq, q_len=T, max_len=n), pools.dev_lens, q.cuda(), torch.from_numpy(lse).cuda(), 0.5, w, ws)
            assert B.fastkv_device_status(ws) == (0, 0)
            want, slack = reference(pools, q64, lse.astype(np.float64), [n], old.astype(np.float64), 0.5, by)
            pools.k64[0] = k64
            with np.errstate(invalid="ignore"):
                there, _ = reference(pools, q64, lse.astype(np.float64), [n], old.astype(np.float64), 0.5, by)
            want[:, :, slots], slack[:, :, slots] = there[:, :, slots], 2.0 ** -22 * old[:, :, slots]
            got = w.cpu().double().numpy()
            finite = np.isfinite(want)
            assert np.array_equal(np.where(finite, 0, got), np.where(finite, 0, want), equal_nan=True), (value, np.argwhere(~finite & (got != want))[:4])
            assert np.all(np.abs(got[finite] - want[finite]) <= slack[finite])
            if value == -math.inf and signs:              # drew nothing: the old weight's half, exactly
                assert np.array_equal(got[0][:, slots[:-3]], old[0][:, slots[:-3]] * 0.5)


def test_rows_of_infinite_lse():
    """A row whose lse is +infinity draws nothing from finite logits, and has no part in what it does not see."""
    n, d = 256, 64
    pools = Pools("bf16", [n], [n], 16, 1, d, 1)
    pools.k[int(pools.table_np[0, (n - 1) // 16]), 0, (n - 1) % 16, 0] = math.inf
    q = torch.ones(1, 2, 2, d, device="cuda", dtype=torch.bfloat16)
    lse = torch.tensor([[[math.inf, math.inf], [10.0, 11.0]]], device="cuda")
    w, ws = torch.zeros(1, 1, n, device="cuda"), workspace()
    B.fastkv_paged_weights(pools.cache(), B.make_query(n_q_heads=2, q_len=2, max_len=n), pools.dev_lens, q, lse, 1.0, w, ws)
    x = w[0, 0].cpu().double().numpy()
    logit = 0.125 * pools.k64[0][:n - 1, 0].sum(axis=-1)
    # a logit and its difference to lse are off by at most 64 2^-23 sum |k| / 8 + 2^-22 (|x| + 11) < 2^-12
    want = np.exp(logit - 10.0) + np.exp(logit - 11.0)
    assert np.abs(pools.k64[0][:n - 1]).sum(axis=-1).max() < 128 and np.all(np.abs(x[:-1] - want) <= 2.0 ** -12 * want)
    assert x[-1] == math.inf                              # of the second token's rows; the first token's do not see it


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_pages_and_rows_beyond_32_bits(fmt):
    """The same entries in the last pages of pools of more than 2^32 elements, weights in rows of 2^30: the same bits."""
    pools = Pools(fmt, [300, 70], [300, 70], 16, 2, 128, 3)
    q = torch.randn(2, 1, 8, 128, device="cuda").to(torch.bfloat16)
    lse, query, ws = torch.full((2, 1, 8), 4.0, device="cuda"), B.make_query(n_q_heads=8, max_len=300), workspace()
    old = torch.rand(2, 2, 300, device="cuda")
    want = old.clone()
    B.fastkv_paged_weights(pools.cache(), query, pools.dev_lens, q, lse, 0.5, want, ws)
    n, k = (1 << 32) // (2 * 16 * 128) + pools.n_pages, pools.k
    pools.k = torch.empty((n, *k.shape[1:]), dtype=k.dtype, device="cuda")
    pools.k[n - pools.n_pages:] = k
    pools.v = pools.k                                     # (not read)
    if fmt == "e4m3":
        ks = pools.ks
        pools.ks = torch.empty((n, 2), device="cuda")
        pools.ks[n - pools.n_pages:] = ks
        pools.vs = pools.ks
    pools.table += torch.where(pools.table >= 0, n - pools.n_pages, 0).to(torch.int32)
    got = torch.empty(2, 2, 1 << 30, device="cuda")
    got[:, :, :300] = old
    B.fastkv_paged_weights(pools.cache(), query, pools.dev_lens, q, lse, 0.5, got, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    assert torch.equal(got[:, :, :300], want)
