"""Decoding behind a shared prefix with a cache that is kept short: every step appends rows, attends over prefix and own entries, adds up
the weights that the entries drew and evicts where there are too many.  Each step against the 64-bit formulas over what the pools hold,
and the steps as one graph against the same calls one by one."""
import math

import numpy as np
import pytest
import torch

from paper_2502_01068_b200 import binding as B
from tests.paged_reference import Pools, attention
from tests.test_gpu_paged_evict import origins
from tests.test_gpu_paged_weights import reference

pytestmark = pytest.mark.gpu

ROOM, STRIDE, HQ, HKV, KEEP, LIMIT, WINDOW, DECAY = 80, 80, 8, 2, 40, 56, 8, 0.75
STARTS = [30, 55, 3, 41]


class Decoder:
    """What a serving loop holds: the pools, lengths, weights and ids of the entries, and one workspace for all calls."""

    def __init__(self, fmt, d, page, T, prefix, seed):
        n = len(STARTS)
        self.fmt, self.d, self.T, self.n, self.n_prefix = fmt, d, T, n, prefix
        self.pools = Pools(fmt, [prefix] + STARTS, [prefix] + [ROOM] * n, page, HKV, d, seed)
        p = self.pools
        self.cache = B.make_paged_cache(p.k, p.v, p.table[1:].contiguous(), p.ks, p.vs)
        self.ptable, self.plen = p.table[:1].contiguous(), p.dev_lens[:1].contiguous()
        self.prefix = B.make_prefix(self.ptable, self.plen, max_len=prefix)
        self.query = B.make_query(n_q_heads=HQ, q_len=T, max_len=ROOM, total_len=n * ROOM)
        self.eviction = B.make_eviction(keep=KEEP, limit=LIMIT, window=WINDOW, max_len=ROOM)
        self.rows = B.make_new_rows(batch=n, total=n * T, n_kv_heads=HKV, head_dim=d)
        self.lens = p.dev_lens[1:].clone()
        self.grown = torch.zeros_like(self.lens)
        self.weights = torch.zeros(n, HKV, STRIDE, device="cuda")
        self.new_weights = torch.zeros_like(self.weights)
        self.ids = torch.arange(STRIDE, dtype=torch.int32, device="cuda").expand(n, HKV, STRIDE).contiguous()
        self.new_ids = torch.zeros_like(self.ids)
        self.next_id = torch.full((n, 1, 1), 1000, dtype=torch.int32, device="cuda")
        self.q, self.k, self.v = (torch.zeros(n, T, h, d, dtype=torch.bfloat16, device="cuda") for h in (HQ, HKV, HKV))
        self.out = torch.zeros_like(self.q)
        self.lse = torch.zeros(n, T, HQ, device="cuda")
        size = max(256, B.fastkv_prefix_attn_workspace_bytes(self.cache, self.prefix, self.query), B.fastkv_paged_evict_workspace_bytes(self.cache, self.eviction))
        self.ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
        self.ws[:256] = 0

    def feed(self, step):
        gen = torch.Generator(device="cuda").manual_seed(step)
        for x in (self.q, self.k, self.v):
            x.copy_(torch.randn(x.shape, device="cuda", generator=gen).to(torch.bfloat16))

    def attend(self):
        T, d = self.T, self.d
        B.fastkv_paged_append(self.cache, self.rows, self.lens, None, self.k.view(-1, HKV, d), self.v.view(-1, HKV, d), None, None, None, None, self.grown, self.ws)
        new = (self.lens[:, None] + torch.arange(T, device="cuda")).view(self.n, 1, T).expand(self.n, HKV, T)
        self.ids.scatter_(2, new, (self.next_id + torch.arange(T, dtype=torch.int32, device="cuda")).expand(self.n, HKV, T))
        self.next_id += T
        B.fastkv_prefix_attn(self.cache, self.prefix, self.query, self.grown, self.q, self.out, self.lse, self.ws)
        B.fastkv_paged_weights(self.cache, self.query, self.grown, self.q, self.lse, DECAY, self.weights, self.ws)

    def cut(self):
        B.fastkv_paged_evict(self.cache, self.eviction, self.grown, self.weights, self.ids, self.new_weights, self.new_ids, self.lens, self.ws)
        self.weights.copy_(self.new_weights)
        self.ids.copy_(self.new_ids)

    def step(self):
        self.attend()
        self.cut()

    def state(self):
        p = self.pools
        return [x.clone() for x in (p.k.view(torch.uint8), p.v.view(torch.uint8), self.lens, self.out.view(torch.int16), self.lse, self.weights, self.ids)
                ] + ([] if p.ks is None else [p.ks.clone(), p.vs.clone()])


def check_attention(dec, lens):
    """A weight is rounded to bf16 (2^-8 of it) and so is the output; a logit is off by at most d 2^-23 of sum scale |q k|, 8-bit entries of
    the prefix by scale 2^-17 max |q| sum |k| more; exponentials, sums and the merge add 2^-20."""
    p, by = dec.pools, 1.0 / math.sqrt(dec.d)
    pk, pv = p.read(0, dec.n_prefix)
    q, out, lse = (x.double().cpu().numpy() for x in (dec.q, dec.out, dec.lse))
    for b, n in enumerate(lens):
        k, v = p.read(b + 1, n)
        k, v = np.concatenate([pk, k]), np.concatenate([pv, v])
        for i in range(dec.T):
            want, want_lse, mass, size = attention(q[b, i], k, v, dec.n_prefix + n - (dec.T - 1 - i), by)
            rel = dec.d * 2.0 ** -23 * size + 2.0 ** -20
            if dec.fmt == "e4m3":
                rel = rel + by * 2.0 ** -17 * np.abs(q[b, i]).max(axis=-1) * np.repeat(np.abs(pk).sum(axis=-1).max(axis=0), HQ // HKV)
            assert np.all(np.abs(out[b, i] - want) <= 2.0 ** -8 * (mass + np.abs(want)) * 1.01 + 2 * rel[:, None] * mass)
            assert np.all(np.abs(lse[b, i] - want_lse) <= rel + 2.0 ** -21 * (np.abs(want_lse) + 1))


def check_weights(dec, before, lens):
    p = dec.pools
    now = type("Now", (), {"Hkv": HKV, "k64": [p.read(b + 1, n)[0] for b, n in enumerate(lens)]})
    want, slack = reference(now, dec.q.double().cpu().numpy(), dec.lse.double().cpu().numpy(), lens, before, DECAY, 1.0 / math.sqrt(dec.d))
    got = dec.weights.double().cpu().numpy()
    for b, n in enumerate(lens):
        assert np.all(np.abs(got[b, :, :n] - want[b, :, :n]) <= slack[b, :, :n])
        assert np.array_equal(got[b, :, n:], before[b, :, n:])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page,T", [(64, 16, 1), (128, 32, 3), (128, 16, 2)])
def test_decoding_with_eviction(fmt, d, page, T):
    dec = Decoder(fmt, d, page, T, 300, seed=d + T)
    lens, cuts = list(STARTS), 0
    for step in range(8):
        dec.feed(step)
        before = dec.weights.double().cpu().numpy()
        dec.attend()
        lens = [n + T for n in lens]
        assert dec.grown.tolist() == lens
        check_attention(dec, lens)
        check_weights(dec, before, lens)
        w, ids = dec.weights.cpu().numpy(), dec.ids.cpu().numpy()
        rows = [dec.pools.read(b + 1, n) for b, n in enumerate(lens)]
        dec.cut()
        got_w, got_ids = dec.weights.cpu().numpy(), dec.ids.cpu().numpy()
        for b, n in enumerate(lens):
            if n > LIMIT:
                cuts += 1
                lens[b] = KEEP
            k, v = dec.pools.read(b + 1, lens[b])
            for g in range(HKV):
                o = origins(w[b, g], n, KEEP, WINDOW) if n > LIMIT else list(range(n))
                assert np.array_equal(got_w[b, g, :len(o)], w[b, g, o]) and np.array_equal(got_ids[b, g, :len(o)], ids[b, g, o])
                for was, is_ in ((rows[b][0], k), (rows[b][1], v)):
                    # 8-bit pages: encoded again in the largest scale of the page's entries, at most half a step of 2^-9 of it or 2^-4 of the value off
                    slack = 0.0 if fmt == "bf16" else 2.0 ** -4 * np.abs(was[o, g]) + 2.0 ** -10 * 2.0 ** -4
                    assert np.all(np.abs(is_[:, g] - was[o, g]) <= slack)
        assert dec.lens.tolist() == lens
    assert cuts >= 1 and B.fastkv_device_status(dec.ws) == (0, 0)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_a_step_as_a_graph(fmt):
    """Six steps one by one on a stream of their own, and as a graph that is replayed, from the same state: the same bits."""
    a, b = (Decoder(fmt, 128, 16, 2, 1500, seed=7) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for step in range(6):
            a.feed(step)
            a.step()
    torch.cuda.current_stream().wait_stream(side)
    b.feed(0)
    b.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for step in range(1, 6):
        b.feed(step)
        graph.replay()
    torch.cuda.synchronize()
    for x, y in zip(a.state(), b.state()):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert a.lens.tolist() != [n + 12 for n in STARTS]                   # some were cut


def test_two_loops_at_once():
    """Two serving loops on two streams, each with pools and a workspace of its own, give what they give one after the other."""
    def loop(dec):
        for step in range(6):
            dec.feed(step)
            dec.step()

    def fresh():
        return Decoder("bf16", 64, 16, 2, 3000, seed=3), Decoder("e4m3", 128, 32, 1, 5000, seed=4)
    alone = fresh()
    for dec in alone:
        loop(dec)
    both, streams = fresh(), [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for step in range(6):
        for dec, stream in zip(both, streams):
            with torch.cuda.stream(stream):
                dec.feed(step)
                dec.step()
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        assert B.fastkv_device_status(b.ws) == (0, 0)
