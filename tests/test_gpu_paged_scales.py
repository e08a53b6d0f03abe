"""Attention over 8-bit pages whose scales of V lie far apart: every column of the output against its own sum of p |v|, so that
a page that is large in some columns and zero in the others hides nothing in those others.

The bounds are those of tests/test_gpu_paged.py, column by column.  They hold here because a step's weights count from the step's
own largest logit (in 22 bits) and meet the scale of its page, a power of two, in 32 bits only."""
import numpy as np
import pytest
import torch

from paper_2502_01068_b200 import binding as B
from tests.paged_reference import Pools, attention
from tests.test_gpu_paged import bf16_rows, check_attention, workspace

pytestmark = pytest.mark.gpu

LENS = [600, 40, 0, 131]
SHAPES = [(66, 0), (600, 0), (200000, 771)]                    # whole, split, dealt out


def attend(pools, lens, q, scale=0.0):
    """The three ways a call is laid out, each against the reference."""
    cache = pools.cache()
    T, Hq, d = q.shape[1:]
    for longest, total in SHAPES:
        query = B.make_query(n_q_heads=Hq, q_len=T, max_len=longest, total_len=total, softmax_scale=scale)
        ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
        out, lse = (torch.full(s, 7.0, device="cuda") for s in ((len(lens), T, Hq, d), (len(lens), T, Hq)))
        dev_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        B.fastkv_paged_attn(cache, query, dev_lens, q.cuda(), out, lse, ws)
        assert B.fastkv_device_status(ws) == (0, 0)
        check_attention(pools, lens, q.double().numpy(), out.cpu().double().numpy(), lse.cpu().double().numpy(), scale or d ** -0.5)


def pages_of(pools, b, n, where):
    last = -(-n // pools.page) - 1
    return [int(pools.table_np[b, {"first": 0, "middle": last // 2, "last": last}[where]])] if n else []


def mirror(pools, lens):
    for b, n in enumerate(lens):
        pools.k64[b], pools.v64[b] = pools.read(b, n)


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("delta", [20, 28, 40, 80, 150])
@pytest.mark.parametrize("page,d,T", [(16, 128, 1), (64, 128, 1), (64, 64, 1), (16, 64, 3), (32, 128, 5)])
def test_columns_that_a_large_page_leaves_to_the_others(where, delta, page, d, T):
    pools = Pools("e4m3", LENS, LENS, page, 2, d, 21, v_exp=(-40, -38))
    for b, n in enumerate(LENS):
        for pid in pages_of(pools, b, n, where):
            pools.vs[pid] *= 2.0 ** (delta // 2)               # in two steps: a factor is an fp32 number
            pools.vs[pid] *= 2.0 ** (delta // 2)
            pools.v[pid, :, :, ::2] &= 0x80                    # zeros of either sign
    mirror(pools, LENS)
    assert all(np.isfinite(x).all() for x in pools.v64)
    attend(pools, LENS, bf16_rows(np.random.default_rng(5), (len(LENS), T, 8, d)))


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("page,d,T", [(16, 128, 1), (64, 128, 4), (32, 64, 1)])
def test_a_large_page_of_little_weight(where, page, d, T):
    """The other way round: entries with some 2^-49 of the weight and 2^60 of the others' size make up the result."""
    pools = Pools("e4m3", LENS, LENS, page, 2, d, 22)
    pools.k[:, :, :, 0] &= 0x80
    for b, n in enumerate(LENS):
        for pid in pages_of(pools, b, n, where):
            pools.vs[pid] *= 2.0 ** 60
            pools.ks[pid] = 2.0 ** -3
            pools.k[pid] = 0
            pools.k[pid, :, :, 0] = torch.tensor(-272.0).to(torch.float8_e4m3fn).view(torch.uint8).item()
    mirror(pools, LENS)
    q = bf16_rows(np.random.default_rng(6), (len(LENS), T, 8, d), 0.1)
    q[..., 0] = 1.0
    attend(pools, LENS, q, scale=1.0)


@pytest.mark.parametrize("page,d,T", [(16, 128, 1), (64, 128, 3), (32, 64, 1)])
def test_small_entries_of_little_weight(page, d, T):
    """One page has all the weight, but zeros in every other column: there the others count alone, with 2^-63 of the weight and 2^-30 of
    the usual scale, which fp32 holds."""
    pools = Pools("e4m3", LENS, LENS, page, 2, d, 26, v_exp=(-30, -28))
    pools.ks[:] = 2.0 ** -3
    pools.k[:] = 0
    pools.k[:, :, :, 0] = torch.tensor(-352.0).to(torch.float8_e4m3fn).view(torch.uint8).item()
    for b, n in enumerate(LENS):
        for pid in pages_of(pools, b, n, "middle"):
            pools.k[pid, :, :, 0] = 0
            pools.v[pid, :, :, ::2] &= 0x80
    mirror(pools, LENS)
    q = bf16_rows(np.random.default_rng(6), (len(LENS), T, 8, d), 0.1)
    q[..., 0] = 1.0
    attend(pools, LENS, q, scale=1.0)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("n,at", [(1, 0), (70, 3), (70, 69)])
def test_an_appended_infinity_costs_its_own_page_alone(page, n, at):
    """Its page takes the largest scale and keeps nothing else; the entries of the other pages stay in the other columns."""
    lens = [300, 37]
    pools = Pools("e4m3", lens, [a + n for a in lens], page, 2, 128, 23)
    rng = np.random.default_rng(7)
    k, v = (bf16_rows(rng, (2 * n, 2, 128)) for _ in range(2))
    v[at, 0, 5] = float("inf")
    ws = workspace()
    rows = B.make_new_rows(batch=2, total=2 * n, n_kv_heads=2, head_dim=128)
    B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, None, k.cuda(), v.cuda(), None, None, None, None, None, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    lens = [a + n for a in lens]
    pools.lens = lens
    mirror(pools, lens)
    assert pools.v64[0].max() == 448.0 * 2.0 ** 120
    attend(pools, lens, bf16_rows(rng, (2, 1, 8, 128)))


@pytest.mark.parametrize("page,d,T", [(16, 128, 1), (64, 128, 1), (128, 64, 3)])
@pytest.mark.parametrize("scale", [0.0, 2.0])
def test_columns_that_single_entries_fill(page, d, T, scale):
    """Within a page: every column of V holds one entry in 32, most often one of little weight.  The weights of a step of 32 entries
    (16 for pages of 16) go in as two terms in fp16, 2^15 times too large, the step's largest being 2^15: each term is off by at most
    half of fp16's smallest step, 2^-25, so that a weight is off by at most 2 * 2^-25 / 2^15 = 2^-39 of the largest: that much of it
    times the step's |v| is added to the bound."""
    pools = Pools("e4m3", LENS, LENS, page, 2, d, 24)
    rng = np.random.default_rng(25)
    alone = torch.from_numpy(rng.random(tuple(pools.v.shape)) < 1 / 32).cuda()
    pools.v[~alone] &= 0x80
    mirror(pools, LENS)
    q = bf16_rows(rng, (len(LENS), T, 8, d))
    cache, s, step = pools.cache(), scale or d ** -0.5, 16 if page == 16 else 32
    for longest, total in SHAPES:
        query = B.make_query(n_q_heads=8, q_len=T, max_len=longest, total_len=total, softmax_scale=scale)
        ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
        out, lse = (torch.full(x, 7.0, device="cuda") for x in ((len(LENS), T, 8, d), (len(LENS), T, 8)))
        B.fastkv_paged_attn(cache, query, pools.dev_lens, q.cuda(), out, lse, ws)
        assert B.fastkv_device_status(ws) == (0, 0)
        out = out.cpu().double().numpy()
        for b, n in enumerate(LENS):
            for i in range(T):
                sees = n - (T - 1 - i)
                if sees <= 0:
                    continue
                ref, ref_lse, mass, size = attention(q[b, i].double().numpy(), pools.k64[b], pools.v64[b], sees, s)
                delta = (d / 16 + 8) * 2.0 ** -23 * size[:, None] + 2.0 ** -23 * np.abs(ref_lse)[:, None]
                tol = (2 * delta + 2.0 ** -20 + (sees / 16 + 16) * 2.0 ** -23) * mass + 1e-30
                for h in range(8):
                    x = s * (pools.k64[b][:sees, h // 4] @ q[b, i, h].double().numpy())
                    p = np.exp(x - ref_lse[h])
                    for t in range(0, sees, step):
                        tol[h] += 2.0 ** -39 * p[t:t + step].max() * np.abs(pools.v64[b][t:t + step, h // 4]).sum(axis=0)
                assert np.all(np.abs(out[b, i] - ref) <= tol), (b, i, float((np.abs(out[b, i] - ref) / tol).max()))
