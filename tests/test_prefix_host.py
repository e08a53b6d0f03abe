"""Shared-prefix attention, host side without a GPU: refusals and workspaces."""
import random

import pytest
import torch

from paper_2502_01068_b200 import binding as B
from paper_2502_01068_b200 import build
from tests.test_paged_host import cache


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build_library()


def plain(**kw):
    return cache(format=B.CACHE_BF16, k_scales=None, v_scales=None, **kw)


def prefix(**kw):
    p = B.Prefix()
    args = dict(n_prefixes=1, max_pages=16, max_len=1000, reserved=0, table=0x1000, lens=0x2000, cu_seqs=None)
    args.update(kw)
    for k, v in args.items():
        setattr(p, k, v)
    return p


def call(c=None, x=None, query=None, lens=0x3000, q=0x4000, out=0x8000, lse=None, ws=0x100000, nbytes=1 << 40):
    query = query or B.make_query(n_q_heads=8, max_len=64)
    return B._load().fastkv_prefix_attn(c or plain(n_kv_heads=2), x or prefix(), query, lens, q, out, lse, ws, nbytes, None)


def test_refusals():
    for kw in (dict(lens=None), dict(q=None), dict(out=None), dict(x=prefix(n_prefixes=0)), dict(x=prefix(max_pages=0)), dict(x=prefix(max_len=0)),
               dict(x=prefix(reserved=1)), dict(x=prefix(table=None)), dict(x=prefix(lens=None)), dict(x=prefix(n_prefixes=2)),
               dict(query=B.make_query(n_q_heads=7, max_len=64)), dict(query=B.make_query(n_q_heads=8, max_len=64, q_len=0)),
               dict(query=B.make_query(n_q_heads=8, max_len=64, softmax_scale=float("nan")))):
        assert call(**kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(q=0x4008), dict(out=0x8008), dict(x=prefix(n_prefixes=1025, cu_seqs=0x5000)), dict(x=prefix(max_pages=1 << 30)),
               dict(query=B.make_query(n_q_heads=258, max_len=64)), dict(c=plain(n_kv_heads=2, page_size=8))):
        assert call(**kw) == B.ERR_UNSUPPORTED, kw
    c, x, q = plain(n_kv_heads=2), prefix(), B.make_query(n_q_heads=8, max_len=64)
    need = B.fastkv_prefix_attn_workspace_bytes(c, x, q)
    for kw in (dict(ws=None), dict(ws=0x100010), dict(nbytes=need - 1)):
        assert call(**kw) == B.ERR_WORKSPACE, kw
    assert B._load().fastkv_prefix_attn(c, None, q, 0x3000, 0x4000, 0x8000, None, 0x100000, need, None) == B.ERR_INVALID_ARG
    assert B._load().fastkv_prefix_attn_workspace_bytes(c, x, q, None) == B.ERR_INVALID_ARG


def test_rows_of_the_table_end_well_before_32_bits():
    """Pages are looked up two chunks ahead: the entry's number has to stay positive."""
    c = plain(n_kv_heads=2)
    most = (1 << 30) // c.page_size
    assert call(c=c, x=prefix(max_pages=most + 1), nbytes=0) == B.ERR_UNSUPPORTED
    assert call(c=c, x=prefix(max_pages=most), nbytes=0) == B.ERR_WORKSPACE


def test_workspace_holds_every_piece():
    """At most one piece for every pair of row tiles and CTA boundary, whatever the groups."""
    rng = random.Random(1)
    for _ in range(500):
        batch, hkv, G, T = rng.randint(1, 80), rng.choice([1, 2, 8]), rng.choice([1, 3, 4, 7, 128]), rng.choice([1, 2, 5])
        n, d = rng.randint(1, 20), rng.choice([64, 128])
        c = plain(n_kv_heads=hkv, batch=batch, head_dim=d)
        size = B.fastkv_prefix_attn_workspace_bytes(c, prefix(n_prefixes=n, cu_seqs=0x5000, max_len=rng.randint(1, 100000)), B.make_query(n_q_heads=hkv * G, q_len=T, max_len=9))
        cuts = sorted(rng.randint(0, batch) for _ in range(n + 1))
        tile = 128 // G
        units = hkv * sum(-(-(b - a) * T // (2 * tile)) for a, b in zip(cuts, cuts[1:]))
        rows = -(-min(batch * T * G, tile * G) // 32) * 32
        assert size >= 256 + batch * T * hkv * G * (d + 1) * 4 + units * 2 * rows * (d + 2) * 4
        assert size % 256 == 0


def test_binding_checks_its_tensors():
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    B.make_prefix(i32(2, 3), i32(2), max_len=5, cu_seqs=i32(3))
    for args in ((i32(6), i32(2), None), (i32(2, 3).long(), i32(2), None), (i32(2, 3), i32(3), None), (i32(2, 3), i32(2).long(), None), (i32(2, 3), i32(2), i32(2)),
                 (i32(3, 2).t(), i32(2), None)):
        with pytest.raises(ValueError):
            B.make_prefix(args[0], args[1], max_len=5, cu_seqs=args[2])
