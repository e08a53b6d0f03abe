"""Accumulated weights and eviction, host side without a GPU: what the calls refuse before they touch a device, and workspaces."""
import math

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


def weights_call(c=None, query=None, lens=0x1000, q=0x2000, lse=0x3000, decay=1.0, weights=0x4000, stride=64, ws=0x100000, nbytes=256):
    query = query or B.make_query(n_q_heads=8, max_len=64)
    return B._load().fastkv_paged_weights(c or plain(n_kv_heads=2), query, lens, q, lse, decay, weights, stride, ws, nbytes, None)


def test_weights_refuses():
    for kw in (dict(lens=None), dict(q=None), dict(lse=None), dict(weights=None), dict(decay=-0.5), dict(decay=math.nan), dict(decay=math.inf),
               dict(stride=0), dict(stride=-1), dict(query=B.make_query(n_q_heads=7, max_len=64)), dict(query=B.make_query(n_q_heads=8, max_len=0)),
               dict(query=B.make_query(n_q_heads=8, max_len=64, q_len=0)), dict(query=B.make_query(n_q_heads=8, max_len=64, softmax_scale=-1.0))):
        assert weights_call(**kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(q=0x2008), dict(stride=(1 << 31) + 1), dict(c=plain(n_kv_heads=2, head_dim=96)), dict(c=plain(n_kv_heads=2, batch=40000))):
        assert weights_call(**kw) == B.ERR_UNSUPPORTED, kw
    for kw in (dict(ws=None), dict(ws=0x100010), dict(nbytes=255)):
        assert weights_call(**kw) == B.ERR_WORKSPACE, kw


def test_rows_of_entries_end_well_before_32_bits():
    """A length is cut to the row, and a warp's first entry of the next unit has to be a positive number still."""
    for call in (weights_call, evict_call):
        assert call(stride=(1 << 30) + 1, nbytes=0) == B.ERR_UNSUPPORTED
    assert weights_call(stride=1 << 30, nbytes=0) == B.ERR_WORKSPACE
    far = dict(weights=1 << 40, ids=2 << 40, new_weights=3 << 40, new_ids=4 << 40)
    assert evict_call(stride=1 << 30, nbytes=0, **far) == B.ERR_WORKSPACE


def evict_call(c=None, ev=None, lens=0x1000, weights=0x10000, ids=0x20000, stride=64, new_weights=0x30000, new_ids=0x40000, new_lens=0x2000, ws=0x100000,
               nbytes=1 << 20):
    ev = ev or B.make_eviction(keep=16, max_len=64)
    return B._load().fastkv_paged_evict(c or plain(n_kv_heads=2, batch=1), ev, lens, weights, ids, stride, new_weights, new_ids, new_lens, ws, nbytes, None)


def test_evict_refuses():
    ev = B.make_eviction
    for kw in (dict(lens=None), dict(weights=None), dict(new_weights=None), dict(ids=None), dict(new_ids=None), dict(stride=0),
               dict(ev=ev(keep=0, max_len=64, window=0)), dict(ev=ev(keep=16, limit=15, max_len=64)), dict(ev=ev(keep=16, window=17, max_len=64)),
               dict(ev=ev(keep=16, window=-1, max_len=64)), dict(ev=ev(keep=16, max_len=0)), dict(new_weights=0x10000), dict(new_weights=0x10100),
               dict(new_weights=0x20000 - 4), dict(new_ids=0x20040), dict(new_ids=0x30000), dict(new_lens=0x1000)):
        assert evict_call(**kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(c=plain(n_kv_heads=2, batch=40000)), dict(c=plain(n_kv_heads=2, page_size=8)), dict(stride=(1 << 31) + 1)):
        assert evict_call(**kw) == B.ERR_UNSUPPORTED, kw
    need = B.fastkv_paged_evict_workspace_bytes(plain(n_kv_heads=2, batch=1), ev(keep=16, max_len=64))
    for kw in (dict(ws=None), dict(ws=0x100080), dict(nbytes=need - 1)):
        assert evict_call(**kw) == B.ERR_WORKSPACE, kw


def test_evict_workspace():
    size = lambda **kw: B.fastkv_paged_evict_workspace_bytes(plain(n_kv_heads=8, batch=3), B.make_eviction(**kw))  # noqa: E731
    assert size(keep=100, max_len=100) == 256 and size(keep=100, limit=200, max_len=150) == 256           # nothing to cut
    assert 256 + 24 * 4 * (2 * 92 + 1) <= size(keep=100, max_len=101) <= 256 + 24 * 4 * (4 * 92 + 4) + 255
    assert size(keep=100, window=100, max_len=1000) <= 256 + 24 * 16 + 255
    assert size(keep=2 ** 31 - 1, window=0, max_len=2 ** 31 - 1) == 256


def test_binding_checks_its_tensors(monkeypatch):
    c = plain(n_kv_heads=2, batch=3)
    monkeypatch.setattr(B, "_here", lambda cache: 0)
    c._device = torch.device("cpu")
    ok = torch.zeros(3, 2, 64)
    bad = [torch.zeros(2, 2, 64), torch.zeros(3, 1, 64), torch.zeros(3, 2), ok.double(), torch.zeros(3, 64, 2).transpose(1, 2)]
    for w in bad:
        with pytest.raises(ValueError):
            B.fastkv_paged_weights(c, None, None, None, None, 1.0, w, None)
        with pytest.raises(ValueError):
            B.fastkv_paged_evict(c, None, None, w, None, ok, None, None, None)
        with pytest.raises(ValueError):
            B.fastkv_paged_evict(c, None, None, ok, None, w, None, None, None)
    for x in (torch.zeros(3, 2, 63), torch.zeros(3, 2, 64, dtype=torch.int64)):
        with pytest.raises(ValueError):
            B.fastkv_paged_evict(c, None, None, ok, x, ok.clone(), x, None, None)
