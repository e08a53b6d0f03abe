"""What the header says of the paged cache beside the arithmetic: the lengths that an append reports, the rows of a padded batch, a
query whose logits are all minus infinity, and how large an attention's workspace can get."""
import math

import numpy as np
import pytest
import torch

from paper_2502_01068_b200 import binding as B
from tests.paged_reference import Pools
from tests.test_gpu_paged import bf16_rows, check_append, check_attention, inv_freq, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("bad", ["page", "index"])
def test_refused_rows_keep_their_slots(fmt, n, bad):
    """A row that is refused for its page id or its index takes up its slot all the same: new_lens counts it, the rows behind it
    stand where they belong, and the status says that not every slot was written."""
    Hkv, d, P = 2, 64, 16
    pools = Pools(fmt, [5, 3], [5 + n, 3 + n], P, Hkv, d, 9)
    k = bf16_rows(np.random.default_rng(4), (2 * n, Hkv, d))
    idx = None
    cu = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
    if bad == "page":
        pools.table[0, :] = pools.n_pages
    else:
        idx = torch.arange(n, dtype=torch.int32, device="cuda").repeat(2).expand(Hkv, 2 * n).contiguous()
        idx[:, 0] = n
    rows = B.make_new_rows(batch=2, total=2 * n, n_kv_heads=Hkv, head_dim=d, total_src=0 if idx is None else 2 * n, cu_src=None if idx is None else cu)
    before = pools.k.cpu().clone()
    new_lens, ws = torch.zeros(2, dtype=torch.int32, device="cuda"), workspace()
    B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, None, k.cuda(), k.cuda(), None, None, idx, None, new_lens, ws)
    assert B.fastkv_device_status(ws)[0] == B.ERR_DEVICE_INDEX
    assert new_lens.tolist() == [5 + n, 3 + n]
    tol = 2.0 ** -8 if fmt == "bf16" else 2.0 ** -4
    x = k.double().numpy()
    near = lambda got, want: np.all(np.abs(got - want) <= tol * np.abs(want) + 2.0 ** -10 * 2.0 ** -4)  # noqa: E731
    assert near(pools.read(1, 3 + n)[0][3:], x[n:])
    if bad == "index":
        got = pools.read(0, 5 + n)[0]
        assert np.isnan(got[5]).all() and near(got[6:], x[1:n])
    else:
        others = [p for p in range(pools.n_pages) if p not in pools.table_np[1]]
        assert torch.equal(pools.k.cpu().view(torch.uint8)[others], before.view(torch.uint8)[others])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("news,pad", [([1, 1, 0], 5), ([2, 0, 8], 1), ([40, 3, 90], 60)])
def test_rows_of_no_sequence(fmt, news, pad):
    """A padded batch: cu_new ends before total.  The rows behind it go into no page; their queries are turned like the others."""
    Hq, Hkv, d, P = 4, 2, 64, 16
    lens = [13, 0, 40]
    total = sum(news) + pad
    rng = np.random.default_rng(total)
    pools = Pools(fmt, lens, [a + b for a, b in zip(lens, news)], P, Hkv, d, 10)
    before = [None if t is None else t.cpu().clone() for t in (pools.k, pools.v, pools.ks, pools.vs)]
    q, k, v = (bf16_rows(rng, (total, H, d)) for H in (Hq, Hkv, Hkv))
    cu = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    rows = B.make_new_rows(batch=3, total=total, max_new=max(news), cu_new=torch.from_numpy(cu).cuda(), n_q_heads=Hq, n_kv_heads=Hkv,
                           head_dim=d, rot_dim=d)
    pos = torch.zeros(total, dtype=torch.int32, device="cuda")            # position 0 turns nothing: every row comes out as it is
    q_out, new_lens, ws = torch.full_like(q, 7.0).cuda(), torch.zeros(3, dtype=torch.int32, device="cuda"), workspace()
    B.fastkv_paged_append(pools.cache(), rows, pools.dev_lens, q.cuda(), k.cuda(), v.cuda(), pos, inv_freq(d).cuda(), None, q_out, new_lens, ws)
    assert B.fastkv_device_status(ws) == (0, 0)
    assert new_lens.tolist() == [a + b for a, b in zip(lens, news)]
    part = lambda x: [x.double().numpy()[cu[b]:cu[b + 1]] for b in range(3)]  # noqa: E731
    check_append(pools, before, lens, news, part(k), part(v), False)
    assert torch.equal(q_out.cpu(), q)


def test_logits_that_are_all_minus_infinity_count_as_no_entry():
    """bf16 pages: an entry whose logit is minus infinity weighs nothing, and a query that sees no other gives out 0, lse -infinity."""
    lens, d = [40, 1, 700], 64
    pools = Pools("bf16", lens, lens, 16, 1, d, 11)
    q = bf16_rows(np.random.default_rng(3), (3, 1, 4, d))
    q[..., 0] = 1.0
    for b, t in ((0, 17), (1, 0), (2, 699)):
        pools.k[int(pools.table_np[b, t // 16]), 0, t % 16, 0] = -math.inf
    cache = pools.cache()
    for b, t in ((0, 17), (2, 699)):                                      # the reference: without the entry
        pools.k64[b], pools.v64[b] = (np.delete(x, t, axis=0) for x in (pools.k64[b], pools.v64[b]))
    for longest, total in ((40, 0), (700, 0), (200000, 741)):
        query = B.make_query(n_q_heads=4, max_len=longest, total_len=total)
        ws = workspace(B.fastkv_paged_attn_workspace_bytes(cache, query))
        out, lse = torch.full((3, 1, 4, d), 7.0, device="cuda"), torch.full((3, 1, 4), 7.0, device="cuda")
        B.fastkv_paged_attn(cache, query, pools.dev_lens, q.cuda(), out, lse, ws)
        assert B.fastkv_device_status(ws) == (0, 0)
        check_attention(pools, [39, 1, 699], q.double().numpy(), out.cpu().double().numpy(), lse.cpu().double().numpy(), d ** -0.5, sequences=[0, 2])
        assert torch.all(out[1] == 0) and torch.all(lse[1] == -math.inf)
