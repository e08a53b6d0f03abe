"""The paged cache without a GPU: the kernels' index arithmetic (compiled for the host from the header that they include)
against a plain restatement, and the refusals of the C ABI."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest

from paper_2502_01068_b200 import binding as B
from paper_2502_01068_b200 import build
from tests.paged_reference import need_scale, rn_e4m3

CSRC = build.CSRC


@pytest.fixture(scope="module")
def index_lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged_index")
    src = os.path.join(str(d), "shim.cpp")
    with open(src, "w") as f:
        f.write('''#include "paged_index.h"
extern "C" {
int t_scale_exponent(uint32_t bits) { return fastkv::scale_exponent(bits); }
uint32_t t_pow2_bits(int e) { return fastkv::pow2_bits(e); }
int t_scale_log2(uint32_t b) { return fastkv::scale_log2(b); }
int t_usable_len(int len, int max_pages, int log2) { return fastkv::usable_len(len, max_pages, log2); }
int t_new_rows(const int* cu, int uniform, int total, int max_new, int b, int len, int max_pages, int log2, int* out) {
  fastkv::RowRange r;
  const bool ok = fastkv::new_rows_of(cu, uniform, total, max_new, b, len, max_pages, log2, &r);
  out[0] = r.first; out[1] = r.count;
  return ok;
}
long long t_pool_block(int page, int n_pages, int heads, int head) { return fastkv::pool_block(page, n_pages, heads, head); }
}
''')
    so = os.path.join(str(d), "shim.so")
    subprocess.check_call(["g++", "-O1", "-shared", "-fPIC", "-I", CSRC, src, "-o", so])
    lib = ctypes.CDLL(so)
    lib.t_pool_block.restype = ctypes.c_longlong
    lib.t_pow2_bits.restype = ctypes.c_uint32
    lib.t_scale_exponent.argtypes = [ctypes.c_uint32]
    return lib


def bits(x):
    return int(np.float32(x).view(np.uint32))


def test_scale_exponent_is_the_smallest_that_holds_the_value(index_lib):
    rng = np.random.default_rng(5)
    values = [0.0, 448.0, np.nextafter(np.float32(448), np.float32(1e9)), 1.0, 1.75, np.nextafter(np.float32(1.75), np.float32(2)),
              3.5, 3.4e38, 1e-30, 2.0 ** -64 * 448, 2.0 ** -65 * 448, 2.0 ** -63 * 448 * 1.0001, 1e-45, np.finfo(np.float32).max]
    values += list(np.exp(rng.uniform(-60, 88, 400)).astype(np.float32))
    for v in values:
        e = index_lib.t_scale_exponent(bits(v))
        assert math.ldexp(1.0, e) == need_scale(float(np.float32(v))), v
        assert index_lib.t_scale_log2(index_lib.t_pow2_bits(e)) == e
    assert index_lib.t_scale_exponent(bits(np.inf)) == 120
    for e in (-126, -64, 0, 120, 127):
        assert np.uint32(index_lib.t_pow2_bits(e)).view(np.float32) == np.float32(2.0) ** e


def test_the_reference_quantiser_agrees_with_torch():
    import torch
    x = np.concatenate([np.linspace(-500, 500, 20001), np.ldexp(1.0, np.arange(-14, 9)), np.ldexp(3.0, np.arange(-14, 6)),
                        np.linspace(-0.05, 0.05, 4001)]).astype(np.float32)
    ref = torch.from_numpy(np.clip(x, -448, 448)).to(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(rn_e4m3(x.astype(np.float64)), ref)


def test_new_rows_are_cut_to_what_exists(index_lib):
    """Every combination of small sizes: the rows a sequence may write lie inside the call's rows and inside its block
    table's room, and nothing is cut (and reported) that fits."""
    out = (ctypes.c_int * 2)()
    for log2 in (4, 5):
        for max_pages in (1, 2):
            room = max_pages << log2
            for length in (-3, 0, 1, room - 2, room - 1, room, room + 5, 2 ** 31 - 1):
                for cu in ([0, 3], [2, 2], [0, 9], [-1, 4], [5, 2], [0, 100], [7, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1]):
                    arr = (ctypes.c_int * 2)(*cu)
                    total, max_new = 9, 6
                    ok = index_lib.t_new_rows(arr, 0, total, max_new, 0, length, max_pages, log2, out)
                    first, count = out[0], out[1]
                    assert 0 <= count <= max_new and first >= 0 and (count == 0 or first + count <= total)
                    if count:
                        assert length >= 0 and length + count <= room
                    fits = (length >= 0 and cu[0] >= 0 and 0 <= cu[1] - cu[0] <= max_new and cu[1] <= total
                            and length + cu[1] - cu[0] <= room)
                    assert bool(ok) == fits, (length, cu, room)
                    if fits:
                        assert (first, count) == (cu[0], cu[1] - cu[0])
    assert index_lib.t_new_rows(None, 4, 12, 4, 2, 10, 4, 4, out) and (out[0], out[1]) == (8, 4)


def test_usable_length_and_pool_blocks(index_lib):
    assert [index_lib.t_usable_len(n, 3, 4) for n in (-1, 0, 47, 48, 49, 2 ** 31 - 1)] == [0, 0, 47, 48, 48, 48]
    assert index_lib.t_usable_len(2 ** 31 - 1, 2 ** 27 - 1, 4) == (2 ** 27 - 1) * 16
    for page in (-1, 7, 2 ** 31 - 1, -2 ** 31):
        assert index_lib.t_pool_block(page, 7, 8, 3) == -1
    assert index_lib.t_pool_block(6, 7, 8, 3) == 51
    # a row of the block, in 64 bits: block * 128 rows * 128 elements passes 2^31 long before the pools do
    assert index_lib.t_pool_block(2 ** 28 - 1, 2 ** 28, 7, 6) == (2 ** 28 - 1) * 7 + 6


# ---- refusals ------------------------------------------------------------------------------------------------------------
class Fake:
    """Stands in for a device tensor: every call below must fail before any pointer is used."""
    def __init__(self, ptr=0x10000, n=1 << 20):
        self.ptr, self.n = ptr, n

    def data_ptr(self):
        return self.ptr

    @property
    def nbytes(self):
        return self.n


class NullStream:
    cuda_stream = 0


@pytest.fixture()
def no_device(monkeypatch):
    build.build_library()
    monkeypatch.setattr(B, "_p", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(B, "_here", lambda cache: 0)


def cache(**kw):
    c = B.PagedCache()
    vals = dict(batch=2, max_pages=4, n_pages=9, page_size=64, n_kv_heads=2, head_dim=128, format=B.CACHE_E4M3, reserved=0,
                k_pages=0x10000, v_pages=0x20000, k_scales=0x30000, v_scales=0x40000, block_table=0x50000)
    vals.update(kw)
    for k, v in vals.items():
        setattr(c, k, v)
    return c


def rows(**kw):
    args = dict(batch=2, total=4, n_kv_heads=2, head_dim=128, n_q_heads=8, rot_dim=128)
    args.update(kw)
    return B.make_new_rows(**args)


def status_of(fn, *a):
    with pytest.raises(B.FastKVError) as e:
        fn(*a)
    return e.value.status


def append(c, r, lens=Fake(), q=Fake(), k=Fake(), v=Fake(), pos=Fake(), inv=Fake(), idx=None, q_out=Fake(0x80000), new_lens=None,
           ws=Fake()):
    B.fastkv_paged_append(c, r, lens, q, k, v, pos, inv, idx, q_out, new_lens, ws, NullStream)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), B.ERR_INVALID_ARG), (dict(max_pages=0), B.ERR_INVALID_ARG), (dict(n_pages=0), B.ERR_INVALID_ARG),
    (dict(n_kv_heads=0), B.ERR_INVALID_ARG), (dict(format=2), B.ERR_INVALID_ARG), (dict(reserved=1), B.ERR_INVALID_ARG),
    (dict(head_dim=96), B.ERR_UNSUPPORTED), (dict(page_size=8), B.ERR_UNSUPPORTED), (dict(page_size=48), B.ERR_UNSUPPORTED),
    (dict(n_pages=2 ** 30), B.ERR_UNSUPPORTED), (dict(max_pages=2 ** 26), B.ERR_UNSUPPORTED), (dict(k_pages=None), B.ERR_INVALID_ARG),
    (dict(block_table=None), B.ERR_INVALID_ARG), (dict(v_pages=0x20008), B.ERR_UNSUPPORTED), (dict(k_scales=None), B.ERR_INVALID_ARG),
    (dict(format=B.CACHE_BF16), B.ERR_INVALID_ARG), (dict(format=B.CACHE_BF16, k_scales=None), B.ERR_INVALID_ARG)])
def test_bad_caches_are_refused(no_device, kw, status):
    assert status_of(append, cache(**kw), rows()) == status
    q = B.make_query(n_q_heads=8, max_len=100)
    assert status_of(B.fastkv_paged_attn_workspace_bytes, cache(**kw), q) == status
    assert status_of(B.fastkv_paged_attn, cache(**kw), q, Fake(), Fake(), Fake(), None, Fake(), NullStream) == status


@pytest.mark.parametrize("kw,call,status", [
    (dict(total=0, max_new=1), {}, B.ERR_INVALID_ARG), (dict(max_new=0), {}, B.ERR_INVALID_ARG),
    (dict(max_new=5), {}, B.ERR_INVALID_ARG), (dict(max_new=3), {}, B.ERR_INVALID_ARG),          # 2 * 3 != 4 without cu_new
    (dict(n_q_heads=7), {}, B.ERR_INVALID_ARG), (dict(n_q_heads=0), {}, B.ERR_INVALID_ARG),      # q without heads
    ({}, dict(q=None), B.ERR_INVALID_ARG), ({}, dict(q_out=None), B.ERR_INVALID_ARG),
    (dict(rot_dim=144), {}, B.ERR_INVALID_ARG), (dict(rot_dim=24), {}, B.ERR_UNSUPPORTED), (dict(rot_pairs=2), {}, B.ERR_INVALID_ARG),
    (dict(rot_dim=-16), {}, B.ERR_INVALID_ARG), (dict(rot_dim=0), {}, B.ERR_INVALID_ARG), ({}, dict(pos=None), B.ERR_INVALID_ARG),
    ({}, dict(inv=None), B.ERR_INVALID_ARG), ({}, dict(inv=Fake(0x10004)), B.ERR_UNSUPPORTED),
    ({}, dict(idx=Fake()), B.ERR_INVALID_ARG), (dict(total_src=8), {}, B.ERR_INVALID_ARG), (dict(total_src=-1), {}, B.ERR_INVALID_ARG),
    (dict(total_src=8), dict(idx=Fake()), B.ERR_INVALID_ARG),                                    # kept rows with rotation
    (dict(total_src=8, rot_dim=0, n_q_heads=0), dict(idx=Fake(), q=None, q_out=None, pos=None, inv=None), B.ERR_INVALID_ARG),  # no cu_src
    (dict(cu_src=Fake()), {}, B.ERR_INVALID_ARG), ({}, dict(lens=None), B.ERR_INVALID_ARG), ({}, dict(k=None), B.ERR_INVALID_ARG),
    ({}, dict(new_lens=Fake(0x10000)), B.ERR_INVALID_ARG), ({}, dict(new_lens=Fake(0x10004)), B.ERR_INVALID_ARG),
    (dict(k_stride_tok=260), {}, B.ERR_UNSUPPORTED), (dict(v_stride_head=64), {}, B.ERR_INVALID_ARG), ({}, dict(v=Fake(0x10008)), B.ERR_UNSUPPORTED),
    ({}, dict(q_out=Fake(0x80002)), B.ERR_UNSUPPORTED), (dict(q_stride_tok=2048), dict(q_out=Fake()), B.ERR_INVALID_ARG),
    ({}, dict(ws=Fake(0x10010)), B.ERR_WORKSPACE), ({}, dict(ws=Fake(0x10000, 255)), B.ERR_WORKSPACE)])
def test_bad_appends_are_refused(no_device, kw, call, status):
    assert status_of(lambda: append(cache(), rows(**kw), **call)) == status


@pytest.mark.parametrize("kw,call,status", [
    (dict(n_q_heads=0), {}, B.ERR_INVALID_ARG), (dict(n_q_heads=5), {}, B.ERR_INVALID_ARG), (dict(q_len=0), {}, B.ERR_INVALID_ARG),
    (dict(max_len=0), {}, B.ERR_INVALID_ARG), (dict(total_len=-1), {}, B.ERR_INVALID_ARG), (dict(q_len=2 ** 30), {}, B.ERR_UNSUPPORTED),
    (dict(softmax_scale=float("nan")), {}, B.ERR_INVALID_ARG), (dict(softmax_scale=-1.0), {}, B.ERR_INVALID_ARG),
    ({}, dict(lens=None), B.ERR_INVALID_ARG), ({}, dict(q=None), B.ERR_INVALID_ARG), ({}, dict(out=None), B.ERR_INVALID_ARG),
    ({}, dict(q=Fake(0x10008)), B.ERR_UNSUPPORTED), ({}, dict(out=Fake(0x10004)), B.ERR_UNSUPPORTED),
    ({}, dict(ws=Fake(0x10080)), B.ERR_WORKSPACE), ({}, dict(ws=Fake(0x10000, 255)), B.ERR_WORKSPACE)])
def test_bad_queries_are_refused(no_device, kw, call, status):
    args = dict(n_q_heads=8, max_len=200)
    args.update(kw)
    a = dict(lens=Fake(), q=Fake(), out=Fake(), ws=Fake(0x10000, 1 << 24))
    a.update(call)
    q = B.make_query(**args)
    assert status_of(B.fastkv_paged_attn, cache(), q, a["lens"], a["q"], a["out"], None, a["ws"], NullStream) == status


def test_the_binding_checks_the_caches_tensors():
    import torch
    k = torch.zeros(3, 2, 16, 64, dtype=torch.float8_e4m3fn)
    s = torch.zeros(3, 2)
    t = torch.zeros(1, 3, dtype=torch.int32)
    c = B.make_paged_cache(k, k, t, s, s)
    assert (c.batch, c.max_pages, c.n_pages, c.n_kv_heads, c.page_size, c.head_dim, c.format) == (1, 3, 3, 2, 16, 64, B.CACHE_E4M3)
    b = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    assert B.make_paged_cache(b, b, t).format == B.CACHE_BF16
    for bad in (lambda: B.make_paged_cache(k, k, t), lambda: B.make_paged_cache(b, b, t, s, s), lambda: B.make_paged_cache(b, k, t),
                lambda: B.make_paged_cache(b, b, t.long()), lambda: B.make_paged_cache(k, k, t, s, s[:2]),
                lambda: B.make_paged_cache(b[:, :, ::2], b[:, :, ::2], t), lambda: B.make_paged_cache(k, k, t, s.double(), s)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        B.make_paged_cache(b.float(), b.float(), t)
