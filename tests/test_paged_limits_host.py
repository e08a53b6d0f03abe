"""The paged attention's host side at its limits, without a GPU: lengths and bounds up to 2^31 - 1, and how large a workspace gets."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2502_01068_b200 import binding as B
from paper_2502_01068_b200 import build
from tests.test_paged_host import cache


@pytest.fixture(scope="module")
def chunk_lib(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("paged_chunks"))
    src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
    with open(src, "w") as f:
        f.write('#include "paged_index.h"\n'
                'extern "C" int t_chunk_count(int len, int log2) { return fastkv::chunk_count(len, log2); }\n'
                'extern "C" int t_chunks_all_see(int len, int q_len, int log2) { return fastkv::chunks_all_see(len, q_len, log2); }\n')
    subprocess.check_call(["g++", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-shared", "-fPIC", "-I", build.CSRC, src, "-o", so])
    return ctypes.CDLL(so)


@pytest.mark.parametrize("log2", [4, 5])
def test_chunks_of_every_length(chunk_lib, log2):
    c = 1 << log2
    top = 2 ** 31 - 1
    for n in list(range(0, 200)) + [top - k for k in range(200)]:
        assert chunk_lib.t_chunk_count(n, log2) == -(-n // c), n
        for q_len in (1, 2, 9, 130, top):
            assert chunk_lib.t_chunks_all_see(n, q_len, log2) == max(n - (q_len - 1), 0) // c, (n, q_len)


@pytest.fixture(scope="module")
def built():
    build.build_library()


@pytest.mark.parametrize("fmt", [B.CACHE_BF16, B.CACHE_E4M3])
def test_any_bound_of_the_length_is_laid_out_like_a_long_one(built, fmt):
    """max_len may be any upper bound: one that is as large as an int goes splits a sequence like one of a million."""
    scales = dict(k_scales=None, v_scales=None) if fmt == B.CACHE_BF16 else {}
    c = cache(batch=1, n_kv_heads=8, format=fmt, **scales)
    size = lambda n, q: B.fastkv_paged_attn_workspace_bytes(c, B.make_query(n_q_heads=32, max_len=n, q_len=q))  # noqa: E731
    for q in (1, 5):
        assert size(10 ** 6, q) > 256
        for n in (2 ** 31 - 1, 2 ** 31 - 15, 2 ** 31 - 16, 2 ** 31 - 32):
            assert size(n, q) == size(10 ** 6, q), n


def test_no_workspace_is_larger_than_five_megabytes(built):
    """What the header promises to who allocates once for every length to come."""
    rng = random.Random(3)
    largest = 0
    for _ in range(4000):
        fmt = rng.choice([B.CACHE_BF16, B.CACHE_E4M3])
        scales = dict(k_scales=None, v_scales=None) if fmt == B.CACHE_BF16 else {}
        hkv, batch = rng.choice([1, 2, 3, 8, 40]), int(2 ** rng.uniform(0, 10))
        c = cache(batch=batch, n_kv_heads=hkv, head_dim=rng.choice([64, 128]), format=fmt, n_pages=1000, **scales)
        longest = int(2 ** rng.uniform(0, 30.9))
        q = B.make_query(n_q_heads=hkv * rng.choice([1, 3, 4, 8, 16]), q_len=rng.choice([1, 1, 2, 5, 40]), max_len=longest,
                         total_len=rng.choice([0, max(1, batch * longest // rng.choice([1, 4, 30, 1000]))]))
        largest = max(largest, B.fastkv_paged_attn_workspace_bytes(c, q))
    assert 4 * 2 ** 20 < largest <= 5 * 2 ** 20
