"""The bounded-wait failure path of the key-mass window kernel: a test copy of it with a wait limit of
200 ns, checked on every poll, gives up while copies and products are in flight, reports
SONIC_ERR_DEVICE_TIMEOUT and winds down; the normal library then runs the same call."""
import os
import shutil
import tempfile

import pytest
import torch

from paper_2601_21927_gb300 import _build, sonic
from tests.test_gpu_key_mass import check_mass, make
from tests.test_gpu_kv4 import dev, i32, status

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def short_wait_lib():
    d = tempfile.mkdtemp(prefix="sonic_short_wait_")
    try:
        path = _build.compile_library(os.path.join(d, "libsonic_short_wait.so"),
                                      ["api.cu", "key_mass.cu", "kv4.cu", "compact.cu"],
                                      defines=["SONIC_WAIT_LIMIT_NS=200ull", "SONIC_WAIT_CHECK_MASK=0u"])
        yield sonic.open_library(path)
    finally:
        shutil.rmtree(d, ignore_errors=True)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("hq,hkv,d,queries,per_head", [(28, 4, 128, 32, True), (16, 2, 64, 70, False)])
def test_window_wait_timeout_then_normal_call(short_wait_lib, bits, hq, hkv, d, queries, per_head):
    lens = [2500, 600, 90]
    K, K64, q, lse, start, rows, nq, q_start = make(hq, hkv, d, lens, queries, bits, 1, 7)
    before = torch.rand((1, hkv if per_head else 1, rows), device=dev())
    kw = dict(kv_start=i32(start), max_len=2500, q_start=i32(q_start), q_len=i32(nq), max_q_len=queries, keep=0.0)
    st, mass, saved = status(), before.clone(), sonic.load()
    sonic._lib = short_wait_lib
    try:
        sonic.sonic_key_mass(q, K, lse, i32(lens), mass, status=st, **kw)
    finally:
        sonic._lib = saved
    torch.cuda.synchronize()  # the context is still usable
    assert st.item() == 5  # SONIC_ERR_DEVICE_TIMEOUT
    # a call with that status word leaves its blocks at once
    mass = before.clone()
    sonic.sonic_key_mass(q, K, lse, i32(lens), mass, status=st, **kw)
    torch.cuda.synchronize()
    assert torch.equal(mass, before)
    st.zero_()
    sonic.sonic_key_mass(q, K, lse, i32(lens), mass, status=st, **kw)
    assert st.item() == 0
    check_mass(mass, before, None, 0.0, K64, q, lse, start, lens, nq, q_start)


@pytest.fixture(scope="module")
def one_warp_gives_up_lib():
    """The library with one of the sixteen warps that add up the weights giving up at its first wait, where the
    others go on."""
    d = tempfile.mkdtemp(prefix="sonic_one_warp_")
    try:
        path = _build.compile_library(os.path.join(d, "libsonic_one_warp.so"),
                                      ["api.cu", "key_mass.cu", "kv4.cu", "compact.cu"],
                                      defines=["SONIC_WAIT_GIVES_UP=(threadIdx.x/32==5)", "SONIC_WAIT_CHECK_MASK=0u"])
        yield sonic.open_library(path)
    finally:
        shutil.rmtree(d, ignore_errors=True)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("hq,hkv,d,queries,per_head", [(28, 4, 128, 32, True), (16, 2, 64, 70, False),
                                                       (64, 1, 128, 90, True)])
def test_a_call_that_gives_up_leaves_entries_whole(one_warp_gives_up_lib, bits, hq, hkv, d, queries, per_head):
    """Where a wait ran out a block writes all of its entries or none: each is as it was, or right, added up in
    place or not.  (Without a status word every block waits for itself.)"""
    lens = [2500, 600, 90, 1300] + [100 + b for b in range(60)]
    K, K64, q, lse, start, rows, nq, q_start = make(hq, hkv, d, lens, queries, bits, 1, 7)
    before = torch.rand((1, hkv if per_head else 1, rows), device=dev())
    kw = dict(kv_start=i32(start), max_len=2500, q_start=i32(q_start), q_len=i32(nq), max_q_len=queries)
    for keep in (0.0, 1.0):
        whole = before.clone()
        sonic.sonic_key_mass(q, K, lse, i32(lens), whole, prev=whole if keep else None, keep=keep, **kw)
        check_mass(whole, before, before, keep, K64, q, lse, start, lens, nq, q_start)
        for _ in range(4):
            mass, saved = before.clone(), sonic.load()
            sonic._lib = one_warp_gives_up_lib
            try:
                sonic.sonic_key_mass(q, K, lse, i32(lens), mass, prev=mass if keep else None, keep=keep, **kw)
            finally:
                sonic._lib = saved
            torch.cuda.synchronize()
            assert bool(((mass == before) | (mass == whole)).all())  # (sums in a fixed order: the same bits)
