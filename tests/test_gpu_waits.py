"""Waits that run out, and what a kernel before them left in shared memory or values that are not finite do to the time of others."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2306_10015_gb300 as jb
from paper_2306_10015_gb300 import build
from test_gpu_tree import case, chain, check, draft

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def helper():
    src, out_dir = os.path.join(HERE, "helpers", "waits.cu"), os.path.join(HERE, "_build")
    os.makedirs(out_dir, exist_ok=True)
    so = os.path.join(out_dir, "libwaits.so")
    subprocess.run([build.nvcc(), *build.ARCH, "-O2", "-std=c++17", "-I", build.CSRC, "-shared", "-Xcompiler", "-fPIC", src, "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.unserved_wait.argtypes = [ctypes.c_void_p]
    lib.drained_products.argtypes = [ctypes.c_void_p]
    lib.fill_shared.argtypes = [ctypes.c_uint32]
    return lib


def test_heads_of_192_do_not_depend_on_what_shared_memory_held(helper):
    """Only three of the four panels of a tile are copied for them; the fourth may hold anything."""
    trees = [chain(255)] * 8
    cache, q = case("bf16", [100] * 8, trees, 4, 1, 192, 16)
    want = check(cache, 0, q, range(8), trees)
    t, out = draft(range(8), trees), torch.empty_like(q)
    times = {}
    for _ in range(6):
        for pattern in (0, 0x7FC07FC0):
            assert helper.fill_shared(pattern) == 0
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            jb.jb_attend_tree(cache, 0, q, t, out=out)
            b.record()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            times[pattern] = min(times.get(pattern, 1e9), a.elapsed_time(b))
    assert times[0x7FC07FC0] <= 1.3 * times[0], times


def test_a_value_that_is_not_finite_slows_its_own_block_alone():
    """In the first head of the first tree or in the last of the last: the CTA with the first block has others after it."""
    n, heads = 120, 8
    trees = [chain(200)] * n
    cache, q = case("bf16", [60] * n, trees, heads, 1, 64, 16)
    t, out, times, values = draft(range(n), trees), torch.empty_like(q), {}, cache.values[0].clone()
    for _ in range(6):
        for tree, head in ((0, 0), (n - 1, heads - 1)):
            cache.values[0].copy_(values)
            cache.values[0][int(cache.pages.table[tree, 259 // 16]), head, 259 % 16] = float("nan")   # the last node
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            jb.jb_attend_tree(cache, 0, q, t, out=out)
            b.record()
            torch.cuda.synchronize()
            last = 200 * tree + 199
            assert torch.isnan(out[last]).all(1).nonzero().tolist() == [[head]] and torch.isfinite(out[:last]).all() and torch.isfinite(out[last + 1:]).all()
            times[tree] = min(times.get(tree, 1e9), a.elapsed_time(b))
    assert times[0] <= 1.5 * times[n - 1], times


def test_a_wait_that_nobody_serves_gives_up_and_later_ones_do_not_wait(helper):
    """The limit is 4e9 cycles, looked at after every 32 looks at the barrier. After it a wait is one look and no more."""
    out = torch.zeros(6, dtype=torch.int64, device="cuda")
    assert helper.unserved_wait(out.data_ptr()) == 0
    first, failed, cycles, look, later, second = out.tolist()
    assert (first, failed, second) == (0, 1, 0)
    assert 4e9 < cycles < 4e9 + 40 * look + 10_000, (cycles, look)
    assert later <= 3 * look + 2000, f"{later} cycles after the limit, {look} a look"


def test_products_are_done_when_they_are_waited_for_at_the_end(helper):
    out = torch.zeros(32, device="cuda")
    for _ in range(50):
        out.zero_()
        assert helper.drained_products(out.data_ptr()) == 0
        assert (out == 64 * 64).all()
