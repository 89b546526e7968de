"""jb_cache_append against the definition in 64 bits.

Tolerance of a turned element a c - b s: c and s are good to 2 units in the last place of their sizes (fp32 angle rounded
once, 2^-24 of at most half a turn, pi 2^-24 absolute; sincospi 2^-23 absolute), so their errors are below (pi + 2) 2^-24; the two
products and the sum round three times: together (|a| + |b|) 8 2^-24, and half a step of the result for bf16.
Everything else is copied: exact.
"""
import numpy as np
import pytest
import torch

import paper_2306_10015_gb300 as jb
from test_gpu_attend import DT, i32, make

pytestmark = pytest.mark.gpu


def turned(x, turns, rotation):
    """(x turned, tolerance), x [n, heads, d]."""
    dims = rotation.dims
    with np.errstate(over="ignore"):
        part = turns.cpu().numpy().astype(np.int64).view(np.uint64)[:, None] * rotation.steps.cpu().numpy().view(np.uint64)[None]
    angle = torch.from_numpy(part.astype(np.float64) * (2 * np.pi / 2.0**64)).cuda()[:, None]
    first, second = (slice(0, dims, 2), slice(1, dims, 2)) if rotation.interleaved else (slice(0, dims // 2), slice(dims // 2, dims))
    y = x.double()
    out, tol = y.clone(), torch.zeros_like(y)
    a, b, c, s = y[..., first], y[..., second], torch.cos(angle), torch.sin(angle)
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    size = (a.abs() + b.abs()) * 8 * 2.0**-24
    tol[..., first], tol[..., second] = size, size
    if x.dtype == torch.bfloat16:
        tol[..., :dims] += 2.0**-8 * out[..., :dims].abs()
    return out, tol


def check(dtype, n, heads, group, d, rotation, page=16, layout="hnd", turns=None, q=True, in_place=False, std=1.0):
    lens = [n // 3 + 5, n - n // 3 + 2]
    cache = make(dtype, lens, heads, d, page, layout, fill=9.0)
    rows, pos = i32([0] * (n // 3) + [1] * (n - n // 3)), i32(list(range(5, n // 3 + 5)) + list(range(2, n - n // 3 + 2)))
    g = torch.Generator(device="cuda").manual_seed(n)
    qkv = (torch.randn(n, (group + 2) * heads * d, generator=g, device="cuda") * std).to(DT[dtype])
    queries, k, v = (x.view(n, -1, d) for x in qkv.split([group * heads * d, heads * d, heads * d], 1))
    before, kept = [cache.keys[0].clone(), cache.values[0].clone()], qkv.clone()
    got = jb.jb_cache_append(cache, 0, queries if q else None, k, v, rows, pos, rotation, turns=turns, q_out=queries if in_place else None)
    angles = pos if turns is None else turns
    want_k, tol_k = turned(kept[:, group * heads * d:-heads * d].view(n, heads, d), angles, rotation)
    if q:
        want_q, tol_q = turned(kept[:, :group * heads * d].view(n, -1, d), angles, rotation)
        assert ((got.double() - want_q).abs() <= tol_q).all()
        assert got.data_ptr() == queries.data_ptr() or not in_place
    else:
        assert got is None
    assert torch.equal(qkv[:, group * heads * d:], kept[:, group * heads * d:]) and (in_place or torch.equal(qkv, kept))
    ids = cache.pages.table[rows.long(), pos.long() // page].long()
    at = cache.keys[0][ids, :, pos.long() % page].double()
    assert ((at - want_k).abs() <= tol_k).all()
    before[1][ids, :, pos.long() % page] = v
    assert torch.equal(before[1], cache.values[0])
    before[0][ids, :, pos.long() % page] = cache.keys[0][ids, :, pos.long() % page]
    assert torch.equal(before[0], cache.keys[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,dims", [(8, 2), (8, 8), (16, 16), (64, 64), (64, 32), (80, 80), (80, 40), (96, 30), (120, 118), (128, 128), (128, 64),
                                    (136, 6), (256, 256), (256, 250)])
def test_heads_and_pairs(dtype, interleaved, d, dims):
    rotation = jb.Rotation.powers(dims, interleaved=interleaved)
    check(dtype, 23, 3, 2, d, rotation)
    check(dtype, 23, 3, 2, d, rotation, in_place=True)
    check(dtype, 7, 1, 1, d, rotation, page=48, layout="nhd", q=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 3, 500, 2049])
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_numbers_of_tokens(dtype, n, layout):
    check(dtype, n, 5, 3, 64, jb.Rotation.powers(64), layout=layout)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_and_negative_positions(dtype):
    far = [0, 1, 2, 1000, 131071, 1 << 24, (1 << 24) + 1, (1 << 30) + 7, 2**31 - 1, -1, -(2**31), -131072]
    for rotation in (jb.Rotation.powers(128), jb.Rotation.powers(64, 1e6, True), jb.Rotation.of([1.0, 3.0, 1e-12, 0.0, -0.5, 2 * np.pi, np.pi, 100.0])):
        check(dtype, 12, 2, 1, 128, rotation, turns=i32(far), std=3.0)


def test_turns_are_exact_at_any_position():
    """Positions 2^30 apart differ by whole turns where steps are multiples of 2^34."""
    steps = torch.tensor([1 << 44, 1 << 50, -(1 << 63), 1 << 34], dtype=torch.int64, device="cuda")
    cache = make("f32", [64], 1, 8, 16)
    x = torch.randn(3, 1, 8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    x[:] = x[:1].clone()
    q = jb.jb_cache_append(cache, 0, x.clone(), x, x, i32([0] * 3), i32(range(3)), jb.Rotation(steps), turns=i32([5, 5 + (1 << 30), 5 - (1 << 30)]))
    assert torch.equal(q[0], q[1]) and torch.equal(q[0], q[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_without_a_place(dtype):
    cache = make(dtype, [40, 20], 2, 64, 16, fill=1.0)
    cache.pages.table[1, 0] = -1
    cap = cache.pages.struct.row_pages * 16
    rows, pos = i32([0, -1, 2, 0, 0, 1, 0, 1 << 30]), i32([-1, 5, 5, cap, 2**31 - 1, 3, 6, 0])
    before = [cache.keys[0].clone(), cache.values[0].clone()]
    k = torch.randn(8, 2, 64, device="cuda").to(DT[dtype])
    rotation = jb.Rotation.powers(64)
    q = jb.jb_cache_append(cache, 0, k, k, k, rows, pos, rotation, turns=i32(range(8)))
    want, tol = turned(k, i32(range(8)), rotation)
    assert ((q.double() - want).abs() <= tol).all()
    page = int(cache.pages.table[0, 0])
    assert torch.equal(cache.values[0][page, :, 6], k[6]) and torch.equal(cache.keys[0][page, :, 6], q[6])
    before[0][page, :, 6], before[1][page, :, 6] = q[6], k[6]
    assert torch.equal(cache.keys[0], before[0]) and torch.equal(cache.values[0], before[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dims", [64, 36])
def test_not_finite(dtype, dims):
    """What is not finite stays in its pair."""
    cache = make(dtype, [40], 1, 64, 16)
    rotation = jb.Rotation.powers(dims)
    k = torch.randn(4, 1, 64, device="cuda").to(DT[dtype])
    clean = jb.jb_cache_append(cache, 0, k, k, k, i32([0] * 4), i32(range(4)), rotation)
    bad = k.clone()
    bad[:, 0, 3], bad[:, 0, dims // 2 + 7] = float("inf"), float("nan")
    got = jb.jb_cache_append(cache, 0, bad, bad, bad, i32([0] * 4), i32(range(4)), rotation)
    away = [j for j in range(64) if j not in (3, dims // 2 + 3, 7, dims // 2 + 7)]
    assert torch.equal(got[:, 0, away], clean[:, 0, away])


def test_a_graph_and_another_stream():
    cache = make("bf16", [200, 200], 2, 64, 16)
    rotation, rows = jb.Rotation.powers(64), i32([0, 1])
    x = torch.randn(2, 8, 64, device="cuda").bfloat16()
    q, k, v = x.split([4, 2, 2], 1)
    pos, out = i32([0, 0]), torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    jb.jb_cache_append(cache, 0, q, k, v, rows, pos, rotation, q_out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jb.jb_cache_append(cache, 0, q, k, v, rows, pos, rotation, q_out=out)
    stream = torch.cuda.Stream()
    for p in (3, 77, 150):
        pos.fill_(p)
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            again = jb.jb_cache_append(cache, 0, q, k, v, rows, pos + 1, rotation, turns=pos)
        stream.synchronize()
        at = lambda t: cache.keys[0][cache.pages.table[0, t // 16].long(), :, t % 16]  # noqa: E731
        assert torch.equal(out, again) and torch.equal(at(p), at(p + 1))


def test_as_many_tokens_as_a_list_can_have():
    """2^31 - 1 of them, of which the last one alone has a place; keys and values are one token's, again and again."""
    n = (1 << 31) - 1
    cache = make("bf16", [5], 2, 64, 16, fill=9.0)
    where = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    where[-1] = 0
    k, v = (torch.randn(1, 2, 64, device="cuda").bfloat16() for _ in range(2))
    before = [x.clone() for x in (cache.keys[0], cache.values[0])]
    none = jb.Rotation(torch.zeros(32, dtype=torch.int64, device="cuda"))
    jb.jb_cache_append(cache, 0, None, k.expand(n, 2, 64), v.expand(n, 2, 64), where, where, none)
    page = int(cache.pages.table[0, 0])
    before[0][page, :, 0], before[1][page, :, 0] = k[0], v[0]
    assert torch.equal(cache.keys[0], before[0]) and torch.equal(cache.values[0], before[1])
