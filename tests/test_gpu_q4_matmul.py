"""jb_q4_matmul against the definition in 64 bits.

Tolerance with A = sum_k |x_k w_k|: a term is a product of a level and an input. In bf16 a level enters with half a step of
fp16, 2^-12, and inputs keep their 8 bits unless they are 2^-28 of the largest of their row and smaller (2^-40 of that one:
far below the sum's own allowance); in fp32 both enter with 2^-24 and their product drops less than 2^-23. The sum of K terms and the
products with scales lose at most (K / 16 + 70) 2^-23 of A in any order of blocks and lanes (16 terms a step of a tensor
core, whose sums may truncate: 2^-22 a step), and a result is rounded once: 2^-8 of it for bf16 with the tie.
"""
import numpy as np
import pytest
import torch

import paper_2306_10015_gb300 as jb
from test_gpu_attend import DT

pytestmark = pytest.mark.gpu


def weights(out, inner, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (out * inner // 2,), dtype=torch.uint8, device="cuda", generator=g)
    scale = torch.rand(out * inner // 64, device="cuda", generator=g) + 0.1
    return jb.Q4Table([(codes, scale, out * inner)])


def dense(table, index, out, inner):
    codes, scale, n = table.tensors[index]
    c = torch.stack([codes & 15, codes >> 4], -1).view(-1)[:n].long()
    w = torch.from_numpy(jb.jb_q4_levels().astype(np.float64)).cuda()[c] * scale.double().repeat_interleave(64)[:n]
    return w.view(out, inner)


def bound(x, w, bias, want):
    a = x.double().abs() @ w.abs().T + (0 if bias is None else bias.double().abs())
    rel = (x.shape[1] / 16 + 70) * 2.0**-22
    if x.dtype == torch.bfloat16:
        return a * (rel + 2.0**-12) + 2.0**-8 * want.abs() + 1e-38
    return a * (rel + 3 * 2.0**-23) + 1e-38


def check(dtype, n, out, inner, bias=True, x=None, table=None, **kw):
    g = torch.Generator(device="cuda").manual_seed(n + out)
    table = weights(out, inner) if table is None else table
    x = torch.randn(n, inner, device="cuda", generator=g).to(DT[dtype]) if x is None else x
    b = torch.randn(out, device="cuda", generator=g).to(DT[dtype]) if bias else None
    got = jb.jb_q4_matmul(table, 0, x, out, bias=b, **kw)
    w = dense(table, 0, out, inner)
    want = x.double() @ w.T + (0 if b is None else b.double())
    err, tol = (got.double() - want).abs(), bound(x, w, b, want)
    assert got.shape == (n, out) and torch.isfinite(got).all()
    assert (err <= tol).all(), f"worst error over tolerance {(err / tol).amax():.3g}"
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 7, 8, 9, 16, 17, 31, 33, 64, 65, 130])
@pytest.mark.parametrize("out,inner", [(100, 256), (33, 1088)])
def test_numbers_of_rows(dtype, n, out, inner):
    check(dtype, n, out, inner)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 6, 20])
@pytest.mark.parametrize("out", [1, 7, 15, 16, 17, 31, 64, 300, 2501])
@pytest.mark.parametrize("inner", [64, 128, 192, 448, 512, 576, 1024])
def test_shapes(dtype, n, out, inner):
    check(dtype, n, out, inner, bias=out % 2 == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 9, 40])
@pytest.mark.parametrize("out,inner", [(40, 20480), (5, 65536), (17, 8256), (20000, 128)])
def test_long_and_wide(dtype, n, out, inner):
    check(dtype, n, out, inner)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("inner", [8192, 13312, 20480, 32768, 65536])
def test_long_rows_that_are_taken_some_at_a_time(dtype, inner):
    """The last rows are fewer than those before them, whatever the number."""
    table = weights(19, inner)
    for n in range(1, 72):
        check(dtype, n, 19, inner, bias=n % 2 == 0, table=table)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 33, 48, 64, 65, 100])
@pytest.mark.parametrize("out,inner", [(4096, 1024), (1000, 4224), (65601, 64), (150, 32768), (130, 65536), (2049, 2112), (777, 704)])
def test_matrices_that_are_cut_into_tiles(dtype, n, out, inner):
    """Tiles of 128 rows: the last one ragged, columns that end inside a step of four blocks, tiles that many CTAs share and
    CTAs that have many."""
    check(dtype, n, out, inner, bias=n % 2 == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("out,inner,ns", [(4100, 4160, (4, 5, 8, 9, 12)), (10001, 6720, (1, 3, 4, 5, 7, 8, 11)),
                                          (1050, 65536, (1, 2, 3))])
def test_large_matrices_and_few_rows(dtype, out, inner, ns):
    """On both sides of the sizes at which the tiles begin to pay."""
    table = weights(out, inner)
    for n in ns:
        check(dtype, n, out, inner, bias=n % 2 == 0, table=table)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [6, 27])
def test_tiles_strides_and_odd_scales(dtype, n):
    """Rows inside wider ones and scales off a 16-byte boundary; codes off one, which take the other kernel."""
    g = torch.Generator(device="cuda").manual_seed(4)
    out, inner = 3000, 1536
    codes = torch.randint(0, 256, (out * inner // 2 + 8,), dtype=torch.uint8, device="cuda", generator=g)
    scale = torch.rand(out * inner // 64 + 3, device="cuda", generator=g)
    x = torch.randn(n, inner + 80, device="cuda", generator=g).to(DT[dtype])[:, 40:40 + inner]
    for skip, first in ((0, 3), (8, 0)):
        table = jb.Q4Table([(codes[skip:skip + out * inner // 2], scale[first:first + out * inner // 64], out * inner)])
        y = torch.full((n, out + 9), 4.0, dtype=DT[dtype], device="cuda")
        got = jb.jb_q4_matmul(table, 0, x, out, out=y[:, 4:4 + out])
        assert (y[:, :4] == 4).all() and (y[:, 4 + out:] == 4).all()
        w = dense(table, 0, out, inner)
        want = x.double() @ w.T
        assert ((got.double() - want).abs() <= bound(x, w, None, want)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("times", [1, 3])
def test_tiles_inputs_that_are_not_finite_or_of_all_sizes(dtype, times):
    table = weights(2100, 2048)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(9, 2048, device="cuda", generator=g)
    x *= torch.tensor([1e-38, 1e-30, 1e-10, 1e-3, 1.0, 1e10, 1e30, 1e35, 0.0], device="cuda")[:, None]
    x[:, ::97] *= 100.0
    x = x.to(DT[dtype]).repeat(times, 1)
    clean = check(dtype, 9 * times, 2100, 2048, bias=False, x=x, table=table)
    x[1, 500], x[3, 70], x[4, 2047] = float("inf"), float("nan"), -float("inf")
    got = jb.jb_q4_matmul(table, 0, x, 2100)
    away = [i for i in range(9 * times) if i not in (1, 3, 4)]
    assert torch.equal(got[away], clean[away])
    want = x.double() @ dense(table, 0, 2100, 2048).T
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_level(dtype):
    """A weight at a time: y is x level scale, each code in each place of a block."""
    table = weights(64, 64)
    codes, scale, _ = table.tensors[0]
    x = torch.zeros(1, 64, device="cuda", dtype=DT[dtype])
    w = dense(table, 0, 64, 64)
    for k in range(64):
        x.zero_()
        x[0, k] = 1.5
        got = jb.jb_q4_matmul(table, 0, x, 64)[0].double()
        want = 1.5 * w[:, k]
        assert ((got - want).abs() <= want.abs() * (2.0**-8 + 2.0**-11 if dtype == "bf16" else 2.0**-21)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_inputs_of_all_sizes(dtype):
    """Inputs from 1e-38 to 1e37, rows of their own sizes, outliers beside small values, zeros."""
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(9, 1024, device="cuda", generator=g)
    x *= torch.tensor([1e-38, 1e-30, 1e-10, 1e-3, 1.0, 1e10, 1e30, 1e35, 0.0], device="cuda")[:, None]
    x[:, ::97] *= 100.0
    x[4, ::5] *= 1e-6
    check(dtype, 9, 50, 1024, bias=False, x=x.to(DT[dtype]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_not_finite_inputs(dtype):
    """They make their own rows' results infinite or NaN, as the sums have it, and no others'."""
    table = weights(40, 576)
    x = torch.randn(5, 576, device="cuda").to(DT[dtype])
    clean = jb.jb_q4_matmul(table, 0, x, 40)
    x[1, 500], x[3, 70] = float("inf"), float("nan")
    got = jb.jb_q4_matmul(table, 0, x, 40)
    assert torch.equal(got[[0, 2, 4]], clean[[0, 2, 4]])
    want = x.double() @ dense(table, 0, 40, 576).T
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    assert (torch.sign(got[1]) == torch.sign(want[1]).to(got.dtype))[~torch.isnan(got[1])].all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_outputs_and_later_tensors(dtype):
    """Rows inside wider ones; a matrix that starts 8 bytes off a 16-byte boundary; the second of a table."""
    g = torch.Generator(device="cuda").manual_seed(4)
    out, inner = 70, 320
    codes = torch.randint(0, 256, (out * inner // 2 + 8,), dtype=torch.uint8, device="cuda", generator=g)
    scale = torch.rand(out * inner // 64 + 3, device="cuda", generator=g)
    a = weights(10, 64)
    table = jb.Q4Table([a.tensors[0], (codes[8:], scale[3:], out * inner)])
    x = torch.randn(6, 400, device="cuda", generator=g).to(DT[dtype])[:, 40:360]
    y = torch.full((6, out + 9), 4.0, dtype=DT[dtype], device="cuda")
    got = jb.jb_q4_matmul(table, 1, x, out, out=y[:, 4:4 + out])
    assert (y[:, :4] == 4).all() and (y[:, 4 + out:] == 4).all() and got.data_ptr() == y[:, 4:].data_ptr()
    w = dense(table, 1, out, inner)
    want = x.double() @ w.T
    assert ((got.double() - want).abs() <= bound(x, w, None, want)).all()
    assert torch.equal(jb.jb_q4_matmul(table, -1, x, out), got)
    assert jb.jb_q4_matmul(table, 1, x[:0], out).shape == (0, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [12, 40])
def test_repeatable_streams_and_graphs(dtype, n):
    table = weights(3000, 2048)
    x = torch.randn(n, 2048, device="cuda").to(DT[dtype])
    want = check(dtype, n, 3000, 2048, bias=False, x=x, table=table)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    a, b = jb.jb_q4_matmul(table, 0, x, 3000), jb.jb_q4_matmul(table, 0, x, 3000, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jb.jb_q4_matmul(table, 0, x, 3000, out=out)
    for scale in (1.0, 3.0):
        x.mul_(scale)
        graph.replay()
        assert torch.equal(out, jb.jb_q4_matmul(table, 0, x, 3000))


def test_between_two_perturbations():
    """The weights are read when the product runs: perturbed codes and scales enter, and theta + eps z - 2 eps z + eps z."""
    table = weights(96, 640)
    x = torch.randn(3, 640, device="cuda")
    for eps in (1e-2, -2e-2, 1e-2):
        jb.jb_perturb_q4(table, (5, 1, 0), eps)
        got = jb.jb_q4_matmul(table, 0, x, 96)
        w = dense(table, 0, 96, 640)
        want = x.double() @ w.T
        assert ((got.double() - want).abs() <= bound(x, w, None, want)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_calls_side_by_side(dtype):
    """Two streams and two captured graphs of one table, which keeps or makes a workspace for each of them."""
    table = weights(8192, 4096)
    x = [torch.randn(n, 4096, device="cuda").to(DT[dtype]) for n in (33, 20)]
    want = [jb.jb_q4_matmul(table, 0, v, 8192) for v in x]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got, graphs, out = [[], []], [], []
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(jb.jb_q4_matmul(table, 0, x[i], 8192))
    torch.cuda.synchronize()
    for i, s in enumerate(streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out.append([jb.jb_q4_matmul(table, 0, x[i], 8192) for _ in range(10)])
        graphs.append(graph)
    torch.cuda.synchronize()
    for s, graph in zip(streams, graphs):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i] + out[i])


@pytest.mark.parametrize("out,inner,n", [(33000, 65536, 2), (140000, 16384, 1)])
def test_large_matrices(out, inner, n):
    """More than 2^31 weights: offsets past 32 bits."""
    codes = torch.zeros(out * inner // 2, dtype=torch.uint8, device="cuda")
    scale = torch.zeros(out * inner // 64, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    tail = 40 * inner
    codes[-tail // 2:] = torch.randint(0, 256, (tail // 2,), dtype=torch.uint8, device="cuda", generator=g)
    scale[-tail // 64:] = torch.rand(tail // 64, device="cuda", generator=g)
    table = jb.Q4Table([(codes, scale, out * inner)])
    for dtype in ("f32", "bf16"):
        x = torch.randn(n, inner, device="cuda", generator=g).to(DT[dtype])
        got = jb.jb_q4_matmul(table, 0, x, out)
        w = dense(jb.Q4Table([(codes[-tail // 2:], scale[-tail // 64:], tail)]), 0, 40, inner)
        want = x.double() @ w.T
        assert (got[:, :-40] == 0).all()
        assert ((got[:, -40:].double() - want).abs() <= bound(x, w, None, want)).all()


# A matrix whose column k has the code k % 16 in all rows, scales of 1: a product with few inputs that are not zero tells
# how well each level is held, whatever the type of the result.
def columns_of_codes(out, inner):
    codes = torch.arange(inner, dtype=torch.uint8, device="cuda") & 15
    return jb.Q4Table([((codes[0::2] | codes[1::2] << 4).repeat(out), torch.ones(out * inner // 64, device="cuda"), out * inner)])


KERNELS = [(130, 704, 5), (777, 704, 64), (150, 4160, 64), (130, 65536, 33), (19, 65536, 7)]  # few rows; tiles; tiles; tiles; long


@pytest.mark.parametrize("out,inner,n", KERNELS)
def test_levels_enter_bf16_products_within_2_to_the_minus_12(out, inner, n):
    """An input of 1 at a code and one at the level -1 that takes away what bf16 has of the code's level: what is left is small
    and tells the level's own error, at most 2^-12 of it. The sum has two terms, 3 roundings of 2^-22 of 2, and the result is
    rounded once, half a step of bf16."""
    table = columns_of_codes(out, inner)
    level = torch.from_numpy(jb.jb_q4_levels()).cuda()
    assert level[0] == -1.0
    for block in (0, 1, inner // 128, inner // 64 - 1):
        for first in range(0, 16, n):
            x = torch.zeros(n, inner, dtype=torch.bfloat16, device="cuda")
            at = torch.arange(first, min(first + n, 16), device="cuda")
            x[at - first, 64 * block + 16 + at] = 1.0
            x[at - first, 64 * block + 32] = level[at].bfloat16()
            got = jb.jb_q4_matmul(table, 0, x, out)[:len(at)].double()
            want = (level[at].double() - level[at].bfloat16().double())[:, None].expand_as(got)
            tol = 2.0**-12 * level[at].double().abs()[:, None] + 3 * 2.0**-22 * 2 + 2.0**-8 * want.abs() + 1e-38
            assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).amax().item()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("out,inner,n", KERNELS)
@pytest.mark.parametrize("width", [1, 64])
def test_blocks_by_themselves(dtype, out, inner, n, width):
    """Inputs that are zero but for one column, or one block of 64, at the first, second, middle and last blocks: the allowance is
    that block's alone. With A = sum |x w|: fp32 levels and inputs are two fp16 numbers each, off by at most 2^-22, and the
    product of two lower parts, 2^-22, is left out; sums take a step for 16 terms, eight of them, each off by at most 2^-22; one
    more for scales and powers of two. bf16: levels 2^-12, four steps, the result half a step with the tie."""
    table, g = weights(out, inner, 3), torch.Generator(device="cuda").manual_seed(inner + n)
    w = dense(table, 0, out, inner)
    for block in (0, 1, inner // 128, inner // 64 - 1):
        k = 64 * block + (0 if width == 64 else 37)
        x = torch.zeros(n, inner, device="cuda")
        x[:, k:k + width] = torch.randn(n, width, device="cuda", generator=g)
        x = x.to(DT[dtype])
        got = jb.jb_q4_matmul(table, 0, x, out).double()
        want = x[:, k:k + width].double() @ w[:, k:k + width].T
        a = x[:, k:k + width].double().abs() @ w[:, k:k + width].abs().T
        tol = a * 12 * 2.0**-22 if dtype == "f32" else a * (2.0**-12 + 5 * 2.0**-22) + 2.0**-8 * want.abs()
        assert ((got - want).abs() <= tol + 1e-38).all(), (block, ((got - want).abs() / (tol + 1e-38)).amax().item())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_level_in_tiles(dtype):
    """Each code in each place of a block and both blocks of a pair, on the kernel that cuts matrices into tiles."""
    out, inner = 2049, 320
    table = weights(out, inner, 5)
    w = dense(table, 0, out, inner)
    for first in range(0, inner, 64):
        x = torch.zeros(64, inner, device="cuda", dtype=DT[dtype])
        at = torch.arange(64, device="cuda")
        x[at, first + at] = 1.5
        got = jb.jb_q4_matmul(table, 0, x, out).double()
        want = 1.5 * w[:, first:first + 64].T
        assert ((got - want).abs() <= want.abs() * (2.0**-8 + 2.0**-12 if dtype == "bf16" else 4 * 2.0**-22)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [24, 40, 100])
def test_tiles_read_weights_that_were_written_just_before(dtype, n):
    """Codes and scales change on the stream directly before each product, by the perturbation and by copies, eagerly and in a
    graph; the kernel reads them ahead of its inputs."""
    out, inner = 2100, 2048
    table = weights(out, inner)
    x = torch.randn(n, inner, device="cuda").to(DT[dtype])
    codes, scale, _ = table.tensors[0]
    steps = []
    for seed in (11, 12, 13):
        other = weights(out, inner, seed).tensors[0]
        steps.append(lambda other=other: (codes.copy_(other[0]), scale.copy_(other[1])))
        steps.append(lambda: jb.jb_perturb_q4(table, (5, 1, 0), 1e-2))
    def wanted(got):
        w = dense(table, 0, out, inner)
        want = x.double() @ w.T
        assert ((got.double() - want).abs() <= bound(x, w, None, want)).all()
    torch.cuda.synchronize()
    for step in steps:
        step()
        wanted(jb.jb_q4_matmul(table, 0, x, out))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    y = torch.empty(len(steps), n, out, dtype=DT[dtype], device="cuda")
    with torch.cuda.graph(graph):
        for i, step in enumerate(steps):
            step()
            jb.jb_q4_matmul(table, 0, x, out, out=y[i])
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for i, step in enumerate(steps):
        step()
        assert torch.equal(jb.jb_q4_matmul(table, 0, x, out), y[i])
