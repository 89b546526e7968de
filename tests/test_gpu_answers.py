"""The calls together, as examples/spsa_answers.py uses them: answers against a model without a cache, the same
answers again from the same words, and training steps that repeat bit for bit."""
import importlib.util
import os

import pytest
import torch

import paper_2306_10015_gb300 as jb

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("spsa_answers", os.path.join(ROOT, "examples", "spsa_answers.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def plain_logits(model, tokens):
    """The decoder over one whole sequence in 64 bits, without a cache."""
    p = {k: v.double() for k, v in model.p.items()}
    t, h = len(tokens), model.heads
    x = p["tokens"][tokens.long()] + p["positions"][:t]
    norm = lambda v, w: torch.nn.functional.layer_norm(v, (model.d,)) * w  # noqa: E731
    mask = torch.full((t, t), -torch.inf, device="cuda", dtype=torch.float64).triu(1)
    for i in range(model.layers):
        q, k, v = (norm(x, p[f"{i}.norm1"]) @ p[f"{i}.qkv"].T).view(t, 3, h, -1).permute(1, 2, 0, 3)
        w = torch.softmax(q @ k.transpose(1, 2) * (model.d // h) ** -0.5 + mask, -1)
        x = x + (w @ v).transpose(0, 1).reshape(t, model.d) @ p[f"{i}.out"].T
        x = x + torch.relu(norm(x, p[f"{i}.norm2"]) @ p[f"{i}.fc1"].T) @ p[f"{i}.fc2"].T
    return norm(x, p["norm"]) @ p["tokens"].T


def test_answers_have_the_probabilities_of_the_whole_sequence(ex):
    """fp32 weights: the log-probability that a token was drawn with is that of a model without pages. Two layers
    of fp32 products of up to 1024 terms and norms of order 1: a thousand roundings of 2^-24, taken linearly
    and times ten for logits of that size, 1e-3."""
    model = ex.Decoder(dtype=torch.float32, seed=3)
    prompts = torch.randint(3, model.vocab, (3, 21), device="cuda", dtype=torch.int32)
    out, lp = ex.write_answers(model, prompts, 3, 20, (5, 6, 7), top_p=1.0)
    for i in range(9):
        answer = out[i][out[i] >= 0]
        seq = torch.cat([prompts[i // 3], answer])
        want = torch.log_softmax(plain_logits(model, seq)[20:-1], -1).gather(1, answer.long()[:, None])[:, 0]
        assert (lp[i][: len(answer)].double() - want).abs().max() < 1e-3
        ended = (answer == ex.END).nonzero()
        assert len(answer) == 20 or ended[0].item() == len(answer) - 1


def test_the_same_words_write_the_same_answers(ex):
    model = ex.Decoder(seed=4)
    prompts = torch.randint(3, model.vocab, (2, 33), device="cuda", dtype=torch.int32)
    a, la = ex.write_answers(model, prompts, 5, 16, (1, 2, 3))
    b, lb = ex.write_answers(model, prompts, 5, 16, (1, 2, 3))
    c, _ = ex.write_answers(model, prompts, 5, 16, (1, 2, 4))
    assert torch.equal(a, b) and torch.equal(la, lb) and not torch.equal(a, c)
    assert len({tuple(r.tolist()) for r in a}) > 2          # forks of one prompt go their own ways


def test_training_steps_repeat(ex):
    a, m = ex.train(steps=2, log=lambda *_: None)
    b, n = ex.train(steps=2, log=lambda *_: None)
    assert a == b and all(torch.equal(x, y) for x, y in zip(m.p.values(), n.p.values()))
    assert all(0 <= p <= 1 and 0 <= q <= 1 for p, q, _ in a)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_whole_step_in_a_graph(dtype):
    """Free, compact, reserve, fork, write, attention and the draw, captured once and replayed, against the same calls
    made one by one on a cache of the same contents: every table, page, output and token."""
    i32 = dict(dtype=torch.int32, device="cuda")

    def make():
        g = torch.Generator(device="cuda").manual_seed(11)
        pages = jb.PageTable.empty(9, 90, 400, 16)
        kv = [torch.randn(400, 2, 16, 64, generator=g, device="cuda").to(dtype) for _ in range(4)]
        cache = jb.KVCache(pages, kv[:2], kv[2:])
        assert jb.jb_cache_reserve(cache, torch.arange(4, **i32), torch.tensor([700, 21, 16, 1], **i32)).item() == 0
        q, new = (torch.randn(n, 8, h, 64, generator=g, device="cuda").to(dtype) for n, h in ((2, 4), (4, 2)))
        return cache, q, new, torch.randn(8, 500, generator=g, device="cuda").to(dtype)

    children = torch.tensor([4, 5, 6, 7], **i32)
    rows, one = torch.arange(8, **i32), torch.ones(8, **i32)

    def step(cache, q, new, logits, words, out):
        pages = cache.pages
        jb.jb_cache_free(cache, children)
        jb.jb_cache_compact(cache, status=out["live"])
        jb.jb_cache_fork(cache, rows[:4], children, status=out["forked"])
        pos = pages.lens[:8].clone()
        jb.jb_cache_reserve(cache, rows, one, status=out["room"])
        for i in range(2):
            jb.jb_cache_write(cache, i, new[2 * i], new[2 * i + 1], rows, pos)
            jb.jb_attend(cache, i, q[i], rows, pos, out=out["o"][i])
        jb.jb_sample(logits, words, temperature=0.8, top_k=60, top_p=0.9, tokens=out["tokens"], logprobs=out["logprobs"])

    def results():
        return dict(live=torch.zeros(1, **i32), forked=torch.zeros(1, **i32), room=torch.zeros(1, **i32), tokens=torch.zeros(8, **i32),
                    o=torch.zeros(2, 8, 4, 64, dtype=dtype, device="cuda"), logprobs=torch.zeros(8, device="cuda"))

    words = torch.zeros(8, **i32)
    eager, captured = make(), make()
    want, got = results(), results()
    step(*eager, words, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(*captured, words, got)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*captured, words, got)
    for turn in range(40):
        words.copy_(torch.randint(-2**31, 2**31, (8,), device="cuda").int())
        step(*eager, words, want)
        graph.replay()
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(want[name], got[name]), (turn, name)
        for a, b in zip((eager[0].pages.table, eager[0].pages.lens, eager[0].pages.refs), (captured[0].pages.table, captured[0].pages.lens, captured[0].pages.refs)):
            assert torch.equal(a, b)
    for a, b in zip(eager[0].keys + eager[0].values, captured[0].keys + captured[0].values):
        assert torch.equal(a, b)
    assert want["forked"].item() == want["room"].item() == 0
