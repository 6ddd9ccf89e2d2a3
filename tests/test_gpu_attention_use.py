"""The attention operators as they are used together: a block's attention half over several steps, captured steps that are
replayed with other lengths, calls on other streams and from several threads."""
import math

import pytest
import torch

from attention_util import attention64, check, check_cache_attention, gen, randn, rotate64
from paper_1908_11263_gb300 import qnn
from test_gpu_attention import paged
from test_gpu_streams import WAIT, outputs, results
from test_gpu_threads import check as check_threads

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16


class Block:
    """The attention half of a decoder block with a cache, and cross attention to an encoder's states."""

    def __init__(self, g, dtype, hidden, heads, kv, d, page, pages, seqs, width):
        self.heads, self.kv, self.d, self.dtype = heads, kv, d, dtype
        w = lambda m, k: (torch.randn(m, k, generator=g, device="cuda") / math.sqrt(k)).to(dtype)  # noqa: E731
        self.qkv, self.out = qnn.PreparedMatmul(w((heads + 2 * kv) * d, hidden)), qnn.PreparedMatmul(w(hidden, heads * d))
        self.cache = qnn.PagedCache(torch.zeros(pages, kv, page, d, dtype=dtype, device="cuda"),
                                    torch.zeros(pages, kv, page, d, dtype=dtype, device="cuda"))
        self.rotary = qnn.Rotary(d, scaling="ramp", factor=4.0, context=128, low=1.0, high=4.0)
        self.table = torch.randperm(pages, generator=g, device="cuda")[:seqs * width].view(seqs, width).int()

    def step(self, x, lengths, offsets, states):
        _, h = qnn.block_norm(x)
        parts = self.qkv(h).split([self.heads * self.d, self.kv * self.d, self.kv * self.d], 1)
        q, k, v = (p.unflatten(1, (-1, self.d)) for p in parts)
        q = self.cache.append(k, v, self.table, lengths, offsets, rotary=self.rotary, q=q)
        o = self.cache.attend(q, self.table, lengths, offsets)
        y = self.out(o.flatten(1), x)
        if states is not None:  # as many new tokens in every sequence
            n = x.shape[0] // self.table.shape[0]
            c = qnn.cross_attention(q.unflatten(0, (-1, n)), *states)
            y = self.out(c.flatten(0, 1).flatten(1), y)
        return y, q, k, v, o


@pytest.mark.parametrize("dtype,heads,kv,d,page", [(BF, 8, 2, 128, 16), (F16, 4, 4, 64, 24)])
def test_prompts_then_tokens(dtype, heads, kv, d, page):
    """Prompts of two sequences in chunks, then tokens one by one: the cache holds the rotated keys at their places, and every
    output is the attention of all tokens so far."""
    g = gen(d)
    hidden, width = 256, 40
    block = Block(g, dtype, hidden, heads, kv, d, page, 2 * width + 3, 2, width)
    chunks = [[70, 33], [130, 1], [1, 1], [1, 1], [5, 300], [1, 1]]
    lengths = [0, 0]
    turns = [t % (1 << 64) for t in block.rotary.turns.tolist()]
    seen_k, seen_v = [[], []], [[], []]
    for news in chunks:
        lengths = [a + b for a, b in zip(lengths, news)]
        x = randn(g, sum(news), hidden, dtype=dtype)
        lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        offsets = torch.tensor([0, news[0], sum(news)], dtype=torch.int32, device="cuda")
        _, q, k, v, o = block.step(x, lens, None if news == [1, 1] else offsets, None)
        check_cache_attention(o, None, q, block.cache.k, block.cache.v, block.table, lens, offsets)
        for s in range(2):
            rows = slice(0, news[0]) if s == 0 else slice(news[0], sum(news))
            seen_k[s].append(k[rows].clone())
            seen_v[s].append(v[rows].clone())
    for s in range(2):
        p = torch.arange(lengths[s], device="cuda")
        pages, rows = block.table[s, p // page].long(), p % page
        want, err = rotate64(torch.cat(seen_k[s]), p.tolist(), turns, 0, 1.0)
        check(block.cache.k[pages, :, rows], want, err)
        assert torch.equal(block.cache.v[pages, :, rows], torch.cat(seen_v[s]))


def test_a_captured_step_is_replayed_with_other_lengths():
    """Two graphs of the same step, replayed in turns; lengths, tables and inputs change in place."""
    g = gen(9)
    seqs, width, page, d = 3, 60, 16, 128
    blocks = [Block(gen(5), BF, 256, 8, 2, d, page, seqs * width, seqs, width) for _ in range(2)]
    states = tuple(randn(g, seqs, 90, 2, d) for _ in range(2))
    x = randn(g, seqs, 256)
    lengths = torch.ones(seqs, dtype=torch.int32, device="cuda")
    blocks[0].step(x, lengths, None, states)
    torch.cuda.synchronize()
    graphs, ys = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = blocks[0].step(x, lengths, None, states)[0]
        graphs.append(graph)
        ys.append(y)
    blocks[0].cache.k.zero_(), blocks[0].cache.v.zero_()
    for i, lens in enumerate(([1, 1, 1], [2, 2, 2], [3, 500, 3], [4, 501, 960], [5, 502, 1])):
        lengths.copy_(torch.tensor(lens, dtype=torch.int32))
        x.copy_(randn(g, seqs, 256))
        graphs[i % 2].replay()
        want = blocks[1].step(x, lengths, None, states)[0]
        assert torch.equal(ys[i % 2], want), lens
    graphs[0].replay()
    graphs[1].replay()
    assert torch.equal(ys[0], ys[1])


def test_a_captured_prompt_with_other_offsets():
    g = gen(4)
    cache, table, lengths, offsets, q = paged(g, BF, [100, 30, 20], [400, 90, 300], 8, 2, 64, 16, nan=False)
    cache.attend(q, table, lengths, offsets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = cache.attend(q, table, lengths, offsets, lse=True)
    for cut in ([0, 100, 130, 150], [0, 1, 149, 150], [0, 0, 0, 150], [0, 50, 60, 61]):
        offsets.copy_(torch.tensor(cut, dtype=torch.int32))
        out.fill_(7), lse.fill_(7)
        graph.replay()
        check_cache_attention(out, lse, q, cache.k, cache.v, table, lengths, offsets, name=str(cut))
        assert bool((out[cut[-1]:] == 7).all()) and bool((lse[cut[-1]:] == 7).all())


def every_call():
    """Name -> a function of the stream; in-place updates leave the same values each time."""
    g = gen(12)
    one = paged(g, BF, [1] * 5, [700, 3, 64, 900, 128], 8, 2, 128, 16, nan=False)
    many = paged(g, BF, [200, 1, 40], [700, 64, 900], 4, 2, 64, 16, nan=False)
    k, v = randn(g, 241, 2, 64), randn(g, 241, 2, 64)
    rotary, x = qnn.Rotary(64), randn(g, 50, 4, 64)
    positions = torch.arange(50, device="cuda")
    qc, kc, vc = randn(g, 3, 70, 4, 64), randn(g, 3, 200, 2, 64), randn(g, 3, 200, 2, 64)
    cache = qnn.PagedCache(many[0].k.clone(), many[0].v.clone())
    return {
        "rope": lambda s: qnn.rope(x, positions, rotary, stream=s),
        "append": lambda s: cache.append(k, v, *many[1:4], rotary=rotary, q=many[4], stream=s),
        "one token": lambda s: one[0].attend(one[4], one[1], one[2], lse=True, stream=s),
        "many tokens": lambda s: many[0].attend(many[4], many[1], many[2], many[3], lse=True, stream=s),
        "cross": lambda s: qnn.cross_attention(qc, kc, vc, lse=True, stream=s),
    }


NAMES = ["rope", "append", "one token", "many tokens", "cross"]


@pytest.mark.parametrize("name", NAMES)
def test_memory_that_the_current_stream_still_reads(name):
    every = every_call()
    assert sorted(every) == sorted(NAMES)
    call, side = every[name], torch.cuda.Stream()
    torch.cuda.synchronize()
    want = [o.clone() for o in results(call(None))]
    sizes = [o.untyped_storage().nbytes() for o in outputs(call(side))]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    read = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    held = [torch.full((n,), 3, dtype=torch.uint8, device="cuda") for n in sizes]
    torch.cuda.synchronize()
    torch.cuda._sleep(WAIT)
    for r, h in zip(read, held):
        r.copy_(h)
    h = None
    held.clear()
    got = call(side)
    torch.cuda.synchronize()
    assert all(bool((r == 3).all()) for r in read)
    assert all(torch.equal(a, b) for a, b in zip(results(got), want))


def test_threads_on_one_stream():
    every = every_call()
    check_threads([lambda f=f: tuple(results(f(None))) for f in every.values()], rounds=100)


def test_a_rotation_made_on_another_stream():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(WAIT)
    r = qnn.Rotary(64, stream=side)
    side.synchronize()
    x, p = randn(gen(1), 9, 2, 64), torch.arange(9, device="cuda")
    assert torch.equal(qnn.rope(x, p, r), qnn.rope(x, p, qnn.Rotary(64)))


def test_weights_of_one_key_and_lse_join():
    """lse joins the attention over two parts of the keys: the same as over both."""
    g = gen(21)
    q, k, v = randn(g, 2, 50, 8, 64), randn(g, 2, 300, 2, 64), randn(g, 2, 300, 2, 64)
    (a, la), (b, lb) = (qnn.cross_attention(q, k[:, s].contiguous(), v[:, s].contiguous(), lse=True) for s in (slice(0, 1), slice(1, 300)))
    w = torch.softmax(torch.stack([la, lb]).double(), 0)[..., None]
    joined = w[0] * a.double() + w[1] * b.double()
    for i in range(2):
        want, err, _, _ = attention64(q[i], k[i], v[i], torch.ones(50, 300, dtype=torch.bool, device="cuda"), 0.125)
        # each part is rounded once more to bf16
        assert bool(((joined[i] - want).abs() <= 2 * err + 2.0 ** -8 * (w[0, i] * a[i].double().abs() + w[1, i] * b[i].double().abs()) * 1.01).all())
