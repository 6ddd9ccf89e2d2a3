"""PagedCache.attend and cross_attention against attention in 64 bits (attention_util says what the tolerances count)."""
import math
import random

import pytest
import torch

from attention_util import attention64, check, check_cache_attention, check_lse, gen, randn, strided_heads
from paper_1908_11263_gb300 import qnn

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16


def paged(g, dtype, news, lengths, heads, kv, d, page, layout="heads", pad=0, nan=True, mul=2.0, spare=3):
    """(cache, table, lengths, offsets, q): pages in random order, NaN in every row that no sequence has."""
    width = max(1, max(-(-n // page) for n in lengths))
    used = [-(-n // page) for n in lengths]
    pages = sum(used) + spare
    shape = (pages, kv, page, d) if layout == "heads" else (pages, page, kv, d)
    kp, vp = (randn(g, *shape, dtype=dtype) for _ in range(2))
    if layout != "heads":
        kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
    ids = torch.randperm(pages, generator=g, device="cuda").int()
    table = torch.full((len(news), width), -1, dtype=torch.int32, device="cuda")
    live = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
    at = 0
    for s, n in enumerate(used):
        table[s, :n] = ids[at:at + n]
        for c in range(n):
            live[ids[at + c], :lengths[s] - c * page] = True
        at += n
    if nan:
        for t in (kp, vp):
            t.masked_fill_(~live[:, None, :, None], math.nan)
    offsets = torch.tensor([0] + news, device="cuda").cumsum(0).int()
    q = strided_heads(g, sum(news), heads, d, dtype, pad, mul=mul)
    return qnn.PagedCache(kp, vp), table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), offsets, q


def run(cache, table, lengths, offsets, q, name="", **kw):
    out, lse = cache.attend(q, table, lengths, offsets, lse=True, **kw)
    assert out.shape == q.shape and out.dtype == q.dtype and lse.shape == q.shape[:2] and lse.dtype == torch.float32
    check_cache_attention(out, lse, q, cache.k, cache.v, table, lengths, offsets, name=name, **kw)
    assert torch.equal(cache.attend(q, table, lengths, offsets, **kw), out)  # the same each time
    return out, lse


# single tokens: many lengths in one batch, across the borders of keys' units and of pages
LENGTHS = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 1000, 3, 700]


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("heads,kv,d,page,layout,pad,window", [
    (32, 8, 128, 16, "heads", 0, None), (32, 8, 128, 64, "rows", 0, 100), (8, 8, 64, 24, "heads", 40, 64), (5, 1, 80, 7, "rows", 6, None),
    (40, 2, 96, 128, "heads", 0, 1), (64, 1, 64, 1, "rows", 0, None), (4, 2, 256, 32, "heads", 0, None), (3, 3, 8, 16, "heads", 1, 33),
    (10, 5, 200, 5, "rows", 0, 500)])
def test_one_token(dtype, heads, kv, d, page, layout, pad, window):
    g = gen(heads * 1000 + d + page)
    run(*paged(g, dtype, [1] * len(LENGTHS), LENGTHS, heads, kv, d, page, layout, pad), window=window)


@pytest.mark.parametrize("length", [1, 64, 65, 5000, 40001])
@pytest.mark.parametrize("heads,kv,d", [(32, 8, 128), (4, 4, 64), (7, 1, 256)])
def test_one_user(length, heads, kv, d):
    """One sequence over all blocks; without offsets."""
    cache, table, lengths, offsets, q = paged(gen(length + d), BF, [1], [length], heads, kv, d, 64)
    out, _ = run(cache, table, lengths, offsets, q)
    assert torch.equal(cache.attend(q, table, lengths), out)


MANY = [
    # news, lengths
    ([5, 1, 0, 130, 2, 64, 33], [5, 90, 40, 130, 700, 129, 1000]),
    ([1, 300, 1, 1, 17], [3000, 400, 1, 64, 17]),
    ([257], [257]), ([1000, 900], [1000, 2500]), ([128, 129, 127, 1], [128, 129, 127, 128])]


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("news,lengths", MANY)
@pytest.mark.parametrize("heads,kv,d,page,layout,pad,kw", [
    (8, 2, 128, 64, "heads", 0, {}), (4, 4, 64, 24, "rows", 8, dict(window=70)), (6, 2, 80, 16, "heads", 6, dict(causal=False)),
    (5, 1, 96, 128, "rows", 0, dict(window=300, scale=0.3)), (2, 1, 256, 32, "heads", 0, dict(window=1)),
    (10, 2, 128, 48, "rows", 0, dict(window=200, causal=False)), (3, 1, 40, 256, "heads", 0, {})])
def test_many_tokens(dtype, news, lengths, heads, kv, d, page, layout, pad, kw):
    g = gen(sum(news) + heads * 100 + d)
    run(*paged(g, dtype, news, lengths, heads, kv, d, page, layout, pad), **kw)


@pytest.mark.parametrize("news", [[1, 1, 1], [4, 40, 400]])
@pytest.mark.parametrize("d", [64, 128])
def test_tokens_that_see_nothing(news, d):
    """Lengths of zero, below the new tokens' number and negative; pages that are not there; rows in no sequence."""
    g = gen(d)
    cache, table, lengths, offsets, q = paged(g, BF, news, [50, 500, 600], 8, 2, d, 16)
    lengths = torch.tensor([0, max(1, news[1] // 2), 600], dtype=torch.int32, device="cuda")
    table[2, :20] = -1
    table[2, 25] = cache.pages
    table[2, 30] = -(1 << 31)
    out, lse = run(cache, table, lengths, offsets, q, "holes")
    assert bool((out[:news[0]] == 0).all()) and bool((lse[:news[0]] == -math.inf).all())
    lengths[0] = -5
    table[2] = -1
    out, lse = run(cache, table, lengths, offsets, q, "holes")
    assert bool((out[offsets[2]:] == 0).all()) and bool((lse[offsets[2]:] == -math.inf).all())
    out, lse = run(cache, table, lengths, offsets, q, window=3, causal=False)
    # more than the table holds; the last page's free rows are keys now, and have to be finite
    cache.k.nan_to_num_(0.5), cache.v.nan_to_num_(0.5)
    lengths[1] = table.shape[1] * 16 + 7
    run(cache, table, lengths, offsets, q)


def test_rows_in_no_sequence_stay():
    for news, lengths in (([3, 1, 2, 1], [30, 70, 2, 9]), ([3, 200, 300, 5], [30, 700, 300, 9])):
        cache, table, lens, offsets, q = paged(gen(2), BF, news, lengths, 4, 2, 64, 16)
        out = torch.full_like(q, 7.0)
        part = table[1:3], lens[1:3].contiguous(), offsets[1:4].contiguous()
        assert cache.attend(q, *part, out=out) is out
        check_cache_attention(out, None, q, cache.k, cache.v, *part)
        lo, hi = int(offsets[1]), int(offsets[3])
        assert bool((out[:lo] == 7).all()) and bool((out[hi:] == 7).all())


@pytest.mark.parametrize("n", [1, 40, 300])
def test_large_scores(n):
    """Scores in the thousands: the maximum moves by much from key to key, float16 weights reach its smallest numbers."""
    for dtype in (BF, F16):
        cache, table, lengths, offsets, q = paged(gen(n), dtype, [n], [n + 700], 4, 2, 64, 16, mul=40.0)
        cache.k.mul_(torch.linspace(0.01, 4, 16, device="cuda").to(dtype)[None, None, :, None])
        run(cache, table, lengths, offsets, q, scale=1.0)
        run(cache, table, lengths, offsets, q, scale=1e-6)


def test_strided_outputs_and_orders():
    for n in (1, 200):
        g = gen(n)
        cache, table, lengths, offsets, q = paged(g, F16, [n, n], [n + 30, n], 4, 2, 64, 16)
        want, even = cache.attend(q, table, lengths, offsets), cache.attend(q, table, lengths)  # may be other kernels
        check_cache_attention(even, None, q, cache.k, cache.v, table, lengths, offsets)
        for make in (lambda: torch.full((2 * n, 4, 65), 7.0, dtype=F16, device="cuda")[..., :64],
                     lambda: torch.full((4, 2 * n, 72), 7.0, dtype=F16, device="cuda")[..., 1:65].transpose(0, 1),
                     lambda: torch.full((2 * n, 4, 72), 7.0, dtype=F16, device="cuda")[..., :64]):
            out = make()
            whole = out._base if out._base is not None else out
            cache.attend(q, table, lengths, offsets, out=out)
            assert torch.equal(out, want)
            assert int((whole == 7).sum()) >= whole.numel() - out.numel()
            assert torch.equal(cache.attend(q, table, lengths, out=out), even)
        other = q.transpose(0, 1).contiguous().transpose(0, 1)
        assert torch.equal(cache.attend(other, table, lengths, offsets), want)
        one = q[:, :1].expand(2 * n, 4, 64)
        assert torch.equal(cache.attend(one, table, lengths, offsets), cache.attend(one.contiguous(), table, lengths, offsets))
        far = torch.full((2, 40), -1, dtype=torch.int32, device="cuda")  # a wider table with other columns behind
        far[:, :table.shape[1]] = table
        assert torch.equal(cache.attend(q, far[:, :table.shape[1]], lengths, offsets), want)


def test_pages_past_32_bits():
    """A cache of more than 2^32 elements: pages at both ends."""
    page, kv, d = 64, 8, 128
    pages = (1 << 32) // (page * kv * d) + 40
    k = torch.zeros(pages, kv, page, d, dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    cache = qnn.PagedCache(k, v)
    g = gen(1)
    ids = torch.tensor([[pages - 1, 0, pages - 20, 1], [pages // 2, pages - 2, 3, 4]], dtype=torch.int32, device="cuda")
    for n in (1, 150):
        lengths = torch.tensor([230, 190], dtype=torch.int32, device="cuda")
        offsets = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
        kn, vn = randn(g, 420, kv, d), randn(g, 420, kv, d)
        cache.append(kn, vn, ids, lengths, torch.tensor([0, 230, 420], dtype=torch.int32, device="cuda"))
        q = randn(g, 2 * n, 16, d)
        run(cache, ids, lengths, offsets, q)


# ---------------------------------------------------------------- cross attention

def check_cross(q, k, v, lengths, out, lse, scale=None, name=""):
    b, n, heads, d = q.shape
    scale = 1 / math.sqrt(d) if scale is None else scale
    for i in range(b):
        keys = k.shape[1] if lengths is None else max(0, min(int(lengths[i]), k.shape[1]))
        seen = torch.ones(n, keys, dtype=torch.bool, device="cuda")
        want, err, wl, le = attention64(q[i], k[i, :keys], v[i, :keys], seen, scale)
        check(out[i], want, err, f"{name} batch {i}")
        if lse is not None:
            check_lse(lse[i], wl, le, f"{name} batch {i}")


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("b,n,src,heads,kv,d", [
    (1, 1, 1, 1, 1, 64), (3, 1, 333, 20, 20, 64), (5, 77, 333, 10, 5, 80), (2, 448, 1500, 4, 4, 64), (4, 129, 257, 8, 2, 128),
    (2, 16, 63, 6, 6, 96), (3, 300, 64, 2, 1, 256), (2, 1, 5000, 8, 1, 128), (1, 1000, 2, 3, 1, 128), (2, 130, 1000, 8, 8, 40),
    (6, 300, 777, 8, 4, 80), (4, 500, 1030, 8, 2, 128), (3, 1000, 600, 20, 5, 40), (20, 40, 513, 16, 4, 64)])
@pytest.mark.parametrize("packed", [False, True])
def test_cross(dtype, b, n, src, heads, kv, d, packed):
    g = gen(b * n + src)
    q = randn(g, b, n, heads, d, dtype=dtype, mul=2.0)
    if packed:  # both of one projection, the queries heads first
        k, v = randn(g, b, src, 2, kv, d, dtype=dtype).unbind(2)
        q = q.transpose(1, 2).contiguous().transpose(1, 2)
    else:
        k, v = randn(g, b, src, kv, d, dtype=dtype), randn(g, b, src, kv, d, dtype=dtype)
    out, lse = qnn.cross_attention(q, k, v, lse=True)
    assert out.shape == q.shape and lse.shape == q.shape[:3]
    check_cross(q, k, v, None, out, lse)
    rng = random.Random(n)
    lengths = torch.tensor([rng.choice([0, 1, src, src + 9, rng.randint(0, src)]) for _ in range(b)], dtype=torch.int32, device="cuda")
    for i in range(b):
        k[i, max(int(lengths[i]), 0):] = math.nan
        v[i, max(int(lengths[i]), 0):] = math.nan
    out, lse = qnn.cross_attention(q, k, v, lengths, lse=True, scale=0.2)
    check_cross(q, k, v, lengths, out, lse, 0.2)
    assert torch.equal(qnn.cross_attention(q, k, v, lengths, scale=0.2), out)


def test_empty_cross():
    q = torch.ones(2, 3, 4, 64, dtype=BF, device="cuda")
    none = torch.zeros(2, 0, 2, 64, dtype=BF, device="cuda")
    out, lse = qnn.cross_attention(q, none, none, lse=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    assert qnn.cross_attention(q[:0], none[:0], none[:0]).shape == (0, 3, 4, 64)
    assert qnn.cross_attention(q[:, :0], none, none).shape == (2, 0, 4, 64)


# ---------------------------------------------------------------- both halves of a tile, and halves without rows

@pytest.mark.parametrize("d", [64, 128])
def test_tiles_without_rows_in_one_half_before_others(d):
    """Many sequences whose rows fill one half of a tile (34 to 128), then some that fill both, many times in a block's share:
    the second half's warps pass the first ones by."""
    news = [30, 64, 17, 50] * 12 + [300, 33, 40, 600] * 3
    lengths = [n + 900 * (i % 5) for i, n in enumerate(news)]
    run(*paged(gen(d), BF, news, lengths, 2, 1, d, 16))


def test_windows_inside_a_tile():
    """Windows shorter than a tile's queries: its first keys are seen by its first rows only."""
    for window in (1, 5, 127, 128, 129, 400):
        run(*paged(gen(window), F16, [700, 90], [1500, 90], 2, 2, 64, 32), window=window)


@pytest.mark.parametrize("group", [3, 12, 20, 33, 64, 96])
def test_shared_heads_that_do_not_divide_a_tile(group):
    run(*paged(gen(group), BF, [37, 1, 90], [500, 300, 90], 2 * group, 2, 64, 16, pad=16))


@pytest.mark.parametrize("d", [8, 24, 40, 72, 104, 120])
@pytest.mark.parametrize("pad", [0, 6])
def test_heads_that_end_inside_a_step(d, pad):
    """Heads of an odd number of eights: the products take sixteen columns at a time, and the columns behind a head are zeros,
    also where q is not aligned.  Infinities in the rows of other tokens and heads may not reach them."""
    for dtype in (BF, F16):
        cache, table, lengths, offsets, q = paged(gen(d + pad), dtype, [300, 21, 130], [400, 90, 1000], 6, 2, d, 16, pad=pad)
        run(cache, table, lengths, offsets, q)
        q[310] = math.inf  # one token's queries: its own output has no value, all others have
        out, lse = cache.attend(q, table, lengths, offsets, lse=True)
        good = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
        good[310] = False
        assert bool(out[good].isfinite().all()) and bool(lse[good].isfinite().all())
        assert bool(out[310].isnan().all()) and bool(lse[310].isnan().all())


def test_a_token_without_a_value_where_few_rows_are_streamed():
    cache, table, lengths, offsets, q = paged(gen(3), BF, [1] * 4, [900, 40, 3000, 70], 8, 2, 128, 16)
    q[2] = math.nan
    out, lse = cache.attend(q, table, lengths, lse=True)
    assert bool(out[2].isnan().all()) and bool(lse[2].isnan().all())
    keep = [0, 1, 3]
    assert bool(out[keep].isfinite().all()) and bool(lse[keep].isfinite().all())
