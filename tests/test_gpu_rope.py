"""qnn.rope and PagedCache.append against the rotation in 64 bits (attention_util says what the tolerances count)."""
import math

import pytest
import torch

from attention_util import check, gen, randn, rotate64, strided_heads
from paper_1908_11263_gb300 import qnn

pytestmark = pytest.mark.gpu
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def turns_of(rotary):
    return [v % (1 << 64) for v in rotary.turns.tolist()]


def check_rope(x, positions, rotary, got, name=""):
    want, err = rotate64(x, [int(p) for p in positions], turns_of(rotary), rotary.interleaved, rotary.amplitude)
    check(got, want, err, name)


@pytest.mark.parametrize("dtype", [BF, F16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("t,heads,d,dim,pad", [(1, 1, 2, 2, 0), (1, 32, 128, 128, 0), (3, 5, 96, 64, 24), (700, 3, 80, 80, 6),
                                               (129, 2, 128, 64, 64), (2, 1, 1024, 1024, 0), (7, 3, 33, 10, 1), (5000, 2, 64, 48, 0)])
def test_rope(dtype, interleaved, t, heads, d, dim, pad):
    g = gen(t * 131 + d)
    x = strided_heads(g, t, heads, d, dtype, pad)
    positions = torch.randint(0, 131072, (t,), generator=g, device="cuda")
    rotary = qnn.Rotary(dim, interleaved=interleaved, amplitude=1.25)
    y = qnn.rope(x, positions, rotary)
    assert y.shape == x.shape and y.dtype == dtype and y.is_contiguous()
    check_rope(x, positions, rotary, y)
    assert torch.equal(y[..., dim:], x[..., dim:])
    assert torch.equal(qnn.rope(x, positions.int(), rotary), y)
    before = x.clone()
    qnn.rope(x, positions, rotary, out=x)
    assert torch.equal(x, y)
    qnn.rope(x, -positions, qnn.Rotary(dim, interleaved=interleaved, amplitude=1 / 1.25), out=x)  # turns back, twice rounded
    u = {BF: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -20}[dtype]
    assert bool(((x - before).abs().float() <= 4 * u * (1 + before.abs().float().amax(-1, keepdim=True))).all())


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "ramp"])
def test_far_positions(scaling):
    positions = [0, 1, -1, 2 ** 20 + 1, 10 ** 6, 2 ** 31 - 1, -2 ** 31, 2 ** 40 + 12345, -(2 ** 52) + 1, 2 ** 63 - 1]
    x = randn(gen(3), len(positions), 4, 128, dtype=F32)
    rotary = qnn.Rotary(128, scaling=scaling, factor=8.0, context=8192)
    p = torch.tensor(positions, device="cuda")
    check_rope(x, positions, rotary, qnn.rope(x, p, rotary), scaling)
    check_rope(x[:7], positions[:7], rotary, qnn.rope(x[:7], p[:7].int(), rotary), scaling)


def test_frequencies_of_ones_own_and_orders():
    g = gen(5)
    f = [0.5, 3.0, -0.25, 1e-6]
    x = randn(g, 6, 3, 20, dtype=F16).transpose(0, 1).contiguous().transpose(0, 1)  # heads apart, tokens within
    p = torch.arange(6, device="cuda")
    rotary = qnn.Rotary(8, frequencies=f)
    got = qnn.rope(x, p, rotary)
    angle = p.double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda")
    a, b = x[..., :4].double(), x[..., 4:8].double()
    want = torch.cat([a * torch.cos(angle)[:, None] - b * torch.sin(angle)[:, None],
                      a * torch.sin(angle)[:, None] + b * torch.cos(angle)[:, None], x[..., 8:].double()], -1)
    check(got, want, 2.0 ** -20 * want.abs().amax(-1, keepdim=True).expand_as(want))
    out = torch.full((6, 3, 24), math.nan, dtype=F16, device="cuda")
    assert qnn.rope(x, p, rotary, out=out[..., :20]) is not None
    assert torch.equal(out[..., :20], got) and bool(out[..., 20:].isnan().all())
    wide = x[:, :1].expand(6, 3, 20)  # one head for all
    assert torch.equal(qnn.rope(wide, p, rotary), qnn.rope(wide.contiguous(), p, rotary))


def test_nothing_to_rotate():
    rotary = qnn.Rotary(8)
    p = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert qnn.rope(torch.zeros(0, 3, 8, dtype=BF, device="cuda"), p, rotary).shape == (0, 3, 8)


# ---------------------------------------------------------------- into the cache

def append_case(g, dtype, news, cached, heads, kv, d, page, layout="heads", pad=0, holes=()):
    """(cache, table, lengths, offsets, k, v, q); pages filled with random values, table entries in `holes` are -1."""
    lengths = [a + b for a, b in zip(news, cached)]
    width = max(1, -(-max(lengths) // page))
    pages = width * len(news) + 2
    shape = (pages, kv, page, d) if layout == "heads" else (pages, page, kv, d)
    kp, vp = (randn(g, *shape, dtype=dtype) for _ in range(2))
    if layout != "heads":
        kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
    table = torch.randperm(pages, generator=g, device="cuda")[:width * len(news)].view(len(news), width).int()
    for s, c in holes:
        table[s, c] = -1
    offsets = torch.tensor([0] + news, device="cuda").cumsum(0).int()
    t = sum(news)
    q, k, v = (strided_heads(g, t, h, d, dtype, pad) for h in (heads, kv, kv))
    return qnn.PagedCache(kp, vp), table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), offsets, k, v, q


def check_append(cache, before, table, lengths, offsets, k, v, q, q_out, rotary, positions=None):
    starts, page, pages = offsets.tolist(), cache.page_size, cache.pages
    place = []
    for s, length in enumerate(lengths.tolist()):
        n = starts[s + 1] - starts[s]
        place += [(s, length - n + i) for i in range(n)]
    at = [p for _, p in place] if positions is None else positions
    f = turns_of(rotary) if rotary is not None else []
    inter, amp = (rotary.interleaved, rotary.amplitude) if rotary is not None else (0, 1.0)
    lo = starts[0]
    if q is not None:
        want, err = rotate64(q[lo:lo + len(place)], at, f, inter, amp)
        check(q_out[lo:lo + len(place)], want, err, "q")
    want, err = rotate64(k[lo:lo + len(place)], at, f, inter, amp)
    kw, ke, vw = before[0].double(), torch.zeros_like(before[0], dtype=torch.float64), before[1].clone()
    touched = torch.zeros(pages, page, dtype=torch.bool)
    for i, (s, p) in enumerate(place):
        if p < 0 or p >= table.shape[1] * page:
            continue
        pg = int(table[s, p // page])
        if 0 <= pg < pages:
            kw[pg, :, p % page], ke[pg, :, p % page], vw[pg, :, p % page] = want[i], err[i], v[lo + i]
            touched[pg, p % page] = True
    check(cache.k, kw, ke, "k")
    keep = ~touched.cuda()
    assert torch.equal(cache.k.transpose(1, 2)[keep], before[0].transpose(1, 2)[keep])
    assert torch.equal(cache.v, vw)


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("news,cached,heads,kv,d,page,dim,layout,pad", [
    ([1], [0], 1, 1, 8, 1, 8, "heads", 0), ([1, 1, 1], [7, 0, 15], 8, 2, 128, 16, 128, "heads", 0),
    ([5, 0, 1, 130, 2], [0, 9, 3, 40, 63], 6, 3, 80, 24, 80, "rows", 0), ([33, 1], [100, 0], 4, 4, 64, 7, 32, "rows", 8),
    ([1300, 1, 700], [0, 1, 64], 4, 2, 96, 64, 96, "heads", 0), ([9, 4], [2, 2], 3, 1, 256, 5, 250, "heads", 2),
    ([4, 4], [1, 0], 2, 2, 64, 16, 0, "heads", 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append(dtype, news, cached, heads, kv, d, page, dim, layout, pad, interleaved):
    g = gen(sum(news) * 7 + d)
    cache, table, lengths, offsets, k, v, q = append_case(g, dtype, news, cached, heads, kv, d, page, layout, pad)
    rotary = qnn.Rotary(dim, interleaved=interleaved, scaling="base" if dim > 2 else "none", factor=4.0) if dim else None
    before = cache.k.clone(), cache.v.clone()
    out = cache.append(k, v, table, lengths, offsets, rotary=rotary, q=q)
    check_append(cache, before, table, lengths, offsets, k, v, q, out, rotary)
    # once more in place, without queries, and by positions of one's own
    assert cache.append(k, v, table, lengths, offsets, rotary=rotary) is None
    check_append(cache, before, table, lengths, offsets, k, v, None, None, rotary)
    if rotary is not None:
        p = torch.randint(-5, 200000, (k.shape[0],), generator=g, device="cuda")
        q2 = q.clone()
        assert cache.append(k, v, table, lengths, offsets, rotary=rotary, q=q2, q_out=q2, positions=p) is q2
        check_append(cache, before, table, lengths, offsets, k, v, q, q2, rotary, p.tolist())


def test_append_without_offsets_is_as_many_for_each():
    g = gen(17)
    cache, table, lengths, offsets, k, v, q = append_case(g, BF, [3, 3, 3], [0, 20, 5], 4, 2, 64, 8)
    rotary = qnn.Rotary(64)
    a = cache.append(k, v, table, lengths, offsets, rotary=rotary, q=q)
    other = qnn.PagedCache(cache.k.clone(), cache.v.clone())
    other.k.zero_(), other.v.zero_()
    b = other.append(k, v, table, lengths, rotary=rotary, q=q)
    assert torch.equal(a, b)
    live = other.k.abs().sum((1, 3)) > 0
    assert int(live.sum()) == 9
    assert torch.equal(other.k.transpose(1, 2)[live], cache.k.transpose(1, 2)[live])


def test_places_outside_the_cache_are_not_written():
    g = gen(23)
    cache, table, lengths, offsets, k, v, q = append_case(g, BF, [6, 4, 5], [10, 0, 3], 2, 2, 64, 4, holes=[(0, 3), (2, 0)])
    table[1, 0] = cache.pages  # just outside
    lengths = lengths.clone()
    lengths[2] = 2  # three of its five tokens lie before the sequence
    before = cache.k.clone(), cache.v.clone()
    out = cache.append(k, v, table, lengths, offsets, rotary=qnn.Rotary(64), q=q)
    check_append(cache, before, table, lengths, offsets, k, v, q, out, qnn.Rotary(64))
    # sequences longer than the table
    lengths[0] = table.shape[1] * 4 + 3
    before = cache.k.clone(), cache.v.clone()
    out = cache.append(k, v, table, lengths, offsets, rotary=qnn.Rotary(64), q=q)
    check_append(cache, before, table, lengths, offsets, k, v, q, out, qnn.Rotary(64))


def test_rows_in_no_sequence_stay():
    g = gen(29)
    cache, table, lengths, offsets, k, v, q = append_case(g, F16, [2, 6, 3, 4], [3, 8, 1, 0], 4, 2, 64, 8)
    mid, ml = offsets[1:4].contiguous(), lengths[1:3].contiguous()  # tokens 2 .. 10 are sequences 1 and 2
    before = cache.k.clone(), cache.v.clone()
    q_out = torch.full_like(q, 7.0)
    cache.append(k, v, table[1:3].contiguous(), ml, mid, rotary=qnn.Rotary(64), q=q, q_out=q_out)
    assert bool((q_out[:2] == 7).all()) and bool((q_out[11:] == 7).all())
    check_append(cache, before, table[1:3], ml, mid, k, v, q, q_out, qnn.Rotary(64))


def test_append_of_nothing():
    g = gen(31)
    cache, table, lengths, offsets, k, v, q = append_case(g, BF, [1], [3], 2, 1, 64, 8)
    before = cache.k.clone()
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    cache.append(k[:0], v[:0], table, lengths, none, rotary=qnn.Rotary(64), q=q[:0])
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    cache.append(k[:0], v[:0], table[:0], empty, rotary=qnn.Rotary(64))
    assert torch.equal(cache.k, before)
