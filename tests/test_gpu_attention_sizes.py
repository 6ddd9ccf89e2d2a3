"""PagedCache.attend where a call has more sequences, or a sequence more rows, than its work lists take in one step."""
import pytest
import torch

from attention_util import gen
from test_gpu_attention import paged, run

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("seqs,d,most", [(4500, 64, 1), (4097, 128, 37), (8200, 64, 37)])
def test_thousands_of_sequences(seqs, d, most):
    """More than 4096 sequences: several groups of 32 a bin; some have no new tokens, some see nothing."""
    g = gen(seqs + d + most)
    news = torch.randint(0, most + 1, (seqs,), generator=g, device="cuda").tolist()
    more = torch.randint(0, 70, (seqs,), generator=g, device="cuda").tolist()
    lengths = [n + m - (i % 7 == 0) * min(n + m, n // 2 + 5) for i, (n, m) in enumerate(zip(news, more))]
    news[-1] = most
    run(*paged(g, BF, news, lengths, 2, 1, d, 16, nan=False))


@pytest.mark.parametrize("d,dtype", [(64, BF), (128, F16)])
@pytest.mark.parametrize("kw", [{}, dict(window=700), dict(causal=False)])
def test_more_row_tiles_than_a_warp_has_lanes(d, dtype, kw):
    """Sequences of 33 and more tiles of 256 rows, between short ones."""
    news = [3, 8449, 300, 4225 * 2 + 1, 1]
    lengths = [40, 8449, 900, 4225 * 2 + 77, 5000]
    run(*paged(gen(d), dtype, news, lengths, 1, 1, d, 32), **kw)
