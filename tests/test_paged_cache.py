"""PagedCache's refusals of caches that it cannot use, without a GPU."""
import pytest

from test_attention_boundary import BF, I32, new  # noqa: F401  (a fixture)
from paper_1908_11263_gb300 import qnn


def batch(new):  # noqa: F811
    return new(3, 4, dtype=I32), new(3, dtype=I32)


def test_a_cache_without_heads_is_refused(new):  # noqa: F811
    cache = qnn.PagedCache(new(9, 0, 16, 64), new(9, 0, 16, 64))
    with pytest.raises(ValueError, match="heads"):
        cache.attend(new(3, 8, 64), *batch(new))
