"""Sizes that no launch holds are refused on the host, as arguments that do not fit are (include/eas_attention.h).  No
GPU: made-up addresses do, as every call here returns before any HIP call."""
import pytest

from paper_2609_31551_amd import attention as A
from test_attention_abi import BAD, UNSUPPORTED, append, attend, cache, prompt, rows, shape


def test_more_threads_than_a_launch_holds():
    """A grid's dimension holds less than 2^32 threads: 2^24 workgroups of 256, 2^23 of 512, 2^26 of 64."""
    # rows: 1,024 sequences of up to 2^20 rows, 16,385 spans of 64 tokens each
    assert rows(n=1024, most=1 << 20, rows=1 << 20) == UNSUPPORTED
    # append: 2^17 sequences of up to 8,192 tokens, 129 pages of 64 tokens each
    assert append(n=1 << 17, most=8192, rows=8192, cu=0x10000, max_pages=200) == UNSUPPORTED
    # attention over the cache: 2^20 sequences of 4 key heads and 5 runs
    assert attend(n=1 << 20, rows=1 << 20, most=5000, max_pages=100, ws_bytes=1 << 62) == UNSUPPORTED
    # and its join: 2 sequences of 2^21 queries and 28 heads, four a workgroup
    assert attend(most_q=1 << 21, ws_bytes=1 << 62) == UNSUPPORTED
    # prompts: 2^22 workgroups of 256 queries for each of two heads
    s = shape(heads=2, kv_heads=2, q=(256, 128), k=(256, 128), v=(256, 128), out=(256, 128))
    assert prompt(s, cu_q=(0, 1 << 30)) == UNSUPPORTED


@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, 3.4e38])
def test_scales_that_are_infinite_in_log2_units(scale):
    assert prompt(shape(scale=scale)) == BAD
    assert attend(s=shape(scale=scale)) == BAD


def test_the_largest_scales():
    """The shape passes: the next argument is refused."""
    for scale in (2.3e38, -2.3e38, 0.0):
        assert prompt(shape(scale=scale), cu_q=(0, 9), cu_k=(0, (1 << 30) + 1)) == UNSUPPORTED
        assert attend(cache(page_tokens=16), shape(scale=scale), max_pages=(1 << 26) + 1) == UNSUPPORTED
