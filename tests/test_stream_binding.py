"""The binding of streamed generation: whole numbers that do not fit the library's 32 bits are
refused (ctypes would cut them: a window of 2^32 + 5 tokens to 5)."""
import pytest

from paper_2607_06631_amd import binding as B

BIG = (2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63, -2 ** 31 - 1, -2 ** 32)


@pytest.mark.parametrize("big", BIG)
@pytest.mark.parametrize("name", ("block", "window", "sinks", "flags"))
def test_attention(big, name):
    kw = dict(block=1, window=7, sinks=2, flags=0)
    kw[name] = big
    for call, n in ((B.dif_attention_paged, 7), (B.dif_attention_window, 5)):
        with pytest.raises(ValueError, match="2\\^31"):
            call(*[None] * n, **kw)


@pytest.mark.parametrize("big", BIG)
@pytest.mark.parametrize("name", ("norm_dim", "axes"))
def test_append(big, name):
    with pytest.raises(ValueError, match="2\\^31"):
        B.dif_cache_append(*[None] * 7, **{name: big})
