"""The paged cache's Python binding on the CPU: options that the C structure has no room for."""
import pytest

from paper_2608_27922_gb300 import build as B


@pytest.mark.parametrize("option", ["window", "sinks", "block"])
@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32 + 5, 2 ** 40, -2 ** 31 - 1])
def test_options_of_more_than_32_bits_are_refused(option, value):
    """A window of 2^32 + 5 is not one of 5 positions."""
    from paper_2608_27922_gb300 import dkv
    try:
        dkv.lib()
    except RuntimeError:
        B.build()
    cache = object.__new__(dkv.PagedCache)
    cache.handle, cache._plans = None, {}
    options = dict(window=0, sinks=0, block=1)
    options[option] = value
    with pytest.raises(ValueError, match=option):
        cache._plan((1, 2, 1, None, options["window"], options["sinks"], options["block"], 1))
    cache._plan((1, 2, 1, None, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 1))
