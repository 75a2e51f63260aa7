"""More host-side checks of the cache's C ABI (no GPU, nothing is launched)."""
import numpy as np
import pytest

from test_cache_abi import ARG, OK, attend, batch, cache, lib, query  # noqa: F401  (lib: a fixture)


@pytest.mark.parametrize("scale", [3.4e38, 2.4e38])
def test_softmax_scales_that_overflow_in_powers_of_two(lib, scale):  # noqa: F811
    """The kernels multiply scores by scale * log2(e): infinite, it would make a score of 0 a NaN."""
    assert np.isfinite(np.float32(scale))
    assert lib.ssba_cache_attend_workspace_size(cache(), batch(), query(softmax_scale=scale), 0, None) == ARG
    assert attend(lib, q=query(softmax_scale=scale)) == ARG
    assert lib.ssba_cache_attend_workspace_size(cache(), batch(), query(softmax_scale=2.3e38), 0, None) == OK
