"""The widest rows of logits: kernels step through a row by up to 1024 elements, so its end has
to leave as many below 2^31; refused on the host before any CUDA call."""
import ctypes

import pytest

import paper_2608_06291_gb300 as P

FAKE = ctypes.c_void_p(0x1000)   # never dereferenced: validation fails first


@pytest.mark.parametrize("v", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 256, 2 ** 31 - 1023])
@pytest.mark.parametrize("dtype", [0, 1])
def test_wider_rows_are_refused(v, dtype):
    P.build()
    L = P.lib()
    assert L.bakron_token_logprobs(FAKE, dtype, 1, v, v, FAKE, 5, FAKE, FAKE, FAKE, FAKE, FAKE, None) == 1
    assert L.bakron_token_logprobs_backward(FAKE, dtype, 1, v, v, FAKE, FAKE, FAKE, None, None, FAKE, v, None) == 1


def test_the_widest_is_looked_at_further():
    """2^31 - 1024 columns fail for what else is wrong with a call, and with no rows they do not."""
    P.build()
    L, v = P.lib(), 2 ** 31 - 1024
    assert L.bakron_token_logprobs(FAKE, 1, 0, v, v, None, 0, None, FAKE, FAKE, None, None, None) == 0
    assert L.bakron_token_logprobs(FAKE, 1, 1, v, v - 1, None, 0, None, FAKE, FAKE, None, None, None) == 1
    assert L.bakron_token_logprobs_backward(FAKE, 1, 0, v, v, FAKE, FAKE, FAKE, None, None, FAKE, v, None) == 0
