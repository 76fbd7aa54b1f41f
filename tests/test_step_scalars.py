"""Without a GPU: spo_adamw_update refuses factor, rate and step counter that lie in what the step writes, and a counter in what it reads."""

import pytest

from paper_2509_13232_b200 import binding as B
from tests.test_step_host import EIGHT, adam, at, lib, no_gpu  # noqa: F401 - fixtures

N = 100                                     # elements of the tensor: w, g, m, v at 0 .. 3, scales at 4 and 5, copy at 6


@pytest.mark.parametrize("word", ["f", "rate", "count"])
@pytest.mark.parametrize("tensor,where", [(dict(), [at(0), at(0, 396), at(2), at(3, 200)]), (dict(w_dtype=1), [at(0), at(0, 196)]),
                                          (dict(copy=at(6)), [at(6), at(6, 196)]),
                                          (EIGHT, [at(0, 396), at(2), at(2, 96), at(3, 48), at(4), at(5)])])
def test_words_in_written_tensors_are_refused(lib, word, tensor, where):  # noqa: F811
    for p in where:
        assert adam(lib, tensor=tensor, **{word: p}) == B.ERR_INVALID_ARG


def test_the_counter_lies_in_nothing_that_is_read(lib):  # noqa: F811
    for p in (at(1), at(1, 396), at(1, -4)):
        assert adam(lib, count=p) == B.ERR_INVALID_ARG
    assert adam(lib, count=at(0, -4)) == B.ERR_INVALID_ARG          # its second word
    for other in ("f", "rate"):
        for p in (at(9), at(9, 4)):
            assert adam(lib, count=at(9), **{other: p}) == B.ERR_INVALID_ARG


def test_words_beside_tensors_are_taken(lib, no_gpu):  # noqa: F811
    for word in ("f", "rate", "count"):
        for tensor, p in ((dict(), at(0, 400)), (dict(w_dtype=1), at(0, 200)), (dict(), at(2, 400)), (EIGHT, at(2, 100)), (EIGHT, at(4, 4)),
                          (dict(copy=at(6)), at(6, 200)), (dict(), at(0, -8))):
            assert no_gpu(adam(lib, tensor=tensor, **{word: p}))
    assert no_gpu(adam(lib, f=at(1), rate=at(1, 4)))                # what is only read may lie in what is only read
    assert no_gpu(adam(lib, count=at(1, 400))) and no_gpu(adam(lib, count=at(9), f=at(9, 8), rate=at(9, -4)))
    assert no_gpu(adam(lib, tensor=dict(n=0), f=at(0), rate=at(2), count=at(3)))
