"""CPU-only checks of the host side of the operators around the quantized projections: constructors and refusals that
need no device."""
import pytest

from paper_2607_02461_b200 import binding as B
from paper_2607_02461_b200 import build as oqbuild


@pytest.fixture(scope="module", autouse=True)
def built():
    oqbuild.build()


def _code(fn, *a, **k):
    with pytest.raises(B.OqError) as e:
        fn(*a, **k)
    return e.value.code


def test_rope_constructor():
    assert B.oq_make_rope([44, 42, 42], [21, 30, 52]).dim == 128
    assert B.oq_make_rope([64], [4096], 500000.0, "halves").dim == 64
    assert _code(B.oq_make_rope, [44, 41], [4, 4]) == 2                  # odd
    assert _code(B.oq_make_rope, [24], [4], 10000.0, "halves") == 2      # half of it is no multiple of 8
    assert _code(B.oq_make_rope, [44, 42], [4]) == 1
    assert _code(B.oq_make_rope, [44, 0], [4, 4]) == 1
    assert _code(B.oq_make_rope, [44], [0]) == 1
    assert _code(B.oq_make_rope, [2] * 5, [4] * 5) == 2                  # axes
    assert _code(B.oq_make_rope, [128, 130], [4, 4]) == 2                # coordinates
    assert _code(B.oq_make_rope, [256], [2 ** 21]) == 2                  # table size
    assert _code(B.oq_make_rope, [64], [4], 0.0) == 1
    assert _code(B.oq_make_rope, [64], [4], float("nan")) == 1
    assert _code(B.oq_make_rope, [64], [4], 10000.0, "thirds") == 1
