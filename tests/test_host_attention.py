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


def _attention_code(**fields):
    """Status of oq_attention for 4 queries and 6 keys, 4 heads on 2 of 64, contiguous but for `fields`.  (The buffers are not
    memory: a call that is not refused for its arguments ends at the device's status word, as there is no device.)"""
    import torch
    if torch.cuda.is_available():
        pytest.skip("made-up buffers are for hosts without a device")
    at = dict(ldq_token=256, ldq_head=64, ldk_token=128, ldk_head=64, ldv_token=128, ldv_head=64, ldo_token=256, ldo_head=64,
              total_q=4, total_k=6, n_heads=4, n_kv_heads=2)
    at.update(fields)
    args = B._ATTENTION_ARGS.pack(4096, 8192, 12288, at["ldq_token"], at["ldq_head"], at["ldk_token"], at["ldk_head"], at["ldv_token"],
                                  at["ldv_head"], 16384, at["ldo_token"], at["ldo_head"], 0, 0, 0, 1, at["total_q"], at["total_k"],
                                  at["n_heads"], at["n_kv_heads"], 64, -1, -1, 0, 0.0)
    return B.lib().oq_attention(args, None, 0, None)


@pytest.mark.parametrize("field", ["ldq_token", "ldk_token", "ldv_token", "ldo_token", "ldo_head"])
@pytest.mark.parametrize("stride", [0, 8, 56, -64])
def test_rows_that_lie_over_each_other_are_refused(field, stride):
    """A token stride of 0, rows that overlap, outputs that overwrite each other: code 1, before anything touches a device."""
    assert _attention_code(**{field: stride}) == 1


@pytest.mark.parametrize("field", ["ldq_head", "ldk_head", "ldv_head"])
@pytest.mark.parametrize("stride", [8, 56, -64])
def test_heads_that_overlap_in_part_are_refused(field, stride):
    assert _attention_code(**{field: stride}) == 1


def test_host_tensors_are_refused():
    """A pointer to host memory never reaches a kernel."""
    import torch
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    assert _code(B.oq_attention, x, x, x) == 1
    assert _code(B.oq_qk_norm_rope, x, x) == 1
    a, b = torch.zeros(1, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 16, 8, dtype=torch.bfloat16)
    start, seg = torch.tensor([0, 3], dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    assert _code(B.oq_adapter_add, x[:, 0], a, b, torch.ones(1), start, seg, torch.zeros(3, 16, dtype=torch.bfloat16)) == 1


def _qk_code(x=4096, y=8192, ld_token=256, ld_head=64, ldy_token=256, ldy_head=64, tokens=3, heads=4, types=(0, 0)):
    """Status of oq_qk_norm_rope for queries of 64 on made-up buffers."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("made-up buffers are for hosts without a device")
    side = B._QK_SIDE.pack(x, ld_token, ld_head, heads, 0, y, ldy_token, ldy_head)
    return B.lib().oq_qk_norm_rope(side, None, tokens, 64, None, None, 0, 1, 1e-6, types[0], types[1], None)


def test_norm_outputs_that_lie_over_each_other_are_refused():
    for stride in (0, 8, 56, -64):
        assert _qk_code(ldy_token=stride) == 1 and _qk_code(ldy_head=stride) == 1
    assert _qk_code(y=4096, ldy_token=512) == 1 and _qk_code(y=4096, ldy_head=128) == 1      # X with other strides
    assert _qk_code(y=4096, types=(0, 1)) == 1                                               # and another type
    for sound in (dict(), dict(ldy_token=0, tokens=1), dict(ldy_head=0, heads=1), dict(ld_token=0), dict(ld_head=0), dict(y=4096)):
        assert _qk_code(**sound) == 4                                                        # as far as the device


def test_more_tokens_than_a_launch_can_walk_over_are_refused():
    assert _qk_code(tokens=2 ** 31 - 1) == 2 and _qk_code(tokens=2 ** 31 - 2 ** 16) == 2
    assert _qk_code(tokens=2 ** 30) == 4                                                     # as far as the device
