"""What the calls of a step take, without a GPU."""
import inspect

import pytest

from paper_2609_11744_b200 import kvc


@pytest.mark.parametrize("name", ["kvc_append", "kvc_append_axes", "kvc_append_q4", "kvc_read_q4", "kvc_attention", "kvc_attention_shared",
                                  "kvc_attention_q4", "kvc_attention_q4_shared", "kvc_map_tokens"])
def test_no_argument_is_private(name):
    fn = getattr(kvc, name)
    have = inspect.signature(fn).parameters
    assert not [p for p in have if p.startswith("_")]
    with pytest.raises(TypeError):               # one argument too many reaches nothing
        fn(*[None] * (len(have) + 1))


@pytest.mark.parametrize("pair_axis", [32, 3.0, True])
@pytest.mark.parametrize("name", ["kvc_append_axes", "kvc_append_q4"])
def test_a_number_is_no_pair_axis(name, pair_axis):
    """bytes(32) is 32 zeros: a number in the place of pair_axis would have every pair turn by the first axis."""
    import torch
    lay = kvc.kvc_layout_create_dense(0x10000, 1, 2, 4, 16, 2, 64, 2, 16) if name == "kvc_append_axes" else kvc.kvc_layout_create_q4(0x10000, 1, 4, 16, 2, 64, 16)
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="pair_axis"):
        getattr(kvc, name)(lay, 0, None, k, k, None, torch.zeros(3, dtype=torch.int64), torch.zeros(3, 3, dtype=torch.int32),
                           torch.zeros(9, 64), pair_axis)
