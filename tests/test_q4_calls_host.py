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
