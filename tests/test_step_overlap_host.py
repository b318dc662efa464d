"""kvc_map_tokens refuses outputs that share memory with an input or another output, before any CUDA call."""
import pytest

from paper_2609_11744_b200 import kvc
from test_step_host import INVALID, fill, layout, status

R, T, F, WIDE, STRIDE = 5, 11, 7, 6, 9
SIZES = dict(context_lens=4 * R, new_lens=4 * R, free_blocks=4 * F, block_tables=4 * ((R - 1) * STRIDE + WIDE), cu_tokens=4 * (R + 1),
             positions=4 * T, slots=8 * T, token_request=4 * T, total_lens=4 * R, counts=12)
OUT = ("block_tables", "cu_tokens", "positions", "slots", "token_request", "total_lens", "counts")
AT = {k: 0x100000 + 0x1000 * i for i, k in enumerate(SIZES)}


def call(**at):
    d = fill(kvc.kvc_map_tokens_desc, table_stride=STRIDE, max_blocks=WIDE, n_requests=R, n_free=F, token_capacity=T, **dict(AT, **at))
    return status("kvc_map_tokens", layout(), d)


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("other", list(SIZES))
def test_an_output_over_another_array_is_refused(out, other):
    if out == other:
        return
    step = 8 if "slots" in (out, other) else 4
    assert call(**{out: AT[other]}) == INVALID
    last = (SIZES[other] - 1) // step * step   # the last element of the other array
    assert call(**{out: AT[other] + last}) == INVALID
    assert call(**{other: AT[out] + (SIZES[out] - 1) // step * step}) == INVALID


@pytest.mark.parametrize("row", range(R))
def test_any_row_of_the_table_counts(row):
    at = AT["block_tables"] + 4 * STRIDE * row
    assert call(counts=at) == INVALID and call(counts=at + 4 * (WIDE - 1)) == INVALID
    assert call(cu_tokens=at - 4 * R) == INVALID   # its last element is the row's first
    if row:
        assert call(positions=at - 4 * (STRIDE - WIDE)) == INVALID   # begins between two rows


def test_arrays_side_by_side_and_shared_inputs_are_not_refused():
    """Past the refusals the call goes to the device, of which there may be none here."""
    at, places = 0x100000, {}
    for k in sorted(SIZES, key=lambda k: k != "slots"):   # the 8-byte array first
        places[k] = at
        at += SIZES[k]
    gap = AT["block_tables"] + 4 * (2 * STRIDE + WIDE)   # between two rows of the table
    for a in (places, dict(places, new_lens=places["context_lens"]), dict(places, total_lens=0, counts=0, token_request=0), dict(counts=gap)):
        try:
            import torch
            if torch.cuda.is_available():   # made-up addresses go no further than a machine without a GPU
                pytest.skip("needs a machine without a GPU")
        except ImportError:
            pass
        assert call(**a) not in (INVALID, kvc.KVC_ERR_ALIGNMENT)
