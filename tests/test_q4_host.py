"""Refusals of the calls on pools held in 4 bits and of positions with several axes that need no GPU: every check
here is made before the first CUDA call, so the addresses are made up."""
import ctypes

import pytest

from paper_2609_11744_b200 import kvc
from test_step_host import A, ALIGN, BAD_ATTENTION, INVALID, LARGE, append_desc, attention_desc, fill, layout, status


def q4_layout(d=64, hkv=2, block=16, planes=2, e=1, row=None, layers=2):
    return kvc.kvc_layout_create_dense(A, layers, planes, 32, block, hkv, row or kvc.KVC_Q4_ROW_BYTES(d), e, 4 * block)


def axes_desc(token=None, pairs=(0, 1, 2), **kw):
    d = kvc.kvc_append_axes_desc()
    d.token = append_desc(**(token or {}))
    d.axis_stride, d.n_axes = 5, 3
    for i in range(kvc.KVC_MAX_PAIRS):
        d.pair_axis[i] = pairs[i % len(pairs)]
    for k, v in kw.items():
        assert hasattr(d, k), k
        setattr(d, k, v)
    return d


BAD_APPEND = [
    (INVALID, dict(layer=2)), (INVALID, dict(dtype=2)), (INVALID, dict(k=0)), (INVALID, dict(v=0)), (INVALID, dict(q=0)),
    (INVALID, dict(q_out=0)), (INVALID, dict(slots=0)), (INVALID, dict(positions=0)), (INVALID, dict(cos_sin=0)),
    (INVALID, dict(cos_sin_stride=63)), (INVALID, dict(rot_dim=24)), (INVALID, dict(rot_dim=80)), (INVALID, dict(interleaved=2)),
    (INVALID, dict(eps=-1.0)), (INVALID, dict(eps=float("nan"))), (INVALID, dict(reserved=1)), (INVALID, dict(n_tokens=1 << 31)),
    (ALIGN, dict(q=A + 8)), (ALIGN, dict(q_out=A + 2)), (ALIGN, dict(k_token_stride=132)), (ALIGN, dict(out_head_stride=68)),
    (ALIGN, dict(q_weight=A + 4)), (ALIGN, dict(slots=A + 4)), (ALIGN, dict(positions=A + 2))]
BAD_AXES = [dict(n_axes=0), dict(n_axes=kvc.KVC_MAX_AXES + 1), dict(axis_stride=4), dict(axis_stride=1 << 61), dict(reserved=1),
            dict(pairs=(0, 1, 3)), dict(pairs=(0,) * 31 + (255,)), dict(n_axes=2)]


@pytest.mark.parametrize("fn,lay", [("kvc_append_axes", layout), ("kvc_append_q4", q4_layout)])
def test_appends_refuse(fn, lay):
    for want, kw in BAD_APPEND:
        assert status(fn, lay(), axes_desc(kw)) == want, kw
    for kw in BAD_AXES:
        assert status(fn, lay(), axes_desc(**kw)) == INVALID, kw
    assert status(fn, None, axes_desc()) == INVALID and status(fn, lay(), None) == INVALID
    assert status(fn, lay(), axes_desc(dict(n_tokens=0))) == kvc.KVC_OK
    # entries behind the pairs of a head are not read, nor is the stride of one axis
    d = axes_desc(dict(n_tokens=0), pairs=(0,), n_axes=1, axis_stride=0)
    d.pair_axis[32] = 77
    assert status(fn, lay(), d) == kvc.KVC_OK


@pytest.mark.parametrize("kw", [dict(planes=1), dict(e=2, row=64), dict(row=64), dict(row=128), dict(row=79), dict(row=160)])
def test_other_layouts_are_refused(kw):
    lay = q4_layout(**kw)
    assert status("kvc_append_q4", lay, axes_desc(dict(rot_dim=0))) == INVALID
    assert status("kvc_read_q4", lay, read_desc()) == INVALID
    assert status("kvc_attention_q4", lay, attention_desc()) == INVALID
    n = ctypes.c_uint64()
    assert kvc.lib().kvc_attention_q4_workspace_bytes(lay.handle, 5, 3, 8, 0, ctypes.byref(n)) == INVALID


def test_the_calls_on_16_bit_pools_refuse_a_pool_in_4_bits():
    lay = q4_layout()
    assert status("kvc_append", lay, append_desc(rot_dim=0)) == INVALID
    assert status("kvc_append_axes", lay, axes_desc(dict(rot_dim=0))) == INVALID
    assert status("kvc_attention", lay, attention_desc()) == INVALID


def test_rows_of_a_head_that_do_not_end_on_16_bytes():
    lay = q4_layout(d=64, hkv=2, block=3)       # 120 bytes a head and block; the slab has 240
    n = ctypes.c_uint64()
    assert status("kvc_append_q4", lay, axes_desc(dict(rot_dim=0))) == ALIGN
    assert status("kvc_read_q4", lay, read_desc()) == ALIGN
    assert status("kvc_attention_q4", lay, attention_desc()) == ALIGN
    assert kvc.lib().kvc_attention_q4_workspace_bytes(lay.handle, 5, 3, 8, 0, ctypes.byref(n)) == ALIGN
    with pytest.raises(kvc.KvcError):           # no slab either
        q4_layout(d=64, hkv=1, block=3)


def read_desc(**kw):
    a = dict(layer=1, dtype=0, k_out=A, v_out=A, k_token_stride=128, k_head_stride=64, v_token_stride=128, v_head_stride=64, slots=A, n_tokens=5)
    a.update(kw)
    return fill(kvc.kvc_read_q4_desc, **a)


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(layer=2)), (INVALID, dict(dtype=2)), (INVALID, dict(slots=0)), (INVALID, dict(reserved=1)), (INVALID, dict(n_tokens=1 << 31)),
    (ALIGN, dict(k_out=A + 8)), (ALIGN, dict(v_out=A + 2)), (ALIGN, dict(k_token_stride=132)), (ALIGN, dict(v_head_stride=60)), (ALIGN, dict(slots=A + 4))])
def test_read_refuses(want, kw):
    assert status("kvc_read_q4", q4_layout(), read_desc(**kw)) == want


def test_nothing_to_read_is_no_error():
    assert status("kvc_read_q4", q4_layout(), read_desc(n_tokens=0)) == kvc.KVC_OK
    assert status("kvc_read_q4", q4_layout(), read_desc(k_out=0, v_out=0)) == kvc.KVC_OK
    assert status("kvc_read_q4", None, read_desc()) == INVALID and status("kvc_read_q4", q4_layout(), None) == INVALID
    assert status("kvc_attention_q4", q4_layout(), attention_desc(n_tokens=0)) == kvc.KVC_OK


@pytest.mark.parametrize("want,kw", BAD_ATTENTION + [
    (INVALID, dict(n_groups=1)), (INVALID, dict(group_starts=A)), (INVALID, dict(prefix_lens=A)), (INVALID, dict(window=(1 << 30) + 1)), (INVALID, dict(sinks=1 << 31)), (INVALID, dict(scale=2e18))])
def test_attention_refuses(want, kw):
    assert status("kvc_attention_q4", q4_layout(), attention_desc(**kw)) == want


@pytest.mark.parametrize("want,kw", BAD_ATTENTION + [
    (INVALID, dict(n_groups=0)), (INVALID, dict(n_groups=4)), (INVALID, dict(group_starts=0)), (INVALID, dict(prefix_lens=0)),
    (INVALID, dict(window=5)), (INVALID, dict(sinks=1))])
def test_attention_shared_refuses(want, kw):
    a = dict(n_groups=1, group_starts=A, prefix_lens=A)
    a.update(kw)
    assert status("kvc_attention_q4_shared", q4_layout(), attention_desc(**a)) == want


def test_pair_axes():
    assert kvc.kvc_pair_axes([16, 24, 24]) == bytes([0] * 16 + [1] * 24 + [2] * 24)
    assert kvc.kvc_pair_axes([3, 3, 3], in_turns=True) == bytes([0, 1, 2] * 3)
    assert kvc.kvc_pair_axes([4, 2, 2], in_turns=True) == bytes([0, 1, 2, 0, 1, 2, 0, 0])
    assert kvc.kvc_pair_axes([0, 2]) == bytes([1, 1]) and kvc.kvc_pair_axes([]) == b""


def test_layout_of_a_pool_in_4_bits():
    for d, row in ((64, 40), (128, 80)):
        lay = kvc.kvc_layout_create_q4(A, 3, 9, 16, 4, d, 32)
        assert kvc.KVC_Q4_ROW_BYTES(d) == row and kvc.kvc_layout_slab_bytes(lay) == 16 * 4 * row
        assert kvc.kvc_layout_bytes_per_token(lay) == 3 * 2 * 4 * row
    with pytest.raises(ValueError):
        kvc.kvc_layout_create_q4(A, 3, 9, 16, 4, 96, 32)


def test_descriptor_sizes_match_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("needs gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ("kvc_append_axes_desc", "kvc_read_q4_desc")
    lines = []
    for n in names:
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (n, f) for f, _ in getattr(kvc, n)._fields_]
        lines.append('printf("%%zu\\n", sizeof(%s));' % n)
    lines.append('printf("%u\\n%u\\n%u\\n%u\\n", KVC_MAX_AXES, KVC_MAX_PAIRS, KVC_Q4_GROUP, KVC_Q4_ROW_BYTES(128));')
    src = tmp_path / "sizes.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"kvc.h\"\nint main(void) { %s return 0; }\n" % "".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "sizes")], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for n in names:
        cls = getattr(kvc, n)
        want += [getattr(cls, f).offset for f, _ in cls._fields_] + [ctypes.sizeof(cls)]
    assert got == want + [kvc.KVC_MAX_AXES, kvc.KVC_MAX_PAIRS, kvc.KVC_Q4_GROUP, 80]
