"""Refusals of the operators of a serving step that need no GPU: every check here is made before the
first CUDA call, so the addresses are made up."""
import ctypes

import pytest

from paper_2609_11744_b200 import kvc

INVALID, ALIGN, LARGE = kvc.KVC_ERR_INVALID_ARG, kvc.KVC_ERR_ALIGNMENT, kvc.KVC_ERR_TOO_LARGE
A = 0x10000


def layout(planes=2, hkv=2, d=64, e=2, layers=2):
    return kvc.kvc_layout_create_dense(A, layers, planes, 32, 16, hkv, d, e, 64)


def status(fn, lay, desc):
    return getattr(kvc.lib(), fn)(lay.handle if lay else None, ctypes.byref(desc) if desc is not None else None, 0)


def fill(cls, **kw):
    d = cls()
    for k, v in kw.items():
        assert hasattr(d, k), k
        setattr(d, k, v)
    return d


def map_desc(**kw):
    a = dict(context_lens=A, new_lens=A, free_blocks=A, block_tables=A, table_stride=8, max_blocks=8, n_requests=4, n_free=3,
             token_capacity=10, cu_tokens=A, positions=A, slots=A)
    a.update(kw)
    return fill(kvc.kvc_map_tokens_desc, **a)


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(cu_tokens=0)), (INVALID, dict(context_lens=0)), (INVALID, dict(new_lens=0)), (INVALID, dict(free_blocks=0)),
    (INVALID, dict(block_tables=0)), (INVALID, dict(positions=0)), (INVALID, dict(slots=0)), (INVALID, dict(table_stride=7)),
    (INVALID, dict(reserved=1)), (INVALID, dict(token_capacity=1 << 31)), (LARGE, dict(n_requests=kvc.KVC_MAP_MAX_REQUESTS + 1)),
    (ALIGN, dict(slots=A + 4)), (ALIGN, dict(context_lens=A + 2)), (ALIGN, dict(counts=A + 1))])
def test_map_tokens_refuses(want, kw):
    assert status("kvc_map_tokens", layout(), map_desc(**kw)) == want


def append_desc(**kw):
    a = dict(layer=1, dtype=0, q=A, k=A, v=A, q_out=A, q_token_stride=512, q_head_stride=64, k_token_stride=128, k_head_stride=64,
             v_token_stride=128, v_head_stride=64, out_token_stride=512, out_head_stride=64, slots=A, positions=A, cos_sin=A,
             cos_sin_stride=64, eps=1e-6, n_tokens=5, n_q_heads=8, rot_dim=64, max_positions=10)
    a.update(kw)
    return fill(kvc.kvc_append_desc, **a)


@pytest.mark.parametrize("want,kw", [
    (INVALID, dict(layer=2)), (INVALID, dict(dtype=2)), (INVALID, dict(k=0)), (INVALID, dict(v=0)), (INVALID, dict(q=0)),
    (INVALID, dict(q_out=0)), (INVALID, dict(slots=0)), (INVALID, dict(positions=0)), (INVALID, dict(cos_sin=0)),
    (INVALID, dict(cos_sin_stride=63)), (INVALID, dict(rot_dim=24)), (INVALID, dict(rot_dim=80)), (INVALID, dict(interleaved=2)),
    (INVALID, dict(eps=-1.0)), (INVALID, dict(eps=float("nan"))), (INVALID, dict(reserved=1)), (INVALID, dict(n_tokens=1 << 31)),
    (ALIGN, dict(q=A + 8)), (ALIGN, dict(q_out=A + 2)), (ALIGN, dict(k_token_stride=132)), (ALIGN, dict(out_head_stride=68)),
    (ALIGN, dict(q_weight=A + 4)), (ALIGN, dict(slots=A + 4)), (ALIGN, dict(positions=A + 2))])
def test_append_refuses(want, kw):
    assert status("kvc_append", layout(), append_desc(**kw)) == want


@pytest.mark.parametrize("lay", [dict(planes=1), dict(e=1), dict(e=4), dict(d=264), dict(d=12, hkv=4)])
def test_append_refuses_layouts(lay):
    assert status("kvc_append", layout(**lay), append_desc(rot_dim=0)) == INVALID


def attention_desc(**kw):
    a = dict(layer=0, dtype=1, q=A, out=A, q_token_stride=512, q_head_stride=64, out_token_stride=512, out_head_stride=64,
             cu_tokens=A, seq_lens=A, block_tables=A, table_stride=8, max_blocks=8, n_tokens=5, n_requests=3, n_q_heads=8,
             scale=0.125, workspace=A, workspace_bytes=1 << 40)
    a.update(kw)
    return fill(kvc.kvc_attention_desc, **a)


BAD_ATTENTION = [
    (INVALID, dict(layer=2)), (INVALID, dict(dtype=7)), (INVALID, dict(q=0)), (INVALID, dict(out=0)), (INVALID, dict(cu_tokens=0)),
    (INVALID, dict(seq_lens=0)), (INVALID, dict(block_tables=0)), (INVALID, dict(workspace=0)), (INVALID, dict(max_blocks=0)),
    (INVALID, dict(table_stride=7)), (INVALID, dict(n_q_heads=0)), (INVALID, dict(n_q_heads=7)), (INVALID, dict(scale=0.0)),
    (INVALID, dict(scale=-1.0)), (INVALID, dict(scale=float("nan"))), (INVALID, dict(scale=float("inf"))), (INVALID, dict(reserved=1)),
    (LARGE, dict(n_tokens=1 << 30)), (ALIGN, dict(q=A + 8)), (ALIGN, dict(out=A + 4)), (ALIGN, dict(workspace=A + 128)),
    (ALIGN, dict(q_head_stride=60)), (ALIGN, dict(out_token_stride=516)), (ALIGN, dict(lse=A + 2)), (ALIGN, dict(block_tables=A + 1))]


@pytest.mark.parametrize("want,kw", BAD_ATTENTION + [
    (INVALID, dict(n_groups=1)), (INVALID, dict(group_starts=A)), (INVALID, dict(prefix_lens=A)), (INVALID, dict(window=(1 << 30) + 1)), (INVALID, dict(sinks=1 << 31))])
def test_attention_refuses(want, kw):
    assert status("kvc_attention", layout(), attention_desc(**kw)) == want


@pytest.mark.parametrize("want,kw", BAD_ATTENTION + [
    (INVALID, dict(n_groups=0)), (INVALID, dict(n_groups=4)), (INVALID, dict(group_starts=0)), (INVALID, dict(prefix_lens=0)),
    (INVALID, dict(window=5)), (INVALID, dict(sinks=1))])
def test_attention_shared_refuses(want, kw):
    a = dict(n_groups=1, group_starts=A, prefix_lens=A)
    a.update(kw)
    assert status("kvc_attention_shared", layout(), attention_desc(**a)) == want


@pytest.mark.parametrize("lay", [dict(planes=1), dict(e=1), dict(d=80), dict(d=256), dict(d=32)])
def test_attention_refuses_layouts(lay):
    assert status("kvc_attention", layout(**lay), attention_desc()) == INVALID
    n = ctypes.c_uint64()
    assert kvc.lib().kvc_attention_workspace_bytes(layout(**lay).handle, 5, 3, 8, 0, ctypes.byref(n)) == INVALID


def test_nothing_to_do_is_no_error_and_needs_no_gpu():
    lay = layout()
    assert status("kvc_append", lay, append_desc(n_tokens=0)) == kvc.KVC_OK
    assert status("kvc_attention", lay, attention_desc(n_tokens=0)) == kvc.KVC_OK
    assert status("kvc_attention", lay, attention_desc(n_requests=0)) == kvc.KVC_OK
    for fn in ("kvc_map_tokens", "kvc_append", "kvc_attention", "kvc_attention_shared"):
        assert status(fn, None, None) == INVALID and status(fn, lay, None) == INVALID
    assert kvc.lib().kvc_attention_workspace_bytes(lay.handle, 1, 1, 8, 2, ctypes.byref(ctypes.c_uint64())) == INVALID
    assert kvc.lib().kvc_attention_workspace_bytes(lay.handle, 1, 1, 8, 0, None) == INVALID
    assert kvc.kvc_layout_launch_count(lay) == 0


def test_descriptor_sizes_match_the_header(tmp_path):
    """The ctypes mirrors have the sizes and last offsets that a C compiler gives the structs."""
    import os
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("needs gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ("kvc_map_tokens_desc", "kvc_append_desc", "kvc_attention_desc")
    lines = []
    for n in names:
        for f, _ in getattr(kvc, n)._fields_:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (n, f))
        lines.append('printf("%%zu\\n", sizeof(%s));' % n)
    src = tmp_path / "sizes.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"kvc.h\"\nint main(void) { %s return 0; }\n" % "".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "sizes")], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for n in names:
        cls = getattr(kvc, n)
        want += [getattr(cls, f).offset for f, _ in cls._fields_] + [ctypes.sizeof(cls)]
    assert got == want
