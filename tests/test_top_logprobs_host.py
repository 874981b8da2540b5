"""Host side of top log-probabilities: struct layout, argument checks before any launch, workspace sizes."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2510_05485_amd as tb
from paper_2510_05485_amd import losses
from test_losses_host import HERE, ROOT, gradient, lib, logits, positions  # noqa: F401


def test_struct_size_matches_the_header(tmp_path):
    src = tmp_path / "size.c"
    src.write_text('#include <stdio.h>\n#include "tensorloss.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %d", '
                   'sizeof(tb_top_t), offsetof(tb_top_t, ids), offsetof(tb_top_t, logprobs), '
                   'offsetof(tb_top_t, id_bytes), offsetof(tb_top_t, K), TB_TOP_MOST); return 0; }\n')
    exe = tmp_path / "size"
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), "-include", "stddef.h", str(src), "-o", str(exe)])
    s = losses.tb_top_t
    assert [int(v) for v in subprocess.check_output([str(exe)], text=True).split()] == \
        [ctypes.sizeof(s), s.ids.offset, s.logprobs.offset, s.id_bytes.offset, s.K.offset, losses.TOP_MOST]


def top(**kw):
    q = losses.tb_top_t(ids=HERE, logprobs=HERE, id_bytes=8, K=4)
    for k, v in kw.items():
        setattr(q, k, v)
    return q


def test_workspace(lib):  # noqa: F811
    n = lib.tensorloss_top_workspace_bytes
    for bad in ((-1, 1, 50, 0, 1), (1 << 16, 1 << 15, 50, 0, 1), (1, 1, 0, 0, 1), (1, 1, 50, 3, 1), (1, 1, 50, -1, 1),
                (1, 1, 50, 0, 0), (1, 1, 50, 0, 51), (1, 1, 5000, 0, 1025)):
        assert n(*bad) == 0, bad
    assert n(1 << 10, 1 << 10, 64, 1, 5) == 0 and n(4096, 1, 32000, 1, 64) == 0
    for V, type_ in ((262144, 0), (1 << 20, 1), (2 ** 31 - 1, 2)):
        for rows, k in ((1, 1), (1, 1024), (3, 64), (100, 256)):
            b = n(rows, 1, V, type_, k)
            assert b == n(1, rows, V, type_, k)
            parts = min(512 // rows, V * (4 if type_ == 0 else 2) // 65536)
            assert b >= rows * parts * (8 * k + 16)      # (every part leaves K keys and its statistics)
        assert n(5000, 1, V, type_, 64) == 0              # (a workgroup for each row)


def test_arguments(lib):  # noqa: F811
    ref = ctypes.byref

    def rc(q, l=None, p=None, lp=HERE, workspace=None, bytes_=0):
        return lib.tensorloss_top_logprobs(ref(l or logits()), ref(p or positions()), ref(q) if q else None, lp, None, None,
                                           None, workspace, bytes_, None)
    assert rc(None) == 1
    for kw in (dict(ids=None), dict(ids=HERE + 4), dict(logprobs=None), dict(id_bytes=2), dict(K=0), dict(K=-1), dict(K=51)):
        assert rc(top(**kw)) == 1, kw
    wide = dict(B=1, T=1, V=5000)
    assert rc(top(K=1025), logits(**wide)) == 1
    assert rc(top(), p=positions(tokens=None)) == 1
    for kw in (dict(V=0), dict(type=3), dict(temperature=0.0), dict(data=None), dict(pos_stride=-1)):
        assert rc(top(), logits(**kw)) == 1, kw
    assert rc(top(ids=None, logprobs=None), logits(B=0, data=None), positions(tokens=None), None) == 0      # nothing to do
    long = logits(B=1, T=1, V=1 << 20, seq_stride=1 << 20, pos_stride=1 << 20)
    n = lib.tensorloss_top_workspace_bytes(1, 1, 1 << 20, 0, 4)
    assert n > 0
    assert rc(top(), long) == rc(top(), long, workspace=HERE + 16, bytes_=n) == rc(top(), long, workspace=HERE, bytes_=n - 1) == 2


def test_gradient_arguments(lib):  # noqa: F811
    ref = ctypes.byref

    def rc(q=None, g=None, state=HERE, d=HERE, l=None, p=None, d_lp=HERE):
        return lib.tensorloss_top_logprobs_grad(ref(l or logits()), ref(p or positions()), ref(q or top(logprobs=None)), state, d,
                                                d_lp, None, ref(g) if g else None, None)
    assert rc() == 1
    for kw in (dict(q=top(K=51)), dict(q=top(ids=None)), dict(q=top(id_bytes=3)), dict(state=None), dict(d=None),
               dict(p=positions(tokens=None)), dict(g=gradient(data=None)), dict(g=gradient(pos_stride=49)),
               dict(g=gradient(data=HERE << 20)), dict(g=gradient(data=(HERE << 20) + 4))):
        assert rc(**{"g": gradient(), **kw}) == 1, kw
    assert rc(g=gradient(), l=logits(B=0)) == 0


def test_python_refuses_what_is_not_on_a_gpu():
    with pytest.raises(tb.TensorBLEUError, match="GPU"):
        tb.top_logprobs(torch.zeros(2, 3, 5), 2)
