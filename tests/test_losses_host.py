"""Host side of the losses' C ABI: symbols, argument checks before any launch, workspace sizes."""
import ctypes
import os
import re

import pytest

import paper_2510_05485_amd as tb
from paper_2510_05485_amd import losses

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "tensorloss.h")
HERE = 4096            # stands for a device address; nothing is launched


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(tb.LIB_PATH):
        from paper_2510_05485_amd import build
        build.build(verbose=False)
    return losses._library()


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(tensorloss_\w+)\s*\(", text)))
    assert names == sorted(losses.EXPORTS)
    for name in names:
        assert hasattr(lib, name)


def test_struct_sizes_match_the_header(tmp_path):
    """The ctypes structures have the layout that a C compiler gives the header's."""
    import subprocess
    names = ["tb_logits_t", "tb_positions_t", "tb_gradient_t", "tb_policy_t", "tb_preference_t", "tb_teacher_t"]
    lines = []
    for n in names:
        lines.append(f'printf("%zu", sizeof({n}));')
        for field, _ in getattr(losses, n)._fields_:
            lines.append(f'printf(" %zu", offsetof({n}, {field}));')
        lines.append('printf("\\n");')
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "tensorloss.h"\nint main(void) {' + "".join(lines) + "return 0;}\n")
    exe = tmp_path / "sizes"
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    for n, line in zip(names, subprocess.check_output([str(exe)], text=True).splitlines()):
        s = getattr(losses, n)
        assert [int(v) for v in line.split()] == [ctypes.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_], n


def test_workspace(lib):
    assert losses.workspace_bytes(-1, 4) == 0 and losses.workspace_bytes(4, -1) == 0
    assert losses.workspace_bytes(1 << 16, 1 << 15) == 0           # positions beyond 32 bits
    for B, T in ((0, 0), (1, 1), (7, 13), (4096, 512), (100000, 1)):
        n = losses.workspace_bytes(B, T)
        assert n >= 16 * B * T + 32 * B
        assert n >= losses.workspace_bytes(max(B - 1, 0), T)


def logits(B=4, T=3, V=50, **kw):
    l = losses.tb_logits_t(data=HERE << 20, seq_stride=T * V, pos_stride=V, B=B, T=T, V=V, type=0, temperature=1.0)
    for k, v in kw.items():
        setattr(l, k, v)
    return l


def positions(**kw):
    p = losses.tb_positions_t(tokens=HERE, token_stride=3, token_bytes=8)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def gradient(**kw):
    g = losses.tb_gradient_t(data=HERE << 24, seq_stride=150, pos_stride=50, scale=1.0)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def test_logprobs_arguments(lib):
    ref = ctypes.byref

    def rc(l, p, out=HERE):
        return lib.tensorloss_token_logprobs(ref(l) if l else None, ref(p) if p else None, out, None, None, None, None)
    assert rc(None, positions()) == rc(logits(), None) == 1
    for kw in (dict(V=0), dict(B=-1), dict(T=-1), dict(type=3), dict(type=-1), dict(temperature=0.0),
               dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-45),
               dict(data=None), dict(data=(HERE << 20) + 2), dict(seq_stride=-1), dict(pos_stride=-1),
               dict(seq_stride=1 << 62), dict(B=1 << 16, T=1 << 16)):
        assert rc(logits(**kw), positions()) == 1, kw
    for kw in (dict(tokens=None), dict(tokens=HERE + 4), dict(token_bytes=2), dict(token_stride=-1)):
        assert rc(logits(), positions(**kw)) == 1, kw
    assert rc(logits(), positions(), None) == 1
    assert rc(logits(B=0, data=None), positions(tokens=None), None) == 0        # nothing to do
    assert rc(logits(T=0, data=None), positions(tokens=None), None) == 0


def test_gradient_arguments(lib):
    ref = ctypes.byref

    def rc(g, l=None):
        return lib.tensorloss_token_logprobs_grad(ref(l or logits()), ref(positions()), None, None, None, 3, 1, None,
                                                  ref(g) if g else None, None)
    assert rc(None) == 1
    # a null row_state is refused last: what is listed here is refused before
    for kw in (dict(data=None), dict(data=(HERE << 24) + 1), dict(pos_stride=49), dict(seq_stride=149),
               dict(seq_stride=0), dict(pos_stride=0), dict(seq_stride=50, pos_stride=50),
               dict(data=(HERE << 20) + 4), dict(data=(HERE << 20) - 4),
               dict(data=HERE << 20, seq_stride=200)):
        assert rc(gradient(**kw)) == 1, kw
    assert rc(gradient(), logits(B=0)) == 0


def test_loss_arguments(lib):
    ref = ctypes.byref
    n = losses.workspace_bytes(4, 3)

    def policy(bytes_=n, workspace=HERE, terms=HERE, lp=HERE, l=None, **kw):
        p = losses.tb_policy_t(old_logprobs=HERE, ref_logprobs=HERE, advantages=HERE, clip_low=0.2, clip_high=0.2)
        for k, v in kw.items():
            setattr(p, k, v)
        return lib.tensorloss_policy(ref(l or logits()), ref(positions()), ref(p), None, terms, lp, None, None, None,
                                     None, workspace, bytes_, None)
    for kw in (dict(terms=None), dict(lp=None), dict(old_logprobs=None), dict(advantages=None), dict(average=3),
               dict(average=-1), dict(clip_low=-0.1), dict(clip_high=float("nan")), dict(kl_coef=-1.0),
               dict(kl_coef=0.1, ref_logprobs=None), dict(entropy_coef=float("nan"))):
        assert policy(**kw) == 1, kw
    assert policy(workspace=None) == policy(workspace=HERE + 16) == policy(bytes_=n - 512) == 2

    def preference(l=None, terms=HERE, **kw):
        p = losses.tb_preference_t(ref_logprobs=HERE, kind=0, beta=0.1)
        for k, v in kw.items():
            setattr(p, k, v)
        return lib.tensorloss_preference(ref(l or logits()), ref(positions()), ref(p), None, terms, HERE, HERE, None,
                                         None, None, None, 0, None)
    for kw in (dict(terms=None), dict(ref_logprobs=None), dict(kind=3), dict(beta=0.0), dict(beta=float("inf")),
               dict(label_smoothing=0.6), dict(label_smoothing=-0.1), dict(kind=1, label_smoothing=0.1),
               dict(l=logits(B=3))):
        assert preference(**kw) == 1, kw
    assert preference() == 2

    def distill(rows=HERE, **kw):
        q = losses.tb_teacher_t(ids=HERE, logits=HERE, id_bytes=8, type=0, K=4)
        for k, v in kw.items():
            setattr(q, k, v)
        return lib.tensorloss_distill(ref(logits()), ref(positions(tokens=None)), ref(q), None, HERE, rows, None, None,
                                      None, None, 0, None)
    for kw in (dict(rows=None), dict(ids=None), dict(logits=None), dict(id_bytes=2), dict(type=3), dict(K=0),
               dict(K=1025), dict(average=3), dict(ids=HERE + 4), dict(logits=HERE + 2)):
        assert distill(**kw) == 1, kw
    assert distill() == 2


def test_python_refuses_what_is_not_on_a_gpu():
    import torch
    x, tokens, v = torch.zeros(2, 3, 5), torch.zeros(2, 3, dtype=torch.int64), torch.zeros(2, 3)
    for f in (lambda: tb.token_logprobs(x, tokens), lambda: tb.policy_loss(x, tokens, v, v),
              lambda: tb.preference_loss_grad(x, tokens, v),
              lambda: tb.distillation_loss(x, tokens.unsqueeze(-1), v.unsqueeze(-1))):
        with pytest.raises(tb.TensorBLEUError, match="GPU"):
            f()
