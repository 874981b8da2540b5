"""Which kernels of the losses the library holds: those that some call reaches, and no others (CPU: from the
library's own symbols).  The rules by which launches choose are written out again here."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2510_05485_amd as tb

TYPES = {"F32": 4, "BF16": 8, "F16": 8}                  # values of a chunk of 16 bytes
LANES = [(2, 3), (2, 4), (4, 3), (4, 4), (8, 3), (8, 4), (16, 3), (16, 4), (16, 5), (16, 6), (32, 4),
         (64, 3), (64, 4), (64, 5), (64, 6), (64, 7), (64, 8)]
SCORE, POLICY, GIVEN = 0, 1, 3


def up(a, b):
    return -(-a // b)


def sizes(per):
    """A size on either side of everything that a rule may compare with."""
    found = set(range(1, 40 * per))
    for unit in (16, 64, 256, 512):
        for n in range(0, 80 if unit == 512 else 40):
            for off in range(-2 * per, 2 * per + 1):
                found.add(unit * n * per + off)
    return sorted(v for v in found if v >= 1)


def lanes(V, per):
    if V < per:
        return None
    return next(((n, c) for n, c in LANES if up(V, per) <= n * c), None)


def in_registers(V, per, long):
    """(threads, chunks, LDS) of a workgroup that holds a row"""
    if V < 2 * per:
        return None
    need, half = up(V // per, 512), up(V // per, 256)
    if long and need > 32:
        return (512, 32, True) if need <= 46 else (512, 46, True) if need - 46 <= 18 else None
    if half <= 8:
        return 256, half, False
    return (512, need, False) if need <= 32 else None


def distilled(V, per, K):
    """(threads, chunks, entries, LDS)"""
    if V < 2 * per:
        return None
    for threads, entries in ([(16, 1)] if K <= 16 else []) + ([(16, 4), (64, 1)] if K <= 64 else [(64, 4)] if K <= 256 else [(64, 16)]):
        if up(V // per, threads) <= 8:
            return threads, up(V // per, threads), entries, False
    held = in_registers(V, per, True)
    if held is None:
        return None
    entries = 1 if K <= 512 else 2
    return held[0], held[1], entries * (2 if held[0] == 256 else 1), held[2]


def reached():
    found = set()
    for name, per in TYPES.items():
        for V in sizes(per):
            few = lanes(V, per)
            for op in (SCORE, POLICY, GIVEN):
                for entropy in (False, True):
                    if few:
                        found.add(("lanes_kernel", name, op, entropy, *few))
                    elif op != GIVEN and in_registers(V, per, op == POLICY):
                        found.add(("held_kernel", name, op, entropy, *in_registers(V, per, op == POLICY)))
            for K in (1, 16, 17, 64, 65, 256, 257, 512, 513, 1024):
                if distilled(V, per, K):
                    found.add(("distill_kernel", name, *distilled(V, per, K)))
    return found


@pytest.mark.skipif(shutil.which("nm") is None, reason="no nm")
def test_every_kernel_is_reached():
    if not os.path.exists(tb.LIB_PATH):
        from paper_2510_05485_amd import build
        build.build(verbose=False)
    names = subprocess.check_output(["nm", "-C", tb.LIB_PATH], text=True)
    held = set()
    for kernel, args in re.findall(r"__device_stub__(lanes_kernel|held_kernel|distill_kernel)<tb::loss::([^>]*)>", names):
        held.add((kernel, *(v if v in TYPES else v == "true" if v in ("true", "false") else int(v) for v in args.split(", "))))
    assert held
    want = reached()
    assert not held - want, (len(held - want), sorted(held - want, key=str)[:12])
    assert not want - held, (len(want - held), sorted(want - held, key=str)[:12])
