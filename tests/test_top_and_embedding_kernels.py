"""Which kernels of top log-probabilities and of embeddings the library holds: those that some call reaches, and no
others (CPU: from the library's own symbols).  The rules by which launches choose are written out again here."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2510_05485_amd as tb

TYPES = {"F32": 4, "BF16": 8, "F16": 8}                  # values of a chunk of 16 bytes
TOP_MOST = 1024


def up(a, b):
    return -(-a // b)


def sizes(per):
    """A size on either side of everything that a rule may compare with."""
    found = set(range(1, 40 * per))
    for unit in (16, 64, 256, 512):
        for n in range(0, 120 if unit >= 256 else 40):
            found.update(unit * n * per + off for off in range(-2 * per, 2 * per + 1, 1 if unit < 256 else 3))
    found.update(range(100_000, 2_000_000, 4099))
    return sorted(v for v in found if v >= 1)


def parts_of(rows, V, per):
    size = V * (16 // per)
    return 1 if size < 131072 else max(1, min(512 // rows, size // 65536))


def top(rows, V, K, per):
    """(kernel, its numbers): what a call of so many rows runs first"""
    chunks = up(V, per)
    if K <= 8 and V >= per:
        for lanes in (2, 4, 8, 16, 32):
            if chunks <= lanes * 4:
                return "best_kernel", lanes, 4, 8 if per == 4 else 2 if K <= 2 else 5 if K <= 5 else 8
    for lanes in (2, 4, 8, 16, 32, 64):
        if chunks <= lanes and (K * lanes <= 2048 or V < per):
            return "short_kernel", lanes
    parts = parts_of(rows, V, per)
    whole = (V // parts + (64 if parts > 1 else 0)) // per
    tried = []
    if parts == 1:
        if K <= 128 or (K <= 256 and whole <= 256):
            tried += [(64, n, 2) for n in (2, 4, 6, 8)]
        tried += [(256, n, 2) for n in (4, 6, 8)]
        if K < 512 and rows >= 512:
            tried += [(256, n, 2) for n in range(10, 28, 2)]
    if K >= 512 or rows < 512:
        tried += [(512, 6, 4)] + [(512, n, 2) for n in (8, 10, 12, 14, 16)]
    for threads, n, step in tried:
        if up(whole, threads) <= n:
            return "top_kernel", threads, n, step, False
    tiles = up(whole, 24 * 256)
    each = lambda: up(whole // tiles + 64 // per + 2, 256)
    if each() > 24:
        tiles += 1
    return "top_kernel", 256, next(n for n in (14, 16, 18, 20, 22, 24) if each() <= n), 2, True


def reached_by_top():
    found = set()
    for name, per in TYPES.items():
        few = set()
        for V in sizes(per):
            for rows in (1, 2, 7, 100, 300, 511, 512):
                for K in (1, 2, 3, 5, 6, 8, 9, 16, 32, 33, 64, 65, 128, 129, 256, 257, 511, 512, TOP_MOST):
                    if K <= V:
                        few.add(top(rows, V, K, per))
                        if parts_of(rows, V, per) > 1:
                            few.add(("join_kernel",))
            chunks = up(V, per)
            few.add(("top_gradient_kernel", next((t for t, most in ((8, 32), (64, 512), (256, 2048)) if chunks <= most), 512)))
        found |= {(kernel, name, entropy, *rest) for kernel, *rest in few for entropy in (False, True)}
    return found


def reached_by_embeddings():
    found = set()
    for name, per in TYPES.items():
        widths = sorted({n * per + off for n in list(range(0, 40)) + [64, 256, 512, 513, 2000] for off in (-1, 0, 1)} - {-1, 0})
        for out in {name, "F32"}:
            for D in widths:
                chunks = up(D, per)
                team = (8, False) if D < per else (next((n for n in (2, 8, 32) if chunks <= n), 64), True)
                found |= {("sum_kernel", name, out, *team), ("join_kernel", name, out, *team)}
            found.add(("part_sums_kernel", out))
            # few positions, up to 65536, more of up to and beyond two million rows: tokens, prepared, parted, ranges of a part
            found |= {("sort_kernel", out, n) for n in range(4)}
        for D in widths:
            chunks = up(D, per)
            lanes = next((n for n, most in ((2, 2), (8, 8), (16, 16), (32, 32), (64, 512)) if chunks <= most), 256)
            found.add(("lookup_kernel", name, 8, False) if D < per else ("lookup_kernel", name, lanes, True))
    return found


def value(text):
    text = re.sub(r"tb::\w+::|\(anonymous namespace\)::|\(\w+(?: \w+)*\)", "", text).strip()
    return {"true": True, "false": False}.get(text, text if text in TYPES else None) if not text.isdigit() else int(text)


@pytest.mark.skipif(shutil.which("nm") is None, reason="no nm")
@pytest.mark.parametrize("space,kernels,reached", [
    ("loss", "best|short|top|join|top_gradient", reached_by_top),
    ("embed", "lookup|sum|join|sort|part_sums", reached_by_embeddings)])
def test_every_kernel_is_reached(space, kernels, reached):
    if not os.path.exists(tb.LIB_PATH):
        from paper_2510_05485_amd import build
        build.build(verbose=False)
    names = subprocess.check_output(["nm", "-C", tb.LIB_PATH], text=True)
    held = set()
    for kernel, args in re.findall(rf"tb::{space}::\(anonymous namespace\)::__device_stub__((?:{kernels})_kernel)<([^>]*)>", names):
        held.add((kernel, *(value(v) for v in args.split(", "))))
    assert held and not any(None in k for k in held)
    want = reached()
    assert not held - want, (len(held - want), sorted(held - want, key=str)[:12])
    assert not want - held, (len(want - held), sorted(want - held, key=str)[:12])
