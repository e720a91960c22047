"""The sizes of tile_cases.py are planned as it says, by the library's own host code: a change of the rules would otherwise leave whole tiles without a test."""
import os
import shutil
import subprocess

import pytest

from tile_cases import GRAD, HEAD, LOSS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _plans(tmp_path, cases, *flags):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    exe = str(tmp_path / "tile_plans")
    subprocess.run([hipcc, "-x", "hip", "--offload-arch=gfx950", "-O0", "-std=c++17", "-w", *flags, "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2512_00719_amd", "csrc"), os.path.join(ROOT, "tests", "tile_plans.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe, *(str(n) for c in cases for n in c)], check=True, capture_output=True, text=True).stdout
    return [tuple(int(x) for x in line.split()) for line in out.splitlines()]


def test_head(tmp_path):
    got = _plans(tmp_path, [(T, V, int(T > 512)) for T, V in HEAD], "-DHEAD")
    assert got == list(HEAD.values())


def test_loss_and_gradient(tmp_path):
    got = _plans(tmp_path, [(T, V, 0) for T, V in LOSS] + list(GRAD))
    assert got == list(LOSS.values()) + [(rows, splits, *g, *dh, *dw) for rows, splits, g, dh, dw in GRAD.values()]


def test_the_cases_have_what_they_are_for():
    plans = list(HEAD.values()) + list(LOSS.values()) + [p for _, _, *ps in GRAD.values() for p in ps]
    assert all(kind == 256 for kind, *_ in plans) and sum(whole > 0 for _, whole, *_ in plans) >= len(plans) - 1
    assert any(whole > wgs for _, whole, wgs, _ in HEAD.values()) and any(parts > 0 for *_, parts in HEAD.values())
    assert any(splits > 1 for _, splits, *_ in GRAD.values()) and any(rows < V for (_, V, _), (rows, *_) in GRAD.items())
    assert any(dw[1] > dw[2] for *_, dw in GRAD.values())
