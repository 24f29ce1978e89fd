"""Lanes of a wave that exchange values through LDS without a workgroup barrier:
`__builtin_amdgcn_wave_barrier` orders no memory, so a fence stands beside every
one of them.  The code that the compiler emits may be the same without it, which
is why this looks at the sources."""

from __future__ import annotations

import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2411_00284_amd", "csrc")
SOURCES = [p for p in sorted(glob.glob(os.path.join(CSRC, "*"))) if p.endswith((".hip", ".h"))]


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_a_fence_beside_every_wave_barrier(path):
    text = re.sub(r"//[^\n]*", "", open(path).read())
    barriers = len(re.findall(r"__builtin_amdgcn_wave_barrier\(\);", text))
    fenced = len(re.findall(r'__builtin_amdgcn_fence\(__ATOMIC_ACQ_REL, "wavefront"\);\s*__builtin_amdgcn_wave_barrier\(\);', text))
    assert barriers == fenced
