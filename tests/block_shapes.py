"""Shapes of the block operators' tests that together launch every kernel that is
built: test_gpu_block_forms.py runs them against 64 bits, test_block_forms_host.py
looks that none is missing."""

from __future__ import annotations

import itertools

# (block type, stream type, weights' type)
NORM_TYPES = [("bf16", "bf16", "bf16"), ("bf16", "bf16", "f32"), ("bf16", "f32", "bf16"), ("bf16", "f32", "f32"),
              ("f16", "f16", "f16"), ("f16", "f16", "f32"), ("f16", "f32", "f16"), ("f16", "f32", "f32"), ("f32", "f32", "f32")]
# One width for each form: a row on 64 lanes once or twice, 256 threads, 512, 1024 once or twice.
NORM_HIDDEN = [250, 1000, 1991, 4096, 8192, 16001]
NORM_TOKENS = 45
NORMS = list(itertools.product(NORM_TYPES, NORM_HIDDEN))

# Products out [m, n] summed over k, for each form of a tile, and with parts of k that are joined; a product is that of
# the forward, of dx or of dweight.
PRODUCTS_16 = [(1976, 4372, 328), (3063, 1288, 328), (9336, 136, 264), (88, 8504, 520), (200, 300, 1200), (64, 256, 8192)]
PRODUCTS_32 = [(5896, 272, 200), (70, 100, 300), (61, 250, 2100)]
PRODUCTS = [(d, kind, s) for d in ("bf16", "f16", "f32") for kind in ("forward", "dx", "dweight")
            for s in (PRODUCTS_32 if d == "f32" else PRODUCTS_16)]
# Rows of x, with k off the grid.
ROWS = [(d, m, 1001, 1237) for d in ("bf16", "f16", "f32") for m in (1, 2, 3, 4)]

# tokens, vocabulary, top: rows that threads hold whole, few tokens, a micro-batch of long rows, and of longer ones.
DISTILLS = [(d, *s) for d in ("bf16", "f16", "f32")
            for s in ((300, 2003, 33), (9, 20011, 100), (300, 20011 if d != "f32" else 12001, 64), (300, 40009 if d != "f32" else 20011, 64))]


def linear_sizes(kind, shape):
    """(m, n, k) of the linear layer whose product this is."""
    m, n, k = shape
    return shape if kind == "forward" else (m, k, n) if kind == "dx" else (k, m, n)
