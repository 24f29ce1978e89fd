"""Shapes of the step's operators' tests that together launch every kernel that is
built: the test_gpu_step_*.py run them against 64 bits, test_step_launch_forms.py
looks that none is missing."""

from __future__ import annotations

# m, n, k of a gated feed-forward for each form of its forward product: one of 256 x 256 with a rest, 128 x 128 in two
# steps and in four, 64 x 128, with parts of k.
FORWARD_16 = [(4101, 2052, 520), (9336, 66, 264), (1976, 2186, 328), (88, 4252, 520), (200, 300, 1200), (64, 256, 8192)]
FORWARD_32 = [(5896, 136, 200), (70, 100, 300), (61, 250, 2100)]
FORWARD = [(d, s) for d in ("bf16", "f16", "f32") for s in (FORWARD_32 if d == "f32" else FORWARD_16)]

# Rows that go without tiles; with k cut among the waves of a workgroup.
ROWS = [(d, m, *s) for d in ("bf16", "f16", "f32") for m in (1, 2, 3, 4) for s in ((501, 1237), (101, 5003))]

# m, n, k for each form of the gradient's products.
GRADIENT_16 = [(3063, 200, 1288), (1976, 164, 4372), (9336, 136, 136), (264, 4700, 136), (88, 264, 8504), (200, 600, 300), (64, 4096, 256),
               (4096, 60, 500), (8192, 32, 256), (328, 1000, 4372)]
GRADIENT_32 = [(5896, 100, 272), (200, 260, 4204), (1000, 470, 1204), (70, 150, 100), (61, 1050, 250), (2100, 61, 125), (200, 3000, 272)]
GRADIENT = [(d, s) for d in ("bf16", "f16", "f32") for s in (GRADIENT_32 if d == "f32" else GRADIENT_16)]

# tokens, vocabulary: rows that a wave holds whole, that 256 threads do, few tokens, a micro-batch of long rows, and of longer ones.
POLICIES = [(d, *s) for d in ("bf16", "f16", "f32")
            for s in ((300, 2003), (300, 6001 if d != "f32" else 3501), (9, 20011), (300, 20011 if d != "f32" else 12001), (300, 40009 if d != "f32" else 20011))]
