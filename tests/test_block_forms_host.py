"""Every kernel that is built is launched by a shape of block_shapes.py, which
test_gpu_block_forms.py runs against 64 bits (on the host, against a stub of
the HIP runtime)."""

from __future__ import annotations

from block_shapes import DISTILLS, NORM_TOKENS, NORMS, PRODUCTS, ROWS, linear_sizes
from test_block_launch_forms import BF16, F16, F32, at, call, distill, linear, linear_grad, norm, norm_grad
from test_block_launch_forms import launches  # noqa: F401

CODE = {"bf16": BF16, "f16": F16, "f32": F32}


def test_every_kernel_has_a_shape(launches):  # noqa: F811
    calls = []
    for types, hidden in NORMS:
        b, s, w = (CODE[t] for t in types)
        calls += [norm(NORM_TOKENS, hidden, b, s, w), norm_grad(NORM_TOKENS, hidden, b, s, w)]
    for d, kind, shape in PRODUCTS:
        m, n, k = linear_sizes(kind, shape)
        if kind == "forward":
            calls.append(linear(m, n, k, CODE[d]))
        else:
            calls.append(linear_grad(m, n, k, CODE[d], 2, **({"dx": at(5)} if kind == "dx" else {"dweight": at(6)}), dbias=at(7)))
    calls += [linear(m, n, k, CODE[d]) for d, m, n, k in ROWS]
    for d, tokens, vocab, _ in DISTILLS:
        calls += [distill(tokens, vocab, CODE[d]), distill(tokens, vocab, CODE[d], grad=True),
                  distill(tokens, vocab, CODE[d], grad=True, backward=True)]
    _, mangled, built = launches(calls)
    reached = {n for names in mangled for n in names}
    assert not built - reached, sorted(built - reached)
