"""What rounding leaves of an orthogonalised matrix whose roundings do not average out, after few steps and many, against 64 bits.

Tolerances, relative to the result's norm.  A product of plane pairs is off by at most 2^-22 (the pairs) and 2^-20 (8 truncated
additions of an accumulator onto a sum that matters, 2^-23 each): 1.2e-6, always towards zero.  What becomes of that was taken
from 64-bit chains with every product made smaller by 1e-6, over the matrices below: up to 5e-6 after 1 to 8 steps, 1.9e-5 after
16 and 7.6e-5 after 64.  Five times that, e = 3e-5, 1.2e-4, 4.6e-4, is allowed.  A 16-bit result is such a value, rounded once: the
distance to the nearest 16-bit value changes by no more than the value does, so a result may be as far off as the exact
one's own rounding, and 2 e of the norm.
"""

import pytest
import torch

import paper_2002_05814_b200 as hpl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2002_05814_b200 import build
    build.build()
    assert torch.cuda.is_available()


def exact(u, steps):
    x = u.double()
    x = x if x.shape[0] <= x.shape[1] else x.T
    x = x / (x.norm() + 1e-7)
    for _ in range(steps):
        a = x @ x.T
        x = 3.4445 * x + (-4.7750 * a + 2.0315 * a @ a) @ x
    return x if u.shape[0] <= u.shape[1] else x.T


def ortho(u, dtype, steps):
    rows, cols = u.shape
    ws = torch.empty(hpl.orthogonalize_workspace(1, rows, cols), dtype=torch.uint8, device="cuda")
    out = torch.full((rows, cols), 777.0, dtype=dtype, device="cuda")
    hpl.orthogonalize(hpl.OrthoArgs(src=u.data_ptr(), dst=out.data_ptr(), dst_dtype=hpl.HPL_BF16 if dtype == torch.bfloat16 else hpl.HPL_F32,
                                    batch=1, rows=rows, cols=cols, steps=steps, workspace=ws.data_ptr(), workspace_bytes=ws.numel()),
                      torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return out.double()


def matrix(kind, rows, cols):
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    u = torch.zeros(rows, cols, device="cuda")
    if kind == "gauss":
        u = torch.randn(rows, cols, device="cuda", generator=gen)
    elif kind == "one row":                           # what a single token leaves of an embedding's gradient
        u[rows // 3] = torch.randn(cols, device="cuda", generator=gen)
    elif kind == "few rows":
        u[::max(1, rows // 20)] = torch.randn(len(range(0, rows, max(1, rows // 20))), cols, device="cuda", generator=gen)
    elif kind == "one entry":
        u[rows // 2, cols - 1] = -3.0
    elif kind == "equal":
        u.fill_(0.3)
    elif kind == "blocks":
        u[:rows // 2, :cols // 2] = 1.0
        u[rows // 2:, cols // 2:] = 0.5
    else:
        u.fill_diagonal_(1.0)
    return u


def check(kind, rows, cols, steps):
    u = matrix(kind, rows, cols)
    want = exact(u, steps)
    norm = want.norm().item()
    e = (3e-5 if steps <= 8 else 1.2e-4 if steps <= 16 else 4.6e-4) * norm
    off = (ortho(u, torch.float32, steps) - want).norm().item()
    assert off <= e, f"fp32, {steps} steps: {off / norm}"
    off, rounding = (ortho(u, torch.bfloat16, steps) - want).norm().item(), (want.bfloat16().double() - want).norm().item()
    assert off <= rounding + 2 * e, f"bf16, {steps} steps: {off / norm}, {rounding / norm} of it the result's own rounding"


KINDS = ["gauss", "one row", "few rows", "one entry", "equal", "blocks", "diagonal"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("steps", [1, 2, 3, 5, 8, 16, 64])
def test_number_of_steps_above_a_side_of_256(kind, steps):
    check(kind, 300, 500, steps)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(257, 300), (512, 512), (700, 260), (1024, 1500), (100, 500), (300, 64), (1100, 129)])
def test_matrices_whose_roundings_do_not_average_out(kind, rows, cols):
    check(kind, rows, cols, 5)
