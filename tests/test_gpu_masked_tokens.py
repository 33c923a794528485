"""The row's own token among the masked ones: its log probability is -inf, its gradient the formula's scale * g, every other masked logit's 0."""
import math

import pytest
import torch

import paper_2002_05814_b200 as hpl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2002_05814_b200 import build
    build.build()
    assert torch.cuda.is_available()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [2, 18, 700, 1500, 40_003])
@pytest.mark.parametrize("both", [True, False], ids=["with_grad", "grad"])
def test_a_masked_token_keeps_the_formulas_gradient(vocab, dtype, both):
    rows, scale = 6, 0.5
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn(rows, vocab, device="cuda", generator=gen).to(dtype)
    t = torch.tensor([0, vocab - 1, vocab // 2, 0, vocab - 1, 1], device="cuda")
    x[torch.arange(rows, device="cuda"), t] = -math.inf
    x[4, ::2] = -math.inf                                       # others beside it
    x[5] = -math.inf                                            # an empty row: no gradient at all
    x[4, 0 if t[4] else 1] = 1.0
    g = torch.tensor([1.0, -2.0, 0.0, 0.25, 8.0, 3.0], device="cuda")     # g * scale is exact in either type
    logprob, d = torch.empty(rows, device="cuda"), torch.full_like(x, 777.0)
    stats = torch.empty(rows, 4, device="cuda")
    a = hpl.LogprobsArgs(logits=x.data_ptr(), dtype=hpl.HPL_BF16 if dtype == torch.bfloat16 else hpl.HPL_F32, rows=rows, vocab=vocab,
                         targets=t.data_ptr(), logprob=logprob.data_ptr(), row_stats=stats.data_ptr(), d_logprob=g.data_ptr(),
                         d_logits=d.data_ptr(), scale=scale)
    stream = torch.cuda.current_stream().cuda_stream
    if both:
        hpl.token_logprobs_with_grad(a, stream)
    else:
        hpl.token_logprobs(a, stream)
        hpl.token_logprobs_grad(a, stream)
    torch.cuda.synchronize()
    assert (logprob == -math.inf).all()
    at = torch.arange(rows, device="cuda")
    want = g * scale
    want[5] = 0.0
    assert torch.equal(d[at, t].float(), want)                  # p is 0 there: nothing is taken off
    others = torch.isinf(x)
    others[at, t] = False
    assert (d[others] == 0).all()
    p = torch.softmax(x[:5].double() * scale, 1)                # and the rest: -scale g p
    rest = -scale * g[:5, None].double() * p
    rest[at[:5], t[:5]] = want[:5].double()
    tol = 2e-5 * rest.abs() + (2.0 ** -8 * rest.abs() if dtype == torch.bfloat16 else 0) + 1e-30
    assert ((d[:5].double() - rest).abs() <= tol).all()
