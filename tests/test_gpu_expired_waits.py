"""Device waits of the learner operators that run out: the kernels end, what depended on the wait is NaN and nothing is finite and
wrong, and the next call is right.

The bounds-checking build lets the waits of one kind in one block run out (HPL_DEBUG_EXPIRE=<waiter>,<block>,<n>: all but the first n
of the call's), whatever they wait for; the block's other waits, and those of other blocks on it, then reach their own limit.  Each group
runs in a process of its own, with that build.
"""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LOADS, PRODUCTS, RESULTS = 1, 2, 3


def _expire(waiter=0, block=0, after=0):
    os.environ["HPL_DEBUG_EXPIRE"] = f"{waiter},{block},{after}"


def _ortho(hpl, torch, u, dtype, steps):
    batch, rows, cols = u.shape
    ws = torch.empty(hpl.orthogonalize_workspace(batch, rows, cols), dtype=torch.uint8, device="cuda")
    out = torch.full((batch, rows, cols), 777.0, dtype=dtype, device="cuda")
    hpl.orthogonalize(hpl.OrthoArgs(src=u.data_ptr(), dst=out.data_ptr(), dst_dtype=hpl.HPL_BF16 if dtype == torch.bfloat16 else hpl.HPL_F32,
                                    batch=batch, rows=rows, cols=cols, steps=steps, workspace=ws.data_ptr(), workspace_bytes=ws.numel()),
                      torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return out


def _check_products(batch, rows, cols, blocks, waiters, counts):
    """An element is NaN or the one of an undisturbed call, bit for bit; from the first wait on, some are NaN."""
    import torch

    import paper_2002_05814_b200 as hpl
    u = torch.randn(batch, rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows))
    for dtype, steps in ((torch.float32, 1), (torch.bfloat16, 2)):
        _expire()
        right = _ortho(hpl, torch, u, dtype, steps)
        assert torch.isfinite(right).all()
        for waiter in waiters:
            for block in blocks:
                for after in counts:
                    _expire(waiter, block, after)
                    got = _ortho(hpl, torch, u, dtype, steps)
                    nan = torch.isnan(got)
                    what = f"{batch} x {rows} x {cols}, {dtype}, waiter {waiter} of block {block} after {after}"
                    assert (nan | (got == right)).all(), f"{what}: {(~nan & (got != right)).sum().item()} elements finite and wrong"
                    assert after or nan.any(), what
                    _expire()
                    assert torch.equal(_ortho(hpl, torch, u, dtype, steps), right), f"the call after {what}"


def products():
    """Tiles on a CTA and on a pair, by themselves (a pair's second CTA starts no products)."""
    _check_products(1, 300, 500, (0, 7), (LOADS, PRODUCTS, RESULTS), (0, 9, 40, 1500))
    _check_products(2, 2048, 2048, (0,), (LOADS, PRODUCTS, RESULTS), (0, 40, 9000))
    _check_products(2, 2048, 2048, (1,), (LOADS, RESULTS), (0, 40, 9000))


def shared_sums():
    """Sums over k that the CTAs of a cluster share: a part that gives up, whichever it is, makes the sum NaN."""
    _check_products(1, 333, 1000, (0, 1, 7, 30), (LOADS, PRODUCTS, RESULTS), (0, 1, 3, 300))
    _check_products(1, 1024, 4096, (0, 1, 2, 106), (LOADS, PRODUCTS, RESULTS), (0, 5, 700))


def small_matrices():
    """Everything in one launch, on a CTA and on a cluster."""
    _check_products(3, 64, 128, (0, 2), (RESULTS,), (0, 100, 256, 700, 1000))
    _check_products(1, 128, 2048, (0, 5), (RESULTS,), (0, 100, 256, 700, 1000))
    _check_products(2, 600, 50, (0, 2), (RESULTS,), (0, 100, 256, 700, 1000))


def _check_rows(rows, vocab, dtype, k, gradient, blocks, waiters, counts):
    """A row is right, or NaN as a whole; its alternatives are found either way.  From the first wait on, some are NaN."""
    import torch

    import paper_2002_05814_b200 as hpl
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn(rows, vocab, device="cuda", generator=gen).to(dtype)
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=gen)
    g, h = torch.randn(rows, device="cuda", generator=gen), torch.randn(rows, device="cuda", generator=gen)

    def call():
        out = {n: torch.full((rows, w), 777.0, device="cuda") for n, w in (("logprob", 1), ("entropy", 1), ("row_stats", 4), ("top_logprob", k))}
        index = torch.full((rows, k), 777, dtype=torch.int64, device="cuda")
        a = hpl.LogprobsArgs(logits=x.data_ptr(), dtype=hpl.HPL_BF16 if dtype == torch.bfloat16 else hpl.HPL_F32, rows=rows, vocab=vocab,
                             targets=t.data_ptr(), top_k=k, top_index=index.data_ptr() if k else 0)
        for name, v in out.items():
            if v.numel():
                setattr(a, name, v.data_ptr())
        if gradient:
            out["d_logits"] = torch.full((rows, vocab), 777.0, dtype=dtype, device="cuda")
            a.d_logprob, a.d_entropy, a.d_logits = g.data_ptr(), h.data_ptr(), out["d_logits"].data_ptr()
        (hpl.token_logprobs_with_grad if gradient else hpl.token_logprobs)(a, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        out["row_stats"] = out["row_stats"][:, 1:]               # the maximum may be of a part
        return out, index

    _expire()
    right, order = call()
    assert all(torch.isfinite(v).all() for v in right.values())
    for waiter in waiters:
        for block in blocks:
            for after in counts:
                _expire(waiter, block, after)
                got, index = call()
                what = f"{rows} x {vocab}, {dtype}, waiter {waiter} of block {block} after {after}"
                given_up = torch.isnan(got["logprob"][:, 0])
                for name, v in got.items():
                    assert torch.isnan(v[given_up]).all(), f"{what}: {name} of a row given up"
                    assert torch.equal(v[~given_up], right[name][~given_up]), f"{what}: {name}, finite and wrong"
                assert torch.equal(index, order), what
                assert after or given_up.any(), what
                _expire()
                again, index = call()
                assert all(torch.equal(v, right[name]) for name, v in again.items()) and torch.equal(index, order), f"the call after {what}"


def streamed_rows():
    """Many rows through a ring: those after one that was given up hold nothing of an earlier pass of the ring."""
    import torch
    for k in (0, 8):
        _check_rows(1500, 70_003, torch.bfloat16, k, False, (0, 300), (LOADS, RESULTS), (0, 5, 1000, 9000))
    _check_rows(1500, 33_001, torch.float32, 3, False, (5,), (LOADS, RESULTS), (0, 7, 2500))


def rows_on_chip():
    """A row in the shared memory of a CTA or a cluster, with and without its gradient."""
    import torch
    _check_rows(5, 3000, torch.float32, 7, True, (0, 5), (RESULTS,), (0, 100, 2000))
    _check_rows(2, 131_072, torch.bfloat16, 32, False, (0, 3, 15), (RESULTS,), (0, 200, 600))
    _check_rows(257, 50_021, torch.bfloat16, 4, True, (0, 101), (RESULTS,), (0, 300, 1000))


GROUPS = {f.__name__: f for f in (products, shared_sums, small_matrices, streamed_rows, rows_on_chip)}


@pytest.mark.parametrize("group", sorted(GROUPS))
def test_expired_waits(group):
    env = dict(os.environ, HPL_DEBUG_BOUNDS="1")
    build = subprocess.run([sys.executable, "-m", "paper_2002_05814_b200.build"], cwd=ROOT, env=env, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-2000:]
    r = subprocess.run([sys.executable, os.path.abspath(__file__), group], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]


if __name__ == "__main__":
    sys.path.insert(0, ROOT)
    GROUPS[sys.argv[1]]()
