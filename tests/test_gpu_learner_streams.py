"""Calls of the learner operators at work at the same time, on streams of their own: each gives what it gives alone, bit for bit.  Their
blocks take tensor memory and clusters, and share SMs."""
import pytest
import torch

import paper_2002_05814_b200 as hpl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2002_05814_b200 import build
    build.build()
    assert torch.cuda.is_available()


class Ortho:
    def __init__(self, batch, rows, cols, dtype, seed):
        self.u = torch.randn(batch, rows, cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))
        self.ws = torch.empty(hpl.orthogonalize_workspace(batch, rows, cols), dtype=torch.uint8, device="cuda")
        self.out = [torch.empty(batch, rows, cols, dtype=dtype, device="cuda")]
        self.args = hpl.OrthoArgs(src=self.u.data_ptr(), dst=self.out[0].data_ptr(), dst_dtype=hpl.HPL_BF16 if dtype == torch.bfloat16 else hpl.HPL_F32,
                                  batch=batch, rows=rows, cols=cols, workspace=self.ws.data_ptr(), workspace_bytes=self.ws.numel())

    def __call__(self, stream):
        hpl.orthogonalize(self.args, stream)


class Rows:
    def __init__(self, rows, vocab, dtype, k, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.x = torch.randn(rows, vocab, device="cuda", generator=gen).to(dtype)
        self.t = torch.randint(0, vocab, (rows,), device="cuda", generator=gen)
        self.g = torch.randn(rows, device="cuda", generator=gen)
        self.out = [torch.empty(rows, device="cuda"), torch.empty_like(self.x), torch.empty(rows, k, dtype=torch.int64, device="cuda")]
        self.args = hpl.LogprobsArgs(logits=self.x.data_ptr(), dtype=hpl.HPL_BF16 if dtype == torch.bfloat16 else hpl.HPL_F32, rows=rows, vocab=vocab,
                                     targets=self.t.data_ptr(), top_k=k, logprob=self.out[0].data_ptr(), d_logprob=self.g.data_ptr(),
                                     d_logits=self.out[1].data_ptr(), top_index=self.out[2].data_ptr() if k else 0)

    def __call__(self, stream):
        hpl.token_logprobs_with_grad(self.args, stream)


def _together(calls, passes=20):
    alone = []
    for c in calls:
        c(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        alone.append([v.clone() for v in c.out])
        for v in c.out:
            v.zero_()
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(passes):
        for c, s in zip(calls, streams):
            c(s.cuda_stream)
    torch.cuda.synchronize()
    for c, want in zip(calls, alone):
        assert all(torch.equal(a, b) for a, b in zip(c.out, want))


def test_small_matrices_on_clusters_and_on_single_blocks():
    _together([Ortho(4, 64, 600, torch.float32, 1), Ortho(2, 128, 2048, torch.bfloat16, 2), Ortho(3, 1000, 40, torch.float32, 3),
               Ortho(200, 32, 48, torch.float32, 4), Ortho(8, 128, 256, torch.bfloat16, 5)])


def test_small_matrices_and_tiles():
    _together([Ortho(4, 64, 600, torch.float32, 1), Ortho(1, 333, 1000, torch.float32, 2), Ortho(2, 2048, 2048, torch.bfloat16, 3),
               Ortho(24, 64, 128, torch.float32, 4)])


def test_rows_beside_matrices():
    _together([Rows(8, 131_072, torch.bfloat16, 8, 1), Rows(300, 50_021, torch.float32, 0, 2), Ortho(1, 128, 2048, torch.float32, 3),
               Ortho(1, 700, 260, torch.bfloat16, 4), Rows(4096, 18, torch.float32, 4, 5)])
