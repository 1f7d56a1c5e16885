"""The embedding's gradient: runs of equal tokens around the ends of chunks of eight sorted positions, and the order of a sum, which is one for given shapes
and tokens."""
import pytest
import torch

from paper_2012_15469_amd import ops
from test_gpu_embedding import DT, check_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("each", [1, 6, 7, 8, 9, 10, 15, 16, 17, 23, 24, 25])
def test_runs_around_the_ends_of_chunks(each):
    """Every token as often: runs that end at, before and behind each border of eight sorted positions; small integers, sums exactly."""
    vocab = 1 + 1025 // each
    tokens = torch.arange(vocab, device="cuda").repeat_interleave(each)
    assert tokens.numel() > 1024          # (more than one launch takes)
    for dtype, width in ((torch.float32, 40), (torch.bfloat16, 13)):
        dy = torch.randint(-8, 9, (tokens.numel(), width), device="cuda").to(dtype)
        for order in (torch.arange(tokens.numel(), device="cuda"), torch.randperm(tokens.numel(), device="cuda")):
            check_backward(dy[order], tokens[order], vocab + 1, exactly=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,width", [(40, 3, 100), (512, 7, 33), (512, 4, 4096), (3000, 11, 64), (20000, 50001, 48), (60000, 5, 40), (60000, 300, 1000)])
def test_one_order_whatever_runs_beside(rows, vocab, width, dtype):
    """The same bits again, also with workgroups of other calls among them, in a workspace of ones, and where the values of other tokens' rows differ."""
    gen = torch.Generator(device="cuda"); gen.manual_seed(rows)
    dy, tokens = torch.randn(rows, width, generator=gen, device="cuda").to(DT[dtype]), torch.randint(vocab, (rows,), generator=gen, device="cuda")
    want = ops.embedding_backward(dy, tokens, vocab)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [ops.embedding_backward(dy, tokens, vocab, stream=s) for _ in range(5) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    ws = torch.full((1 << 28,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(ops.embedding_backward(dy, tokens, vocab, workspace=ws), want)
    other = torch.where((tokens == 1)[:, None], dy, -dy)
    assert torch.equal(ops.embedding_backward(other, tokens, vocab)[1], want[1])
