"""Beam selection over rows in which most logits are equal: masked vocabularies, one value everywhere, values next to one another."""
import pytest
import torch

import paper_2504_05598_b200 as dl
from test_gpu_branching import check_beam

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("batch,beams,vocab,k", [(1, 1, 300001, 5), (2, 3, 40000, 8), (40, 2, 33000, 3), (1, 2, 9000, 64)])
def test_few_allowed_tokens(batch, beams, vocab, k, dtype):
    """Fewer than k, k and a few more tokens above -inf, at the front, at the end and in every chunk of a slice."""
    g = torch.Generator().manual_seed(k)
    base = torch.randn(batch, beams, vocab, generator=g).to(dtype)
    scores = -torch.rand(batch, beams, generator=g)
    for n in (1, k - 1, k, 3 * k):
        for where in ("front", "end", "anywhere"):
            logits = torch.full_like(base, -INF)
            for b in range(batch):
                for r in range(beams):
                    at = torch.arange(n) if where == "front" else vocab - 1 - torch.arange(n) if where == "end" else torch.randperm(vocab, generator=g)[:n]
                    logits[b, r, at] = base[b, r, at]
            check_beam(logits, scores, k)


@pytest.mark.parametrize("value", [0.0, -0.0, 1.0, -1.0, 2.0 ** -149, -2.0 ** -149, 3.0e38, -3.4028234663852886e38])
def test_values_at_and_next_to_the_bar(value):
    """One value everywhere but for a few tokens late in the row that lie one step of fp32 above or below it."""
    vocab = 70000
    row = torch.full((vocab,), value)
    above, below = torch.nextafter(row[:1], torch.tensor([INF])), torch.nextafter(row[:1], torch.tensor([-INF]))
    up, down = row.clone(), row.clone()
    up[[8191, 8192, 30000, 69999]] = above
    down[[0, 1, 5, 9000]] = below if abs(float(below)) < INF else row[:1]
    logits = torch.stack([up, down, row])[None]
    for k in (3, 20):
        check_beam(logits, torch.tensor([[-1.0, -1.25, -8.0]]), k)


def test_masked_rows_cost_little_more():
    """16 x 8 rows of 128256 with 10 allowed tokens: less than three times what rows of different logits take (a visit to every masked
    logit made it four times)."""
    x = torch.randn(16, 8, 128256, device="cuda")
    masked = torch.full_like(x, -INF)
    masked[:, :, 100::12000] = x[:, :, 100::12000]
    scores = -torch.rand(16, 8, device="cuda")
    outs = [torch.zeros(16, 16, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)]

    def ms(logits):
        best = INF
        for _ in range(8):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(20):
                dl.beam_select(logits, scores, *outs)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    assert ms(masked) < 3 * ms(x)


@pytest.mark.parametrize("batch,beams,vocab,k,dtype", [(4, 4, 128257, 8, torch.float32), (4, 4, 128257, 8, torch.bfloat16), (4, 4, 50257, 8, torch.float16),
                                                       (12, 8, 50257, 16, torch.float32), (12, 8, 50257, 16, torch.float16)])
def test_rows_of_odd_length_at_size(batch, beams, vocab, k, dtype):
    """Rows that start anywhere between 16-byte boundaries, in one launch and in two, slices of several chunks."""
    g = torch.Generator().manual_seed(vocab + k)
    logits = (2.5 * torch.randn(batch, beams, vocab, generator=g)).to(dtype)
    check_beam(logits, -10 * torch.rand(batch, beams, generator=g), k, torch.rand(batch, beams, generator=g) < 0.1, 2)
