"""examples/train_workers.py on the GPU with the server's orthogonalised step and an
entropy bonus: it runs, and its gradient is the one torch works out in 64 bits."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import train_workers
    finally:
        sys.path.pop(0)
    return train_workers


def test_runs(example):
    said = []
    out = example.train(3, 3, log=said.append, orthogonal=True, bonus=0.01)
    assert len(said) == 2 and all(torch.isfinite(torch.tensor(v)) for v in out)


def test_gradient(example):
    import paper_1905_12948_amd as gmc
    g = torch.Generator(device="cuda:0").manual_seed(2)
    R, T, V, bonus = 3, 4, 37, 0.05
    logits = 2 * torch.randn(R, T, V, device="cuda:0", generator=g)
    tokens = torch.randint(0, V, (R, T), device="cuda:0", generator=g)
    scores = gmc.token_scores(logits, tokens)
    noise = torch.randn(2, R, T, device="cuda:0", generator=g)
    old, ref, A = scores[0] - 0.05 * noise[0], scores[0] + 0.2 * noise[1], torch.randn(R, T, device="cuda:0", generator=g)
    got = example.policy_gradient(logits, tokens, old, A, ref, scores, bonus)
    x = logits.double().requires_grad_()
    table = torch.log_softmax(x, -1)
    logp = table.gather(-1, tokens[..., None])[..., 0]
    ratio = (logp - old.double()).exp()
    free, bounded = ratio * A.double(), ratio.clamp(0.8, 1.2) * A.double()
    d = ref.double() - logp
    loss = (-torch.minimum(free, bounded) + 0.01 * (d.exp() - d - 1) + bonus * (table.exp() * table).sum(-1)).mean()
    loss.backward()
    # a dozen roundings of terms no larger than a token's share of the advantages, bonus and KL slopes
    size = ((A.abs() + 0.01 + bonus * 8) / (R * T)).max().item()
    assert (got.double() - x.grad).abs().max() < 40 * 2.0 ** -24 * size * 4
