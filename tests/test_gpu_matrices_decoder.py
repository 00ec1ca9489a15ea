"""The server's step over a whole decoder's vector (12 layers of width 768, vocabulary 50257): 48 matrices
orthogonalised, embeddings, biases and norms outside them, 4-byte offsets of up to half a gigabyte.

Every matrix is held to four times the error of the same steps with 32-bit products (both against torch's in
64 bits), the rest to w + update."""
import math

import pytest

import scores_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def steps(x):
    x = x / (x.double().norm().to(x.dtype) + 1e-7)
    wide = x if x.shape[0] <= x.shape[1] else x.T
    a, b, c = ref.QUINTIC
    for _ in range(5):
        gram = wide @ wide.T
        wide = a * wide + (b * gram + c * (gram @ gram)) @ wide
    return wide if x.shape[0] <= x.shape[1] else wide.T


def test_a_decoders_step():
    import paper_1905_12948_amd as gmc
    import synth
    sizes, h = synth.gpt2_small_sizes(), 768
    shapes = {h * 3 * h: (h, 3 * h), h * h: (h, h), h * 4 * h: (h, 4 * h)}
    table, at = [], 0
    for k, n in enumerate(sizes):
        if k >= 2 and n in shapes:      # not the embeddings; a layer's last matrix leads back to the width
            r, c = shapes[n]
            table.append((at, c, r) if n == h * 4 * h and sizes[k - 1] == 4 * h else (at, r, c))
        at += n
    assert len(table) == 48 and at == 124439808
    g = torch.Generator("cuda:0").manual_seed(8)
    w, m, u = (torch.randn(at, device="cuda:0", generator=g) * s for s in (0.02, 1e-3, 1e-3))
    plan = gmc.Matrices(at, table)
    past, rate, mu = m.clone(), 0.02, 0.9
    out = gmc.orthogonal_step(plan, w, u, past, rate, mu=mu, w_out=torch.empty_like(w))
    outside = torch.ones(at, dtype=torch.bool, device="cuda:0")
    for o, r, c in table:
        outside[o:o + r * c] = False
        x = (u + mu * past)[o:o + r * c].view(r, c)
        exact = steps(x.double())
        theirs = (steps(x).double() - exact).norm()
        mine = (((out.double() - w.double())[o:o + r * c].view(r, c)) / rate - exact).norm()
        # the step is seen through w's own rounding
        assert mine <= 4 * theirs + 2 * U * w[o:o + r * c].double().norm() / rate + 2 * U * math.sqrt(r), (o, r, c, mine.item(), theirs.item())
    assert torch.equal(out[outside], (w + u)[outside]) and torch.equal(past[outside], m[outside])
