"""The worker-side operators on the GPU at the ends of their ranges of sizes."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24
HALF = 2.0 ** -8     # half a step of bfloat16, of the value


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def summed(f, n, step=2 ** 27):
    """The sum over [0, n) of f(a, b), fp64 tensors of sums over [a, b)."""
    return sum(f(a, min(n, a + step)) for a in range(0, n, step))


def test_group_norm_of_the_longest_image():
    """One image of 2^31 - 1 pixels, forward and backward."""
    import paper_1905_12948_amd as gmc
    S = 2 ** 31 - 1
    g = torch.Generator(device="cuda:0").manual_seed(5)
    x = torch.empty(1, S, 1, device="cuda:0", dtype=torch.bfloat16).normal_(0.5, 1.0, generator=g)
    dy = torch.empty_like(x).normal_(0.25, 1.0, generator=g)
    gamma, beta = torch.tensor([1.25], device="cuda:0"), torch.tensor([0.125], device="cuda:0")
    y, mean, rstd = gmc.group_norm(x, 1, gamma, beta, act="relu")
    v, d = x.view(-1), dy.view(-1)
    mu = summed(lambda a, b: v[a:b].double().sum(), S).item() / S
    size = summed(lambda a, b: v[a:b].double().abs().sum(), S).item() / S
    var = summed(lambda a, b: ((v[a:b].double() - mu) ** 2).sum(), S).item() / S
    # sums of 64 values a thread, 6 steps of a wavefront, 4 wavefronts, then 2048 pieces a lane and
    # 6 steps: 2200 roundings of at most the mean size of a term; a thread's terms are differences
    # from a value of its own, which add that value's mean size
    many = 2200 * U
    assert abs(mean.item() - mu) <= many * 2 * size, (mean.item(), mu)
    assert abs(rstd.item() - 1 / math.sqrt(var + 1e-5)) <= 2 * many * rstd.item(), (rstd.item(), var)
    dx, dgamma, dbeta = gmc.group_norm_backward(dy, x, mean, rstd, gamma, beta, act="relu")
    m, r = mean.item(), rstd.item()

    def parts(a, b):
        # relu's side as the kernels take it: z in 32 bits, one rounding an operation
        on = ((v[a:b].float() - mean) * rstd).view(-1) * gamma + beta > 0
        hat = (v[a:b].double() - m) * r
        dz = d[a:b].double() * on
        return hat, dz

    def sums(a, b):
        hat, dz = parts(a, b)
        return torch.stack([dz.sum(), (dz * hat).sum(), dz.abs().sum(), (dz * hat).abs().sum()])

    sb, sg, ab, ag = summed(sums, S).tolist()
    assert abs(dbeta.item() - sb) <= many * ab, (dbeta.item(), sb)
    assert abs(dgamma.item() - sg) <= many * 2 * ag, (dgamma.item(), sg)
    for a, b in [(0, 5000), (2 ** 30 - 2500, 2 ** 30 + 2500), (S - 40000, S)]:
        hat, dz = parts(a, b)
        z = (hat * 1.25 + 0.125).clamp(min=0)
        err = (y.view(-1)[a:b].double() - z).abs()
        assert (err <= HALF * z + 8 * U * (hat.abs() + 1)).all(), (a, err.max().item())
        want = r * (1.25 * dz - 1.25 * (sb + hat * sg) / S)
        slack = 8 * U * r * 1.25 * (dz.abs() + hat.abs() + 1) + many * 2 * r * 1.25 * (ab + hat.abs() * ag) / S
        err = (dx.view(-1)[a:b].double() - want).abs()
        assert (err <= HALF * want.abs() + 1.01 * slack).all(), (a, err.max().item())


@pytest.mark.parametrize("N,C,G,dtype", [
    (2 ** 24 + 4099, 12, 4, torch.bfloat16),     # 256 threads an image
    (2 ** 26 + 4099, 16, 2, torch.bfloat16),     # 64
    (2 ** 26 + 4099, 32, 4, torch.bfloat16),     # 64
    (2 ** 24 + 4099, 4, 2, torch.float32),       # 64, in one launch
])
def test_group_norm_of_more_images_than_a_launch_has(N, C, G, dtype):
    """As many calls of fewer images give the same bits, at both ends and across 2^32 threads."""
    import paper_1905_12948_amd as gmc
    g = torch.Generator(device="cuda:0").manual_seed(C)
    x = torch.empty(N, 1, C, device="cuda:0", dtype=dtype).normal_(0.5, 1.0, generator=g)
    dy = torch.randint(0, 2, x.shape, device="cuda:0", generator=g, dtype=torch.uint8).to(dtype)
    gamma, beta = torch.linspace(0.5, 1.5, C, device="cuda:0"), torch.linspace(-0.2, 0.2, C, device="cuda:0")
    y, mean, rstd = gmc.group_norm(x, G, gamma, beta)
    dx, dgamma, dbeta = gmc.group_norm_backward(dy, x, mean, rstd, gamma, beta)
    # enough for thresholds on the images' number and bytes to fall as in the whole call
    few = 4099 if C in (12, 32) else 2 ** 22
    for a in (0, 2 ** 24 - few // 2, 2 ** 24 - few + 5, N - few):
        part = x[a:a + few].contiguous()
        want = gmc.group_norm(part, G, gamma, beta)
        for got, w in zip((y, mean, rstd), want):
            assert torch.equal(got[a:a + few], w), a
        assert torch.equal(dx[a:a + few], gmc.group_norm_backward(dy[a:a + few].contiguous(), part, *want[1:], gamma, beta)[0]), a
    # zeros and ones: every slot of 16 has a whole number below 2^24, exactly; then four roundings
    exact = dy.float().view(N, C).sum(0, dtype=torch.float64)
    assert ((dbeta.double() - exact).abs() <= 4 * U * exact).all(), (dbeta, exact)
    # a slot's N / 16 terms and a tree: its worst case, loose as it is, and the sums' own sizes
    hat = (x.view(N, G, -1).float() - mean[:, :, None]) * rstd[:, :, None]
    terms = dy.view(N, C).double() * hat.view(N, C)
    bound = (N / 16 + 8) * U * terms.abs().sum(0)
    assert ((dgamma.double() - terms.sum(0)).abs() <= bound).all()


def test_group_norm_in_pieces_of_more_images_than_a_launch_has():
    """A wavefront a group joins the pieces: 1442 images of 46,523 groups have 2^32 threads."""
    import paper_1905_12948_amd as gmc
    N, G, C = 1600, 46523, 3 * 46523
    g = torch.Generator(device="cuda:0").manual_seed(1)
    x = torch.empty(N, 1, C, device="cuda:0", dtype=torch.bfloat16).normal_(0.5, 1.0, generator=g)
    dy = torch.randint(0, 2, x.shape, device="cuda:0", generator=g, dtype=torch.uint8).bfloat16()
    gamma, beta = torch.linspace(0.5, 1.5, C, device="cuda:0"), torch.linspace(-0.2, 0.2, C, device="cuda:0")
    y, mean, rstd = gmc.group_norm(x, G, gamma, beta, act="relu")
    dx, dgamma, dbeta = gmc.group_norm_backward(dy, x, mean, rstd, gamma, beta)
    for a, b in ((0, 300), (1300, 1600)):
        want = gmc.group_norm(x[a:b].contiguous(), G, gamma, beta, act="relu")
        for got, w in zip((y, mean, rstd), want):
            assert torch.equal(got[a:b], w), a
        back = gmc.group_norm_backward(dy[a:b].contiguous(), x[a:b].contiguous(), *want[1:], gamma, beta)
        assert torch.equal(dx[a:b], back[0]), a
    assert torch.equal(dbeta.double(), dy.double().sum((0, 1)))   # whole numbers, exactly
    hat = (x.view(N, G, 3).float() - mean[:, :, None]) * rstd[:, :, None]
    terms = dy.view(N, C).double() * hat.view(N, C)
    assert ((dgamma.double() - terms.sum(0)).abs() <= (N / 16 + 8) * U * terms.abs().sum(0)).all()
