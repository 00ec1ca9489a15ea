"""Group norm through every kernel and branch of its plan (norm_forms.SHAPES) against the
formulas in 64 bits, on the GPU.

Tolerances, with u = 2^-24: a sum passes through at most `many` additions (128 values or 64
pixels of a thread, 6 steps of a wavefront, 16 wavefronts, a lane's share of the pieces and
6 steps again), so it is off by at most many u of the sum of its terms' sizes; a thread's terms
of the moments are differences from its first value, whose size adds that of the group's
largest one.  Values are held against the formulas of the call's own mean and rstd, so they
are off by the roundings of one element."""
import pytest

import norm_forms as forms

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": (0.0, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -24)}  # half a step, of the value and least


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    return forms.build(str(tmp_path_factory.mktemp("plan")))


def within(got, want, slack, dtype, what):
    rel, least = HALF[dtype]
    got = got.double()
    tol = slack + rel * (want.abs() + slack) + least
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %g of the tolerance" % (
        what, bad.sum().item(), bad.numel(), ((got - want).abs() / tol)[bad].max().item())


def many_u(plan, dtype, N, S, C, G, backward):
    p = plan(4 if dtype == "f32" else 2, N, S, C, G, backward)
    return U * (128 + 6 + 16 + 8 + p["chunks"] * (C // G) / 64 + 6)


def activated(z, kind):
    return z.clamp(min=0) if kind == "relu" else z * torch.sigmoid(z) if kind == "silu" else z


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("N,S,C,G", forms.SHAPES)
def test_group_norm(plan, N, S, C, G, kind, dtype):
    import paper_1905_12948_amd as gmc
    g = torch.Generator(device="cuda:0").manual_seed(N * S + C)
    normal = lambda *shape: torch.randn(*shape, device="cuda:0", generator=g)  # noqa: E731
    x = (normal(N, S, C) * torch.exp(0.5 * normal(C)) + 0.7 * normal(C)).to(TYPES[dtype])
    dy = normal(N, S, C).to(TYPES[dtype])
    gamma, beta = 1 + 0.3 * normal(C), 0.3 * normal(C)
    y, mean, rstd = gmc.group_norm(x, G, gamma, beta, act=kind)
    dx, dgamma, dbeta = gmc.group_norm_backward(dy, x, mean, rstd, gamma, beta, act=kind)

    grouped = lambda t: t.reshape(N, S, G, C // G)  # noqa: E731
    v, m = grouped(x.double()), S * (C // G)
    mu = v.mean((1, 3))
    var = ((v - mu[:, None, :, None]) ** 2).mean((1, 3))
    many = many_u(plan, dtype, N, S, C, G, 0)
    sizes = v.abs().mean((1, 3)) + v.abs().amax((1, 3))
    within(mean, mu, many * sizes, "f32", "mean")
    # an error e of the mean adds e^2 to the variance; a pivot as far out as a group's value can be, among the
    # at most 128 values of its thread, leaves 128 times the rounding of a share of the squares
    want = 1 / torch.sqrt(var + 1e-5)
    wrong = many * var + 128 * U * var + (many * sizes) ** 2
    within(rstd, want, 0.5 * want ** 3 * wrong + 8 * U * want, "f32", "rstd")

    # by the call's own mean and rstd
    mu, rs = (t.double()[:, None, :, None] for t in (mean, rstd))
    ga, be = gamma.double(), beta.double()
    hat = ((v - mu) * rs).reshape(N, S, C)
    z = hat * ga + be
    ez = U * (6 * (hat * ga).abs() + 2 * be.abs())
    silu = U * z.abs() * (8 + 2 * z.abs()) if kind == "silu" else 0
    within(y, activated(z, kind), 1.1 * ez + silu, dtype, "y")

    d = dy.double()
    if kind == "relu":  # the kernels' side of the corner: z in 32 bits, one rounding an operation
        z32 = ((grouped(x.float()) - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(N, S, C) * gamma + beta
        dz, edz = d * (z32 > 0), torch.zeros_like(d)
    elif kind == "silu":
        gate = torch.sigmoid(z)
        dz = d * gate * (1 + z * (1 - gate))
        edz = d.abs() * (U * 20 * (1 + z.abs()) + 1.1 * ez)
    else:
        dz, edz = d, torch.zeros_like(d)
    many = many_u(plan, dtype, N, S, C, G, 1)
    images = U * (N / 16 + 8)
    size, eh = dz.abs(), 3 * U * hat.abs()
    within(dbeta, dz.sum((0, 1)), (edz + (many + images) * size).sum((0, 1)), "f32", "dbeta")
    within(dgamma, (dz * hat).sum((0, 1)), (edz * hat.abs() + (many + images) * size * hat.abs() + size * eh).sum((0, 1)), "f32",
           "dgamma")
    wide = lambda t: (t.reshape(N, S, G, -1).sum((1, 3), keepdim=True) / m).expand(N, S, G, C // G).reshape(N, S, C)  # noqa: E731
    s1, s2 = wide(dz * ga), wide(dz * ga * hat)
    e1 = wide((edz + (many + 4 * U) * size) * ga.abs())
    e2 = wide((edz * hat.abs() + (many + 4 * U) * size * hat.abs() + size * eh) * ga.abs())
    r = rstd.double()[:, None, :, None].expand(N, S, G, C // G).reshape(N, S, C)
    err = edz * ga.abs() + e1 + hat.abs() * e2 + 8 * U * ((dz * ga).abs() + s1.abs() + (hat * s2).abs())
    within(dx, r * (dz * ga - (s1 + hat * s2)), r * err, dtype, "dx")


@pytest.mark.parametrize("N,S,C,G", forms.SHAPES)
def test_group_norm_sums_of_whole_numbers(plan, N, S, C, G):
    """Whole numbers, whose sums over a group or over the images below 2^24 are exact in any
    order: no pixel, channel or image is left out or taken twice, in any of the three types."""
    import paper_1905_12948_amd as gmc
    g = torch.Generator(device="cuda:0").manual_seed(N + S + C)
    x = torch.randint(-2, 4, (N, S, C), device="cuda:0", generator=g)
    d = torch.randint(-1, 3, (N, S, C), device="cuda:0", generator=g)
    exact_mean = x.reshape(N, S, G, -1).double().mean((1, 3))
    exact_beta = d.sum((0, 1)).double()
    assert x.reshape(N, S, G, -1).abs().sum((1, 3)).max() < 2 ** 24 and d.abs().sum((0, 1)).max() < 2 ** 24
    for dtype, code in TYPES.items():
        _, mean, rstd = gmc.group_norm(x.to(code), G)
        dx, dgamma, dbeta = gmc.group_norm_backward(d.to(code), x.to(code), mean, rstd)
        size = 4 if dtype == "f32" else 2
        # the reciprocal of the number of values and its product; pieces hold their channels' means, which round
        slack = 2 * U * exact_mean.abs() if plan(size, N, S, C, G, 0)["held"] else many_u(plan, dtype, N, S, C, G, 0) * 5
        assert ((mean.double() - exact_mean).abs() <= 1.01 * slack).all(), dtype
        assert torch.equal(dbeta.double(), exact_beta), dtype
