"""gmc_orthogonalize and gmc_orthogonal_step on the GPU against their 64-bit
statement (scores_ref.py).

Tolerance: what is kept between the products (X, X X^T and the polynomial) is off by up to
2^-22 of each value, and a product's terms by 2^-22 of theirs.  How far such errors carry depends
on the matrix (the steps amplify small singular values by hundreds), so it is worked out for each: the
steps in 64 bits with errors of up to 2^-21 (both of the above) drawn at random for every value
kept, eight times; the result may be off by four times the largest of the eight, in the Frobenius
norm, and 4 * 2^-24 of the norm for the roundings of input and output; single entries by eight
times a row's or column's share of that.  16-bit outputs are rounded
once more, by half a step of each entry."""
import math

import numpy as np
import pytest

import scores_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
CUBIC = (1.5, -0.5, 0.0)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def host(t):
    return t.detach().double().cpu().numpy()


def near(got, m, factor, what, dtype="f32", **how):
    """`got` (64-bit array) is factor times the steps' result on m."""
    want = factor * ref.polar(m, **how)
    size = np.linalg.norm(want)
    tol = 4 * abs(factor) * ref.polar_spread(m, 2.0 ** -21, **how) + 4 * U * size
    off = np.linalg.norm(got - want)
    rounding = HALF[dtype] * size + (2.0 ** -24 * math.sqrt(want.size) if dtype == "f16" else 0.0)
    assert off <= tol + rounding, "%s: off by %g of %g, at %g" % (what, off, size, tol + rounding)
    entry = 8 * tol / math.sqrt(min(want.shape)) + HALF[dtype] * np.abs(want) + (2.0 ** -24 if dtype == "f16" else 0.0)
    assert (np.abs(got - want) <= entry + 1e-300).all(), what


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 2), (3, 33), (31, 5), (32, 32), (33, 32), (63, 65), (64, 64), (64, 147), (65, 64), (100, 300),
          (129, 127), (200, 37), (256, 256), (257, 640), (700, 96), (384, 384)]


def entries(rows, cols, seed):
    """A few strong directions over noise."""
    rng = np.random.default_rng(seed)
    rank = max(1, min(6, rows // 2, cols // 2))
    return rng.normal(size=(rows, rank)) @ rng.normal(size=(rank, cols)) + rng.normal(size=(rows, cols))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_orthogonalize(rows, cols, dtype):
    """Every shape, the vector longer than its matrix on both sides."""
    import paper_1905_12948_amd as gmc
    d = rows * cols + 11
    x = torch.randn(d).to(TYPES[dtype])
    x[5:5 + rows * cols] = torch.as_tensor(entries(rows, cols, rows * 1000 + cols)).reshape(-1).to(TYPES[dtype])
    x = x.cuda()
    plan = gmc.Matrices(d, [(5, rows, cols)], scales=[1.25])
    m = host(x)[5:-6].reshape(rows, cols)
    out = gmc.orthogonalize(plan, x, alpha=-0.5)
    near(host(out)[5:-6].reshape(rows, cols), m, -0.625, "out", dtype)
    assert torch.equal(out[:5], x[:5]) and torch.equal(out[-6:], x[-6:])
    same = x.clone()
    assert gmc.orthogonalize(plan, same, out=same, alpha=-0.5) is same
    assert torch.equal(same, out)


def test_larger_matrices():
    """Sides of several tiles of the larger kind, many of them, both ways round."""
    import paper_1905_12948_amd as gmc
    shapes = [(1030, 2050), (1500, 600), (640, 640), (2000, 130)] + [(64, 64)] * 9
    at, table = 0, []
    for r, c in shapes:
        table.append((at, r, c))
        at += r * c + 3
    x = torch.randn(at, device="cuda:0")
    plan = gmc.Matrices(at, table)
    out = gmc.orthogonalize(plan, x)
    for o, r, c in table:
        near(host(out[o:o + r * c]).reshape(r, c), host(x[o:o + r * c]).reshape(r, c), 1.0, (r, c))
        assert torch.equal(out[o + r * c:o + r * c + 3], x[o + r * c:o + r * c + 3])


@pytest.mark.parametrize("shapes", [
    [(5, 9), (40, 10), (64, 64), (1, 1), (30, 70), (64, 200)],     # of one workgroup each, by their longest side
    [(96, 160), (160, 96), (3, 3)], [(1, 600), (600, 1), (32, 32)], [(96, 161), (64, 64)],
    [(3, 4)] * 300 + [(4, 3)] * 40, [(512, 4608), (512, 2304), (64, 576), (10, 512)],   # long contractions
    [(1000, 2048), (64, 147), (128, 512)], [(300, 300), (64, 64), (1, 40)],
    # the longest that one workgroup takes, and those beyond
    [(32, 1248), (1248, 32)], [(64, 576), (576, 64), (50, 60)], [(96, 320), (33, 320)], [(128, 192), (192, 128), (100, 100)],
    [(32, 1249)], [(64, 577)], [(321, 96)], [(128, 193)], [(129, 129)],
    # G's product by large tiles, its square's by small ones
    [(1000, 1000)] + [(512, 3400)] * 8 + [(600, 512)] * 6])
def test_several_matrices(shapes):
    """Plans that take different ways through the launches, with and without momentum."""
    import paper_1905_12948_amd as gmc
    at, table = 1, []
    for r, c in shapes:
        table.append((at, r, c))
        at += r * c + 1
    g = torch.Generator(device="cuda:0").manual_seed(len(shapes))
    x, w, v = (torch.randn(at, device="cuda:0", generator=g) for _ in range(3))
    plan = gmc.Matrices(at, table)
    out = gmc.orthogonalize(plan, x)
    past, into = v.clone(), torch.empty_like(w)
    gmc.orthogonal_step(plan, w, x, past, 0.5, mu=0.5, w_out=into)
    outside = torch.ones(at, dtype=torch.bool, device="cuda:0")
    for o, r, c in table:
        outside[o:o + r * c] = False
    assert torch.equal(out[outside], x[outside]) and torch.equal(past[outside], v[outside])
    assert torch.equal(into[outside], w[outside] + x[outside])
    inside = past - (0.5 * v + x)
    assert (inside[~outside].abs() <= 4 * U * (v.abs() + x.abs())[~outside]).all()
    for o, r, c in table[:8] + table[-1:]:
        near(host(out[o:o + r * c]).reshape(r, c), host(x[o:o + r * c]).reshape(r, c), 1.0, (r, c))
        u = (x + 0.5 * past)[o:o + r * c]
        step = host(into[o:o + r * c]) - host(w[o:o + r * c])
        want = 0.5 * ref.polar(host(u).reshape(r, c)).reshape(-1)
        tol = 2 * ref.polar_spread(host(u).reshape(r, c), 2.0 ** -21) + 4 * U * np.linalg.norm(host(w[o:o + r * c]))
        assert np.linalg.norm(step - want) <= tol + 4 * U * np.linalg.norm(want), (r, c)


def test_columns_and_single_rows():
    """Column slices of one array, a narrower one between them, rows of the rest in the gaps."""
    import paper_1905_12948_amd as gmc
    rows, wide = 50, 240
    d = rows * wide + 9
    table = [(2, rows, 64, wide), (66, rows, 100, wide), (180, rows, 33, wide), (230, 1, 6)]
    x = torch.randn(d, device="cuda:0")
    plan = gmc.Matrices(d, table)
    out = gmc.orthogonalize(plan, x)
    free = np.ones(d, bool)
    for e in table:
        pitch = e[3] if len(e) > 3 else e[2]
        at = e[0] + np.arange(e[1])[:, None] * pitch + np.arange(e[2])[None, :]
        near(host(out)[at], host(x)[at], 1.0, e)
        free[at] = False
    assert free.sum() > 0 and np.array_equal(host(out)[free], host(x)[free])


@pytest.mark.parametrize("steps,coefficients", [(1, ref.QUINTIC), (2, CUBIC), (12, CUBIC), (3, [(2.0, -1.5, 0.5), CUBIC, (1.875, -1.25, 0.375)]),
                                                (1, (700.0, 0.0, 0.0)), (2, [(1.0, 0.0, 0.0), (0.0, 1.0, 0.0)])])
def test_coefficients(steps, coefficients):
    import paper_1905_12948_amd as gmc
    for rows, cols in ((40, 90), (90, 40)):
        m = entries(rows, cols, steps)
        x = torch.as_tensor(m, dtype=torch.float32).reshape(-1).cuda()
        plan = gmc.Matrices(rows * cols, [(0, rows, cols)])
        got = host(gmc.orthogonalize(plan, x, steps=steps, coefficients=coefficients)).reshape(rows, cols)
        near(got, host(x).reshape(rows, cols), 1.0, coefficients, steps=steps, coefficients=coefficients)


def test_singular_values_and_vectors():
    """A cubic iteration ends at the nearest matrix with orthonormal rows; the quintic one leaves
    a diagonal matrix diagonal, each entry taken as a number is."""
    import paper_1905_12948_amd as gmc
    g = torch.Generator().manual_seed(1)
    m = torch.randn(96, 200, generator=g)
    plan = gmc.Matrices(m.numel(), [(0, 96, 200)])
    o = gmc.orthogonalize(plan, m.reshape(-1).cuda(), steps=24, coefficients=CUBIC).view(96, 200).double().cpu()
    u, _, v = torch.linalg.svd(m.double(), full_matrices=False)
    # An error that turns the rows stays, so those of 24 steps add up, independent of one another: of a
    # step the kept X's rounding (2^-22 of a value at most), the products' left out part (2^-22) and the
    # roundings of 18 sums in 32 bits (96 columns, 16 at a time, three products: 2^-24 each), as a sum of squares.
    step = (2 * 2.0 ** -44 + 18 * 2.0 ** -48) ** 0.5
    assert torch.linalg.matrix_norm(o - u @ v) < 24 ** 0.5 * step * 96 ** 0.5
    values = torch.linspace(0.01, 1.0, 70, dtype=torch.float64)
    plan = gmc.Matrices(4900, [(0, 70, 70)])
    got = host(gmc.orthogonalize(plan, torch.diag(values).float().reshape(-1).cuda(), eps=0.0)).reshape(70, 70)
    s = values.numpy() / np.linalg.norm(values.numpy())
    for _ in range(5):
        s = s * (3.4445 + s * s * (-4.7750 + 2.0315 * s * s))
    assert np.array_equal(got != 0, np.eye(70) != 0)
    # relative: 22 bits in each of five steps' sums, whose terms cancel to a fifth at most
    assert np.abs(np.diag(got) / s - 1).max() < 5 * 5 * 3 * 2.0 ** -22


@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-7, 1.0, 1e12, 1e30, 1e37])
def test_sizes(size):
    """Sums of squares beyond 32 bits' range, below and above."""
    import paper_1905_12948_amd as gmc
    m = torch.randn(50, 60) * size
    plan = gmc.Matrices(3000, [(0, 50, 60)])
    for eps in (0.0, 1e-7):
        got = host(gmc.orthogonalize(plan, m.reshape(-1).cuda(), eps=eps)).reshape(50, 60)
        near(got, host(m), 1.0, (size, eps), eps=float(np.float32(eps)))


def test_zero_and_odd_matrices_keep_to_themselves():
    """A matrix of zeros stays zero, one with a NaN or an infinity becomes NaN, its neighbours do not."""
    import paper_1905_12948_amd as gmc
    n = 40 * 70
    x = torch.randn(6 * n, device="cuda:0")
    plan = gmc.Matrices(6 * n, [(k * n, 40, 70) for k in range(6)])
    want = gmc.orthogonalize(plan, x)
    x[n:2 * n] = 0
    x[3 * n + 5] = math.nan
    x[5 * n - 1] = math.inf
    for eps in (0.0, 1e-7):
        out = gmc.orthogonalize(plan, x, eps=eps).view(6, n)
        assert (out[1] == 0).all() and torch.isnan(out[3]).all() and torch.isnan(out[4]).all()
        if eps:
            for k in (0, 2, 5):
                assert torch.equal(out[k], want.view(6, n)[k])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("momentum", [True, False])
def test_step(dtype, nesterov, momentum):
    """Momentum, direction, decay and the components outside, into another buffer and in place."""
    import paper_1905_12948_amd as gmc
    table = [(3, 30, 50), (1510, 50, 30), (3020, 33, 40, 97), (3062, 33, 50, 97), (6300, 1, 9)]
    d, scales = 6320, [1.0, 1.3, 0.5, 1.0, 2.0]
    g = torch.Generator().manual_seed(9)
    w, m = torch.randn(d, generator=g), torch.randn(d, generator=g) * 0.1
    u = (torch.randn(d, generator=g) * 0.2).to(TYPES[dtype])
    w0, m0, u0 = w.double().numpy(), m.double().numpy(), u.double().numpy()
    plan = gmc.Matrices(d, table, scales=scales)
    rate, mu, decay = 0.05, 0.9, 0.01
    w, u, m = w.cuda(), u.cuda(), m.cuda()
    out = torch.empty_like(w)
    v = m.clone() if momentum else None
    how = dict(mu=mu, nesterov=nesterov, decay=decay)
    assert gmc.orthogonal_step(plan, w, u, v, rate, w_out=out, **how) is out
    got, free = host(out), np.ones(d, bool)
    for e, s in zip(table, scales):
        pitch = e[3] if len(e) > 3 else e[2]
        at = e[0] + np.arange(e[1])[:, None] * pitch + np.arange(e[2])[None, :]
        free[at] = False
        past = mu * m0[at] + u0[at] if momentum else u0[at]
        if momentum:   # two roundings of its terms, mu's own
            assert (np.abs(host(v)[at] - past) <= 3 * U * (np.abs(m0[at]) + np.abs(past))).all()
            x = u0[at] + mu * past if nesterov else past
        else:
            x = u0[at]
        want = rate * s * ref.polar(x)
        rough = 4 * ref.polar_spread(x, 2.0 ** -21) * rate * s
        off = got[at] - (1 - decay) * w0[at] - want
        # x's own roundings (four of 2^-24) are amplified as the kept values' are: within `rough`
        assert np.linalg.norm(off) <= rough + 4 * U * (np.linalg.norm(w0[at]) + np.linalg.norm(want)), e
    if momentum:
        assert np.array_equal(host(v)[free], m0[free])
    assert np.array_equal(got[free], (w.cpu() + u.float().cpu()).double().numpy()[free])
    assert torch.equal(w.cpu().double(), torch.as_tensor(w0))
    again = m.clone() if momentum else None
    assert gmc.orthogonal_step(plan, w, u, again, rate, **how) is w
    assert torch.equal(w, out) and (v is None or torch.equal(again, v))
    assert torch.equal(u.cpu().double(), torch.as_tensor(u0))


def test_step_without_matrices_is_apply():
    import paper_1905_12948_amd as gmc
    w, u = torch.randn(20000, device="cuda:0"), torch.randn(20000, device="cuda:0")
    plan = gmc.Matrices(20000, [])
    assert torch.equal(gmc.orthogonal_step(plan, w, u, None, 0.1, w_out=torch.empty_like(w)), w + u)
    assert torch.equal(gmc.orthogonalize(plan, w), w)


def test_vectors_longer_than_the_plan():
    """What lies behind the plan's components stays as it is; a new result has the plan's."""
    import paper_1905_12948_amd as gmc
    d = 40 * 30 + 5
    x, w, m = (torch.randn(d + 100, device="cuda:0") for _ in range(3))
    plan = gmc.Matrices(d, [(0, 40, 30)])
    out = gmc.orthogonalize(plan, x)
    assert out.shape == (d,)
    into = torch.full((d + 60,), 3.0, device="cuda:0")
    gmc.orthogonalize(plan, x, out=into)
    assert torch.equal(into[:d], out) and (into[d:] == 3).all()
    shaped = gmc.orthogonalize(plan, x[:d].view(5, 241))
    assert shaped.shape == (5, 241) and torch.equal(shaped.reshape(-1), out)
    before = m.clone()
    into.fill_(3.0)
    gmc.orthogonal_step(plan, w, x, m, 0.1, w_out=into)
    assert (into[d:] == 3).all() and torch.equal(m[1200:], before[1200:])


def test_long_vector_without_matrices_in_most_of_it():
    import paper_1905_12948_amd as gmc
    d = (1 << 30) + 12345
    x = torch.ones(d, device="cuda:0", dtype=torch.float16)
    x[77:77 + 900] = torch.randn(900, device="cuda:0").half()
    plan = gmc.Matrices(d, [(77, 30, 30), (d - 5, 1, 5)])
    out = gmc.orthogonalize(plan, x)
    near(host(out[77:977]).reshape(30, 30), host(x[77:977]).reshape(30, 30), 1.0, "first", "f16")
    near(host(out[-5:]).reshape(1, 5), host(x[-5:]).reshape(1, 5), 1.0, "last", "f16")
    assert (out[:77] == 1).all() and (out[977:-5] == 1).all()


def test_same_bits_streams_and_graphs():
    """The same bits twice, on a side stream, and in two graphs that share a plan and are replayed in
    turn with other inputs between eager calls."""
    import paper_1905_12948_amd as gmc
    d = 300 * 200 + 64 * 500
    plan = gmc.Matrices(d, [(0, 300, 200), (60000, 64, 500)])
    x, w, m = (torch.randn(d, device="cuda:0") for _ in range(3))
    want = gmc.orthogonalize(plan, x)
    assert torch.equal(gmc.orthogonalize(plan, x), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = gmc.orthogonalize(plan, x)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, want)
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    held_m = m.clone()
    with torch.cuda.graph(one):
        held = gmc.orthogonalize(plan, x)
    with torch.cuda.graph(two):
        stepped = gmc.orthogonal_step(plan, w, x, held_m, 0.02, w_out=torch.empty_like(w))
    eager_m = m.clone()
    held_m.copy_(m)
    for _ in range(4):
        x.copy_(torch.randn(d, device="cuda:0"))
        one.replay()
        two.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, gmc.orthogonalize(plan, x))
        assert torch.equal(stepped, gmc.orthogonal_step(plan, w, x, eager_m, 0.02, w_out=torch.empty_like(w)))
        assert torch.equal(held_m, eager_m)


def test_far_offsets():
    """A matrix that begins more than 2^32 bytes into the vector."""
    import paper_1905_12948_amd as gmc
    far = (1 << 31) + 12345
    d = far + 70 * 90 + 2
    x = torch.zeros(d, device="cuda:0", dtype=torch.bfloat16)
    m = torch.randn(70, 90).to(torch.bfloat16)
    x[far:far + 6300] = m.reshape(-1).cuda()
    plan = gmc.Matrices(d, [(far, 70, 90)])
    gmc.orthogonalize(plan, x, out=x)
    near(host(x[far:far + 6300]).reshape(70, 90), host(m), 1.0, "far", "bf16")
    assert (x[:far] == 0).all() and (x[-2:] == 0).all()


def test_one_row_of_the_most_columns():
    """Parts of G's sum lie beyond 32 bits of halves.  With 1.5 - 0.5 s^2 a singular value of
    1 stays, and an error of G counts half: of 2^26 squares summed in 512 parts, 16 to a step, at most (8192 + 512)
    2^-24, once a step (the slope at 1 is 0)."""
    import paper_1905_12948_amd as gmc
    d = 1 << 26
    x = torch.randn(d, device="cuda:0", generator=torch.Generator("cuda:0").manual_seed(5)).half()
    plan = gmc.Matrices(d, [(0, 1, d)])
    out = gmc.orthogonalize(plan, x, steps=2, coefficients=(1.5, -0.5, 0.0))
    want = x.double() / x.double().norm()
    # halves below 2^-14 round to multiples of 2^-24
    error = (out.double() - want).abs() - want.abs() * (0.5 * 8704 * 2.0 ** -24 * 1.1 + 2.0 ** -11 + 2.0 ** -20) - 2.0 ** -25
    assert (error <= 0).all(), float(error.max())
    del plan, out, want, error
    torch.cuda.empty_cache()


def test_refusals():
    import paper_1905_12948_amd as gmc
    d = 64
    plan = gmc.Matrices(d, [(0, 4, 5), (20, 3, 3)])
    x, y, z = (torch.randn(3 * d, device="cuda:0")[:d] for _ in range(3))
    both = torch.randn(2 * d, device="cuda:0")
    calls = [
        (lambda: gmc.orthogonalize(plan, x.cpu()), ValueError), (lambda: gmc.orthogonalize(plan, x.double()), TypeError),
        (lambda: gmc.orthogonalize(plan, x[:60]), ValueError), (lambda: gmc.orthogonalize(plan, both[::2]), ValueError),
        (lambda: gmc.orthogonalize(plan, x, out=x.half()), TypeError), (lambda: gmc.orthogonalize(plan, x, steps=0), ValueError),
        (lambda: gmc.orthogonalize(plan, x, steps=65), ValueError), (lambda: gmc.orthogonalize(plan, x, coefficients=(1, 2)), ValueError),
        (lambda: gmc.orthogonalize(plan, x, steps=2, coefficients=[(1.0, 0.0, 0.0)]), ValueError),
        (lambda: gmc.orthogonalize(plan, x, coefficients=(3.0, 0.0, 0.0)), RuntimeError),       # grows beyond 2.5
        (lambda: gmc.orthogonalize(plan, x, steps=2, coefficients=[(0.2, 0.0, 0.0), (2.0, -1.0, 0.0)]), RuntimeError),   # below 0.25
        (lambda: gmc.orthogonalize(plan, x, steps=2, coefficients=[(0.0, 0.0, 0.0), (1e300, 0.0, 0.0)]), RuntimeError),
        (lambda: gmc.orthogonalize(plan, x, coefficients=(1.0, -61.0, 0.0)), RuntimeError),
        (lambda: gmc.orthogonalize(plan, x, coefficients=(math.nan, 0.0, 0.0)), RuntimeError),
        (lambda: gmc.orthogonalize(plan, x, eps=-1.0), RuntimeError), (lambda: gmc.orthogonalize(plan, x, eps=math.nan), RuntimeError),
        (lambda: gmc.orthogonalize(plan, x, alpha=1e39), RuntimeError), (lambda: gmc.orthogonalize(plan, both[:d], out=both[8:8 + d]), RuntimeError),
        (lambda: gmc.orthogonalize(None, x), TypeError),
        (lambda: gmc.orthogonal_step(plan, x, y.double(), z, 0.1), TypeError), (lambda: gmc.orthogonal_step(plan, x.half(), y, z, 0.1), TypeError),
        (lambda: gmc.orthogonal_step(plan, x, y, z.half(), 0.1), TypeError), (lambda: gmc.orthogonal_step(plan, x, x, z, 0.1), RuntimeError),
        (lambda: gmc.orthogonal_step(plan, x, y, y, 0.1), RuntimeError), (lambda: gmc.orthogonal_step(plan, x, y, x, 0.1), RuntimeError),
        (lambda: gmc.orthogonal_step(plan, x, y, z, math.inf), RuntimeError), (lambda: gmc.orthogonal_step(plan, x, y, z, 0.1, mu=1.5), RuntimeError),
        (lambda: gmc.orthogonal_step(plan, x, y, z, 0.1, decay=math.nan), RuntimeError),
        (lambda: gmc.orthogonal_step(plan, both[:d], y, z, 0.1, w_out=both[4:4 + d]), RuntimeError),
        (lambda: gmc.Matrices(d, [(0, 4)]), ValueError), (lambda: gmc.Matrices(d, [(0, 4, 4)], scales=[1, 2]), ValueError),
        (lambda: gmc.Matrices(d, [(0, 9, 9)]), RuntimeError), (lambda: gmc.Matrices(d, [], device="cpu"), ValueError),
        (lambda: gmc.Matrices(d, [(0, 2 ** 64, 1)]), ValueError),
    ]
    before = [t.clone() for t in (x, y, z, both)]
    for k, (bad, error) in enumerate(calls):
        with pytest.raises(error):
            bad()
            print("call", k, "was taken")
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, (x, y, z, both)))
    plan.close()
    with pytest.raises(ValueError):
        gmc.orthogonalize(plan, x)


def test_scores_losses_and_the_server_together():
    """A worker's pass and the server's step as they follow each other: scores of the rollouts, the policy
    loss with an entropy bonus, K workers' messages, and the orthogonalised step from their sum;
    every figure against the same in 64 bits."""
    import paper_1905_12948_amd as gmc
    g = torch.Generator(device="cuda:0").manual_seed(4)
    K, F, V, R, T = 3, 24, 60, 4, 5
    d = F * V + V
    w = torch.randn(d, device="cuda:0", generator=g) * 0.3
    plan = gmc.Matrices(d, [(0, F, V)])
    server = gmc.Gmc(d, K, "topk", ratio=0.05, beta=0.0, eta=1.0)
    idx, val, ln = server.alloc_messages()
    err, update, momentum, nxt = torch.zeros(K, d, device="cuda:0"), torch.empty(d, device="cuda:0"), torch.zeros(d, device="cuda:0"), torch.empty(d, device="cuda:0")
    rows, bonus, total = [], 0.01, np.zeros(d)
    for k in range(K):
        h = torch.randn(R, T, F, device="cuda:0", generator=g)
        logits = (h @ w[:F * V].view(F, V) + w[F * V:]).contiguous()
        tokens = torch.randint(0, V, (R, T), device="cuda:0", generator=g)
        old, entropy, _, _, norm = gmc.token_scores(logits, tokens)
        A = torch.randn(R, device="cuda:0", generator=g)
        stats, logp, grad = gmc.policy_loss(logits, tokens, old, A)
        assert torch.allclose(logp, old, rtol=0, atol=1e-5)
        grad = grad + gmc.token_scores_backward(logits, norm, tokens, entropy=entropy, dentropy=torch.full((R, T), -bonus / (R * T), device="cuda:0"))
        # at ratio 1 the policy's slope is -A / tokens
        want = ref.scores_gradient(host(logits).reshape(R * T, V), 1.0, tokens.cpu().numpy().reshape(-1),
                                   np.repeat(-host(A), T) / (R * T), np.full(R * T, -bonus / (R * T)), np.zeros((R * T, 0), int), np.zeros((R * T, 0)))
        assert np.abs(host(grad).reshape(R * T, V) - want).max() < 1e-6
        rows.append(torch.cat([(h.reshape(-1, F).T @ grad.view(-1, V)).reshape(-1), grad.view(-1, V).sum(0)]))
    grads = torch.stack(rows)
    server.step(w, w.clone(), grads, err, idx, val, ln)
    server.aggregate(idx, val, ln, update)
    for k in range(K):
        np.add.at(total, idx[k, :int(ln[k])].cpu().numpy(), host(val[k, :int(ln[k])]))
    assert np.allclose(host(update), -total / K, rtol=0, atol=1e-6)
    gmc.orthogonal_step(plan, w, update, momentum, 0.02, w_out=nxt)
    u = host(update)[:F * V].reshape(F, V)
    near((host(nxt) - host(w))[:F * V].reshape(F, V) / 0.02, u * 1.95, 1.0, "step", "bf16")   # w's roundings are 2^-8 of a step's size
    assert torch.equal(nxt[F * V:], w[F * V:] + update[F * V:])
    server.close()
