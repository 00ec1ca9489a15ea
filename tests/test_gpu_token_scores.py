"""gmc_token_scores and its gradient on the GPU against their 64-bit statements
(scores_ref.py).

Tolerances, with u = 2^-24 (one 32-bit rounding), z = (x - max) / tau <= 0 and S = sum
exp z:
  S       a thread adds at most 8 * 13 + 1 terms, a row's threads join by 6 + 8 more: 120
          roundings; an exponential is within 2 roundings and its exponent's 2 are
          |z| log2(e) 2 u in it, with the mean of |z| under p at most ln V: 120 + 2 + 3 ln V
  logp    z's three roundings 3 |z| u, ln S's own, the difference's, and S's: (4 |z| +
          2 |ln S| + 123 + 3 ln V) u
  H       ln S - U / S, U = sum e z: S's error twice, |U / S| its roundings (123 + 3) |U / S| and
          its exponents' 3 mean(z^2): (250 + 130 ln V + 3 mean(z^2)) u at most
  gradient p (c + d q): p's relative error is 2 |ln p| + |ln S| (norm's own rounding and
          its use: twice) + 6, c's three terms' 8 u each; the single entries' sums 40 u
16-bit outputs are rounded once more, by half a step."""
import math

import numpy as np
import pytest

import scores_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": (0.0, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -24)}
IGNORE = -100


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def host(t):
    return t.detach().double().cpu().numpy()


def within(got, want, tol, what):
    got = host(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    same = (got == want) | np.isnan(want)          # infinities
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - want) <= tol))
    assert not bad.any(), "%s: %d of %d off, worst %g at %g" % (
        what, bad.sum(), bad.size, np.abs(got - want)[bad].max(), np.broadcast_to(tol, bad.shape)[bad].min())


def compare(x, labels, tau, top, got=None):
    """A forward call on x [R, T, V] against the 64-bit one; labels without ignored tokens, or None."""
    import paper_1905_12948_amd as gmc
    R, T, V = x.shape
    logp, entropy, top_logp, top_ids, norm = got or gmc.token_scores(x, labels, top=top, temperature=tau)
    rows = host(x).reshape(R * T, V)
    table, H, spread, order = ref.scores(rows, tau, top)
    best = rows.max(-1)
    with np.errstate(invalid="ignore"):
        ls = -np.take_along_axis(table, order[:, :1] if top else table.argmax(-1)[:, None], -1)[:, 0]
    lnV = math.log(V + 1)
    within(norm[..., 0].reshape(-1), best, 0.0, "largest logit")
    within(norm[..., 1].reshape(-1), ls, (2 * ls + 123 + 3 * lnV) * U, "log of the sum")
    within(entropy.reshape(-1), H, (250 + 130 * lnV + 3 * spread) * U, "entropy")

    def tolerance(v):
        with np.errstate(invalid="ignore"):
            return (4 * np.abs(v + ls[:, None]) + 2 * ls[:, None] + 123 + 3 * lnV) * U
    if labels is None:
        assert logp is None
    else:
        want = np.take_along_axis(table, labels.cpu().numpy().reshape(-1, 1), -1)
        within(logp.reshape(-1, 1), want, tolerance(want), "log-probability")
    if top:
        assert np.array_equal(top_ids.cpu().numpy().reshape(R * T, top), order)
        want = np.take_along_axis(table, order, -1)
        within(top_logp.reshape(R * T, top), want, tolerance(want), "alternatives")
    else:
        assert top_logp is None and top_ids is None


SIZES = [(1, 1), (2, 1), (3, 2), (17, 17), (33, 32), (64, 5), (511, 20), (1000, 0), (4096, 8), (4097, 32), (4104, 0), (8191, 5),
         (16384, 3), (16391, 20), (32003, 8), (50257, 0), (50257, 20), (53248, 4), (53255, 1), (53256, 32), (65536, 0), (131073, 20)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V,top", SIZES)
def test_forward(V, top, dtype):
    g = torch.Generator(device="cuda:0").manual_seed(V + top)
    x = (3 * torch.randn(2, 3, V, device="cuda:0", generator=g)).to(TYPES[dtype])
    labels = torch.randint(0, V, (2, 3), device="cuda:0", generator=g)
    compare(x, labels, 1.0, top)
    compare(x[:1, :1], None, 0.7, top)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V", [40, 5000, 60001])
def test_orders_and_ties(V, dtype):
    """Rising, falling, equal and few-valued rows, zeros of both signs, the type's lowest values, few
    entries that are not -inf: the first of equals wins, whatever number of them there is."""
    T = TYPES[dtype]
    j = torch.arange(V, device="cuda:0")
    low = torch.finfo(T).min
    rows = [j * (8.0 / V), -j * (8.0 / V), torch.zeros(V, device="cuda:0"), (j % 3) * 1.0, (j % 2) * -0.0,
            torch.where(j % 2 == 0, -0.0, 0.0), torch.full((V,), low, device="cuda:0"), torch.where(j < V - 3, low, 1.0),
            torch.where((j % 11 == 3) & (j < 60), 1.0 * (j % 7), -math.inf), torch.where(j == V - 1, 0.5, -math.inf),
            torch.where(j == 7, 30.0, 0.0), torch.where(j >= V - 40, 2.0, 1.0)]
    x = torch.stack([r.float() for r in rows])[:, None].to(T)
    labels = torch.full((len(rows), 1), V - 1, device="cuda:0")
    for top in (1, 9, 32):
        compare(x, labels, 1.0, top)
    compare(x, None, 2.5, 0)


@pytest.mark.parametrize("V", [30, 3000, 20000, 70000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_without_scores_16(V, dtype):
    """The same in 16 bits: NaN of both signs in either place of a pair, alone and beside an infinity."""
    import paper_1905_12948_amd as gmc
    x = torch.randn(7, 1, V, device="cuda:0").to(dtype)
    x[0, 0, 6] = math.nan
    x[1, 0, 7] = -math.nan
    x[2, 0, 17], x[2, 0, 16] = math.nan, math.inf
    x[3, 0, 2] = math.inf
    x[4] = -math.inf
    x[5, 0, :V - 1] = -math.inf
    logp, entropy, top_logp, top_ids, norm = gmc.token_scores(x, torch.full((7, 1), V - 1, device="cuda:0"), top=3)
    assert torch.isnan(logp[:5]).all() and torch.isnan(entropy[:5]).all() and torch.isnan(top_logp[:5]).all()
    assert torch.isfinite(logp[5:]).all() and torch.isfinite(entropy[5:]).all() and logp[5, 0] == 0 and entropy[5, 0] == 0
    assert np.array_equal(top_ids.cpu().numpy()[:, 0], ref.scores(host(x[:, 0]), 1.0, 3)[3])


@pytest.mark.parametrize("V", [30, 3000, 20000, 70000])
def test_rows_without_scores(V):
    """NaN, +inf and nothing but -inf: NaN scores, and places all the same."""
    import paper_1905_12948_amd as gmc
    x = torch.randn(5, 1, V, device="cuda:0")
    x[0, 0, 5] = math.nan
    x[0, 0, V - 2] = -math.nan
    x[1, 0, 3] = math.inf
    x[2] = -math.inf
    x[3, 0, V // 2] = math.nan
    logp, entropy, top_logp, top_ids, norm = gmc.token_scores(x, torch.zeros(5, 1, dtype=torch.int64, device="cuda:0"), top=6)
    assert torch.isnan(logp[:4]).all() and torch.isnan(entropy[:4]).all() and torch.isnan(top_logp[:4]).all()
    assert torch.isfinite(logp[4]).all() and torch.isfinite(entropy[4]).all()
    order = ref.scores(host(x[:, 0]), 1.0, 6)[3]
    assert np.array_equal(top_ids.cpu().numpy()[:, 0], order)
    assert order[0][:2].tolist() == [5, V - 2] and order[2].tolist() == list(range(6))
    grad = gmc.token_scores_backward(x, norm, entropy=entropy, dentropy=torch.ones(5, 1, device="cuda:0"))
    assert torch.isnan(grad[:4]).all() and torch.isfinite(grad[4]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [100, 9000, 60000])
def test_ignored_tokens_and_unknown_labels(V, dtype):
    """Ignored tokens are not looked at; a label outside the vocabulary makes its log-probability NaN."""
    import paper_1905_12948_amd as gmc
    x = torch.randn(2, 4, V, device="cuda:0").to(TYPES[dtype])
    labels = torch.tensor([[3, IGNORE, V, V - 1], [IGNORE, -1, 0, IGNORE]], device="cuda:0")
    x[labels == IGNORE] = math.nan
    logp, entropy, top_logp, top_ids, norm = gmc.token_scores(x, labels, top=3)
    off, odd = labels == IGNORE, (labels == V) | (labels == -1)
    for t in (logp, entropy, top_logp, norm):
        assert (t[off] == 0).all()
    assert (top_ids[off] == -1).all() and (top_ids[~off] >= 0).all()
    assert torch.isnan(logp[odd]).all() and torch.isfinite(logp[~odd]).all()
    assert torch.isfinite(entropy).all() and torch.isfinite(top_logp).all()
    g = torch.randn(2, 4, device="cuda:0")
    dtop = torch.randn(2, 4, 3, device="cuda:0")
    g[off] = math.nan          # nor are their gradients
    dtop[off] = math.nan
    grad = gmc.token_scores_backward(x, norm, labels, dlogp=g, top_ids=top_ids, dtop=dtop)
    assert (grad[off] == 0).all() and torch.isnan(grad[odd]).all() and torch.isfinite(grad[~odd]).all()
    # without dlogp the label says only whether the token counts
    grad = gmc.token_scores_backward(x, norm, labels, top_ids=top_ids, dtop=dtop)
    assert (grad[off] == 0).all() and torch.isfinite(grad).all()
    # another number as `ignore`
    first = gmc.token_scores(x[:, 2:3], labels[:, 2:3], ignore=0)[0]
    assert first[1, 0] == 0


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V,pitch", [(7, 9), (1000, 1003), (8191, 8200), (50257, 50257), (60007, 60013)])
def test_strides(V, pitch, dtype):
    """Rows of a wider buffer, each sequence's last token left out, labels of a wider buffer, no sequence before the first byte."""
    data = torch.randn(2 * 4 * pitch + 3, device="cuda:0").to(TYPES[dtype])
    wide = data[3:].view(2, 4, pitch)
    labels = torch.randint(0, V, (2, 9), device="cuda:0")[:, 2:5]
    compare(wide[:, :3, :V], labels, 1.3, min(V, 6))
    compare(wide.transpose(0, 1)[1:2, :, :V], labels[:1, :2], 1.0, 0)


def gradient(x, tau, labels, dlogp, dentropy, ids, dtop, got):
    """The gradient against the 64-bit one."""
    R, T, V = x.shape
    rows = host(x).reshape(R * T, V)
    lab = np.full(R * T, -1) if labels is None else labels.cpu().numpy().reshape(-1)
    zero = np.zeros(R * T)
    gl, gh = (zero if t is None else host(t).reshape(-1) for t in (dlogp, dentropy))
    k = 0 if ids is None else ids.shape[2]
    at = np.zeros((R * T, 0), np.int64) if ids is None else ids.cpu().numpy().reshape(R * T, k)
    gt = np.zeros((R * T, 0)) if ids is None else host(dtop).reshape(R * T, k)
    want = ref.scores_gradient(rows, tau, lab, gl, gh, at, gt)
    table = ref.log_softmax(rows, tau)
    p, lp = np.exp(table), np.abs(np.maximum(table, -120))
    ls = np.abs(table.max(-1, keepdims=True))
    H = np.where(p > 0, p * lp, 0).sum(-1, keepdims=True)
    size = (np.abs(gl) + np.abs(gt).sum(-1))[:, None]
    steep = size + np.abs(gh)[:, None] * (lp + H)
    tol = U / tau * (p * steep * (3 * lp + 3 * ls + 16))
    # H as it was given, to the forward call's tolerance
    tol = tol + U / tau * p * np.abs(gh)[:, None] * (250 + 130 * math.log(V + 1) + 3 * H * H * 4)
    extra = np.zeros_like(want)
    for r in range(R * T):
        if lab[r] >= 0:
            extra[r, lab[r]] += abs(gl[r])
        for j, g in zip(at[r], gt[r]):
            if 0 <= j < V:
                extra[r, j] += abs(g)
    tol = tol + 40 * U / tau * extra
    name = {v: k for k, v in TYPES.items()}[x.dtype]
    rel, least = HALF[name]
    within(got.reshape(R * T, V), want, tol + rel * (np.abs(want) + tol) + least + 2.0 ** -140, "gradient")


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V,top", [(1, 1), (5, 2), (33, 32), (1000, 0), (4096, 5), (4099, 8), (8191, 5), (20000, 0), (50257, 20)])
def test_gradient(V, top, dtype):
    import paper_1905_12948_amd as gmc
    g = torch.Generator(device="cuda:0").manual_seed(7 * V + top)
    x = (3 * torch.randn(2, 2, V, device="cuda:0", generator=g)).to(TYPES[dtype])
    labels = torch.randint(0, V, (2, 2), device="cuda:0", generator=g)
    for tau in (1.0, 0.6):
        logp, H, _, ids, norm = gmc.token_scores(x, labels, top=top, temperature=tau)
        a, b = torch.randn(2, 2, device="cuda:0", generator=g), torch.randn(2, 2, device="cuda:0", generator=g)
        c = torch.randn(2, 2, top, device="cuda:0", generator=g) if top else None
        for dl, dh, dt in ((a, b, c), (a, None, None), (None, b, None), (None, None, c)):
            got = gmc.token_scores_backward(x, norm, labels, dlogp=dl, entropy=H, dentropy=dh, top_ids=None if dt is None else ids,
                                            dtop=dt, temperature=tau)
            gradient(x, tau, labels, dl, dh, None if dt is None else ids, dt, got)


def test_gradient_places_twice_and_outside():
    """A place that occurs several times, the label among them, and places outside the vocabulary."""
    import paper_1905_12948_amd as gmc
    for V in (50, 6000, 40000):
        x = torch.randn(1, 2, V, device="cuda:0")
        labels = torch.tensor([[4, V - 1]], device="cuda:0")
        ids = torch.tensor([[[4, 9, 4, -1, V, 4, 9], [V - 1, 0, V - 1, 2 ** 40, -2 ** 40, 0, 1]]], device="cuda:0")
        dt, dl = torch.randn(1, 2, 7, device="cuda:0"), torch.randn(1, 2, device="cuda:0")
        norm = gmc.token_scores(x)[4]
        got = gmc.token_scores_backward(x, norm, labels, dlogp=dl, top_ids=ids, dtop=dt)
        gradient(x, 1.0, labels, dl, None, ids, dt * ((ids >= 0) & (ids < V)), got)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("V", [100, 4100, 50257])
def test_gradient_over_the_logits(V, dtype):
    """In place, and into rows that lie differently."""
    import paper_1905_12948_amd as gmc
    x = torch.randn(3, 2, V, device="cuda:0").to(TYPES[dtype])
    labels = torch.randint(0, V, (3, 2), device="cuda:0")
    logp, H, _, ids, norm = gmc.token_scores(x, labels, top=4)
    how = dict(dlogp=torch.randn(3, 2, device="cuda:0"), entropy=H, dentropy=torch.randn(3, 2, device="cuda:0"), top_ids=ids,
               dtop=torch.randn(3, 2, 4, device="cuda:0"))
    want = gmc.token_scores_backward(x, norm, labels, **how)
    wide = torch.full((3, 2, V + 5), 7.0, device="cuda:0", dtype=x.dtype)
    gmc.token_scores_backward(x, norm, labels, out=wide[:, :, 3:V + 3], **how)
    assert torch.equal(wide[:, :, 3:V + 3], want)
    assert (wide[:, :, :3] == 7).all() and (wide[:, :, V + 3:] == 7).all()
    assert gmc.token_scores_backward(x, norm, labels, out=x, **how) is x
    assert torch.equal(x, want)


def test_gradient_against_differences():
    """Along random directions the scores change as the gradient says: central differences of
    64-bit scores with step h are off by h^2 / 6 of the third derivative, below |v|^3 (1 + H) h^2."""
    import paper_1905_12948_amd as gmc
    V, tau = 300, 0.9
    x = torch.randn(1, 1, V, device="cuda:0")
    labels = torch.tensor([[11]], device="cuda:0")
    logp, H, _, ids, norm = gmc.token_scores(x, labels, top=3, temperature=tau)
    dl, dh, dt = 0.7, -1.3, np.array([0.2, -0.5, 0.9])
    one = torch.ones(1, 1, device="cuda:0")
    got = host(gmc.token_scores_backward(x, norm, labels, dlogp=dl * one, entropy=H, dentropy=dh * one, top_ids=ids,
                                         dtop=torch.as_tensor(dt, dtype=torch.float32, device="cuda:0").view(1, 1, 3), temperature=tau))[0, 0]
    row, at = host(x)[0, 0], ids.cpu().numpy()[0, 0]

    def value(r):
        t = ref.log_softmax(r, tau)
        return dl * t[11] + dh * -(np.exp(t) * t).sum() + (dt * t[at]).sum()
    rng = np.random.default_rng(3)
    h = 1e-4
    for _ in range(20):
        v = rng.normal(size=V)
        slope = (value(row + h * v) - value(row - h * v)) / (2 * h)
        assert abs(slope - got @ v) < 1e-4 * np.linalg.norm(v)


def test_peaked_and_far_rows():
    """Nearly certain tokens, logits far from zero and far apart."""
    V = 2000
    base = torch.randn(V, device="cuda:0")
    rows = []
    for far, gap in ((0.0, 12.0), (1e4, 0.0), (-3e4, 5.0), (3e38, 0.0), (0.0, 200.0)):
        r = base + far if far < 1e38 else torch.full((V,), far, device="cuda:0")
        r[77] = r.max() + gap if gap else r[77]
        rows.append(r)
    rows.append(base * 1e5)
    compare(torch.stack(rows)[:, None], torch.full((len(rows), 1), 77, device="cuda:0"), 1.0, 5)


def test_far_offsets():
    """Rows that begin more than 2^32 bytes from the first."""
    import paper_1905_12948_amd as gmc
    V, far = 300, (1 << 31) + 77
    data = torch.zeros(far + 2 * V, device="cuda:0", dtype=torch.bfloat16)
    x = torch.as_strided(data, (2, 2, V), (far, V, 1))
    x.copy_(torch.randn(2, 2, V, device="cuda:0").to(torch.bfloat16))
    labels = torch.randint(0, V, (2, 2), device="cuda:0")
    got = gmc.token_scores(x, labels, top=3)
    for a, b in zip(got, gmc.token_scores(x.contiguous(), labels, top=3)):
        within(a, host(b), 200 * U * (1 + np.abs(host(b))), "far rows")
    assert torch.equal(got[3], gmc.token_scores(x.contiguous(), labels, top=3)[3])
    how = dict(dlogp=torch.randn(2, 2, device="cuda:0"))
    want = gmc.token_scores_backward(x.contiguous(), got[4], labels, **how)
    gmc.token_scores_backward(x, got[4], labels, out=x, **how)
    assert torch.equal(x, want)


@pytest.mark.parametrize("V", [700, 30000, 90000])
def test_same_bits_streams_and_graphs(V):
    """The same call gives the same bits, on a side stream and in a graph that is replayed with
    other logits between eager calls."""
    import paper_1905_12948_amd as gmc
    x = torch.randn(2, 3, V, device="cuda:0")
    labels = torch.randint(0, V, (2, 3), device="cuda:0")
    dl = torch.randn(2, 3, device="cuda:0")

    def run():
        logp, H, top_logp, ids, norm = gmc.token_scores(x, labels, top=7)
        return logp, H, top_logp, ids, norm, gmc.token_scores_backward(x, norm, labels, dlogp=dl, entropy=H, dentropy=dl,
                                                                       top_ids=ids, dtop=top_logp)
    want = run()
    assert all(torch.equal(a, b) for a, b in zip(run(), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(other, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for k in range(4):
        x.copy_(torch.randn(2, 3, V, device="cuda:0"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, run()))


@pytest.mark.parametrize("dtype,V,R", [("f32", 1_000_003, 1), ("bf16", 700_001, 2), ("f32", 200_000, 300)])
def test_long_vocabularies(dtype, V, R):
    """Rows in many pieces, whose keys the joining launch looks at in several turns; equal logits among them."""
    g = torch.Generator(device="cuda:0").manual_seed(V)
    x = (2 * torch.randn(R, 1, V, device="cuda:0", generator=g)).to(TYPES[dtype])
    x[0, 0] = (x[0, 0] * 2).round() / 2
    labels = torch.randint(0, V, (R, 1), device="cuda:0", generator=g)
    if R > 8:
        import paper_1905_12948_amd as gmc
        got = [None if t is None else t[:8] for t in gmc.token_scores(x, labels, top=32)]
        compare(x[:8], labels[:8], 1.0, 32, got)
    else:
        compare(x, labels, 1.0, 32)
        x[0] = 1.5
        compare(x, labels, 1.0, 32)


def test_no_tokens_and_refusals():
    import paper_1905_12948_amd as gmc
    x = torch.randn(2, 3, 50, device="cuda:0")
    labels = torch.zeros(2, 3, dtype=torch.int64, device="cuda:0")
    for shape in ((0, 3, 50), (2, 0, 50)):
        got = gmc.token_scores(x.new_empty(shape), top=2)
        assert got[1].shape == shape[:2] and got[3].shape == shape[:2] + (2,)
        assert gmc.token_scores_backward(x.new_empty(shape), got[4]).shape == shape
    norm = gmc.token_scores(x)[4]
    for bad, error in ((lambda: gmc.token_scores(x[0]), ValueError), (lambda: gmc.token_scores(x.double()), TypeError),
                       (lambda: gmc.token_scores(x.cpu()), ValueError), (lambda: gmc.token_scores(x, labels.int()), TypeError),
                       (lambda: gmc.token_scores(x, labels[:1]), ValueError), (lambda: gmc.token_scores(x, top=33), RuntimeError),
                       (lambda: gmc.token_scores(x, top=-1), RuntimeError), (lambda: gmc.token_scores(x, top=2 ** 33), ValueError),
                       (lambda: gmc.token_scores(x, temperature=0.0), RuntimeError),
                       (lambda: gmc.token_scores(x, labels, ignore=2 ** 63), ValueError),
                       (lambda: gmc.token_scores(x.transpose(1, 2)), ValueError),
                       (lambda: gmc.token_scores_backward(x, norm[..., :1], labels), ValueError),
                       (lambda: gmc.token_scores_backward(x, norm, dlogp=norm[..., 0].contiguous()), RuntimeError),
                       (lambda: gmc.token_scores_backward(x, norm, labels, dentropy=norm[..., 0].contiguous()), ValueError),
                       (lambda: gmc.token_scores_backward(x, norm, labels, dtop=norm), ValueError),
                       (lambda: gmc.token_scores_backward(x, None, labels), RuntimeError),
                       (lambda: gmc.token_scores_backward(x, norm, labels, out=x.half()), TypeError)):
        with pytest.raises(error):
            bad()
    # the losses still need labels
    with pytest.raises(TypeError):
        gmc.policy_loss(x, None, None, torch.zeros(2, device="cuda:0"))
