"""How many bits the orthogonalised matrices keep (gmc_orthogonalize): held to the error of the same steps
with products in 32 bits, also where rows or columns are of very different sizes, and row by row to
a model of what is kept.

The model, in 64 bits: of every kept value v (X and its products with itself in units of 1, the polynomial in units of
8) an error of up to 2^-21 of v, or 2^-48 of the unit where that is more (two f16 halves, the lower one times 2^11:
2^-22 of v, and no finer than half a step of the smallest f16 number, 2^-25, at scales of 2^24 and 2^21; the
products leave out as much again); and of every entry of a product an error of up to 2^-21 of the norms of its row and
column (sums in 32 bits, 16 terms at a time, three products: for 300 terms 57 roundings, each
2^-24 of a partial sum that the norms bound, of independent signs: sqrt(57) 2^-24 < 2^-21).
Rows of the result may be off by four times the largest distance of eight such runs.

Against 32-bit products: four times their own error in the Frobenius norm, and of single rows and columns
four times their largest relative error, as long as the entries are above 2^-28 of the norm: 2^-49 is then no more
than 2^-21 of them, what the model allows for every value (an entry of 2^-28 is not the limit of what is
exact but of what this test compares)."""
import numpy as np
import pytest

import scores_ref as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def in_32_bits(x):
    """The steps with torch's products of 32-bit matrices."""
    x = x if x.shape[0] <= x.shape[1] else x.T
    x = x / (x.double().norm().float() + 1e-7)
    a, b, c = ref.QUINTIC
    for _ in range(5):
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x


def ours(m):
    import paper_1905_12948_amd as gmc
    rows, cols = m.shape
    plan = gmc.Matrices(rows * cols, [(0, rows, cols)])
    return gmc.orthogonalize(plan, m.reshape(-1)).view(rows, cols)


def entries(rows, cols, seed):
    rng = np.random.default_rng(seed)
    rank = min(6, rows // 2, cols // 2)
    return rng.normal(size=(rows, rank)) @ rng.normal(size=(rank, cols)) + rng.normal(size=(rows, cols))


# sizes of rows (or columns): as they are, falling by powers of ten, a few small ones among many
SIZES = {"even": lambda n: np.ones(n), "falling": lambda n: 10.0 ** (-7 * np.arange(n) / max(1, n - 1)),
         "some": lambda n: np.where(np.arange(n) % 8 == 3, 10.0 ** -(3 + np.arange(n) % 5), 1.0)}


def matrix(rows, cols, sizes, along):
    m = entries(rows, cols, rows + cols)
    s = SIZES[sizes](rows if along == "rows" else cols)
    return torch.as_tensor(m * (s[:, None] if along == "rows" else s[None, :]), dtype=torch.float32).cuda()


@pytest.mark.parametrize("along", ["rows", "columns"])
@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("rows,cols", [(64, 147), (100, 300), (128, 192), (256, 256), (700, 96), (384, 384), (300, 1100)])
def test_as_near_as_products_in_32_bits(rows, cols, sizes, along):
    m = matrix(rows, cols, sizes, along)
    exact = ref.polar(m.double().cpu().numpy())
    plain = in_32_bits(m).double().cpu().numpy()
    theirs = np.linalg.norm((plain if rows <= cols else plain.T) - exact)
    mine = np.linalg.norm(ours(m).double().cpu().numpy() - exact)
    print("error / 32 bits' error %.2f, relative %.2e" % (mine / theirs, mine / np.linalg.norm(exact)), flush=True)
    assert mine <= 4 * theirs


def model(x, rng):
    """The steps on a wide matrix with the errors of the docstring."""
    def keep(v, unit):
        return v + rng.uniform(-1, 1, v.shape) * np.maximum(2.0 ** -21 * np.abs(v), 2.0 ** -48 * unit)

    def product(p, q):
        return p @ q + rng.uniform(-1, 1, (p.shape[0], q.shape[1])) * 2.0 ** -21 * np.outer(
            np.linalg.norm(p, axis=1), np.linalg.norm(q, axis=0))
    a, b, c = ref.QUINTIC
    x = keep(x / (np.linalg.norm(x) + 1e-7), 1.0)
    for _ in range(5):
        gram = keep(product(x, x.T), 1.0)
        poly = keep(a * np.eye(len(x)) + b * gram + c * product(gram, gram), 8.0)
        x = keep(product(poly, x), 1.0)
    return x


@pytest.mark.parametrize("sizes", ["falling", "some"])
@pytest.mark.parametrize("rows,cols,along", [(64, 147, "rows"), (128, 192, "rows"), (200, 300, "rows"), (96, 300, "columns"), (300, 200, "columns")])
def test_rows_of_different_sizes(rows, cols, sizes, along):
    m = matrix(rows, cols, sizes, along)
    got = ours(m).double().cpu().numpy()
    x = m.double().cpu().numpy()
    if rows > cols:
        x, got = x.T, got.T
    exact, rng = ref.polar(x), np.random.default_rng(1)
    runs = [model(x, rng) for _ in range(8)]
    for axis in (1, 0):
        tol = 4 * np.max([np.linalg.norm(v - exact, axis=axis) for v in runs], axis=0) + 4 * U * np.linalg.norm(exact, axis=axis)
        off = np.linalg.norm(got - exact, axis=axis)
        print("axis %d: worst share of its bound %.2f, worst relative error %.1e" % (
            axis, (off / tol).max(), (off / np.linalg.norm(exact, axis=axis)).max()), flush=True)
        assert (off <= tol).all()


@pytest.mark.parametrize("along", ["rows", "columns"])
@pytest.mark.parametrize("size", [1e-2, 1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("rows,cols", [(64, 147), (128, 256), (300, 300), (300, 128), (1000, 1100)])
def test_small_rows_as_exact_as_with_products_in_32_bits(rows, cols, size, along):
    m = entries(rows, cols, 7)
    n = rows if along == "rows" else cols
    small = np.arange(n) % 8 == 3
    s = np.where(small, size, 1.0)
    x = torch.as_tensor(m * (s[:, None] if along == "rows" else s[None, :]), dtype=torch.float32).cuda()
    exact = ref.polar(x.double().cpu().numpy())
    assert size * np.abs(m).mean() > 2.0 ** -28 * np.linalg.norm(m)
    axis = 1 if along == "rows" else 0

    def worst(v):
        v = v.double().cpu().numpy()
        v = v if v.shape == exact.shape else v.T
        return (np.linalg.norm(v - exact, axis=axis) / np.linalg.norm(exact, axis=axis))[small].max()
    mine, theirs = worst(ours(x)), worst(in_32_bits(x))
    print("worst relative error %.1e, with products in 32 bits %.1e" % (mine, theirs), flush=True)
    assert mine <= 4 * theirs
