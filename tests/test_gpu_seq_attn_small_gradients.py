"""fp16 gradients of attention for output gradients of any size that fp16 holds: as near the formula's as the roundings of P and dS
relative to themselves, and of the results, allow."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_seq_attn import FP, Batch, starts  # noqa: E402

pytestmark = pytest.mark.gpu


def hold(b, rows=None, what=("dq", "dk", "dv")):
    """0.7 half steps of a result's norm for what is rounded relative to itself (the result, and P or dS over hundreds of terms: 0.56
    expected, as in test_gradients_of_few_keys); and the multiples of 2^-24 that the result is rounded to below 2^-14: a
    step over sqrt 12 for each element, 1.1 times as room for the spread of a sum of many squares."""
    torch.cuda.synchronize()
    assert int(b.status) == 0
    for name, got, (want, _) in zip(("dq", "dk", "dv"), (b.dq, b.dk, b.dv), b.case().backward(b.g, b.o)):
        if name not in what:
            continue
        x, y = (t if rows is None else t[rows] for t in (got.cpu().double(), want))
        live = ~torch.isnan(y)
        far, norm, n = float((x - y)[live].norm()), float(y[live].norm()), int(live.sum())
        assert far <= 0.7 * 2.0 ** -11 * norm + 1.1 * 2.0 ** -24 / 12 ** 0.5 * n ** 0.5, (name, far / norm, n)


def run(b):
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    b.check_guards()


@pytest.mark.parametrize("size", [300.0, 30.0, 1.0, 1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("d,hq,hkv", [(64, 2, 2), (64, 4, 1), (40, 2, 1), (128, 2, 1), (128, 1, 1)])
@pytest.mark.parametrize("causal", [False, True])
def test_sizes_of_g(size, d, hq, hkv, causal):
    for lens in ([2048], [300, 77, 500], [128] * 5):
        b = Batch(starts(lens), starts(lens), hq, hkv, d, FP, causal, seed=3)
        b.g.mul_(size)
        run(b)
        hold(b)


@pytest.mark.parametrize("d", [64, 128])
def test_few_tiles_and_long_walks(d):
    """Clusters share the walks, some of whose CTAs may have no step."""
    for qn, kn in [([17], [4500]), ([3000, 5], [90, 40]), ([200], [5000]), ([2500], [2]), ([1, 1500], [1500, 1])]:
        b = Batch(starts(qn), starts(kn), 2, 1, d, FP, False, seed=4)
        b.g.mul_(1e-3)
        run(b)
        hold(b)


@pytest.mark.parametrize("d", [64, 128])
def test_unlike_rows_and_sequences(d):
    """Rows of g that differ by powers of ten, sequences alike; zeros, rows outside the sequences that are huge or no numbers.
    dq goes by its own row, dk by the walk's largest: both hold for a sequence whose g is a thousandth of its neighbour's."""
    n = [200, 150, 300, 60]
    at = [10, 240, 400, 720]
    b = Batch(at, at, 2, 1, d, FP, True, q_len=n, k_len=n, q_rows=800, k_rows=800, seed=6)
    b.g.mul_(10.0 ** (torch.arange(800, device="cuda") % 3 - 2.0)[:, None, None])
    b.g[240:390] *= 1e-3
    b.g[400:410] = 0
    outside = torch.ones(800, dtype=torch.bool)
    for s, m in zip(at, n):
        outside[s:s + m] = False
    for x in (b.q, b.k, b.v):
        x[outside.cuda()] = torch.nan
    b.g[outside.cuda()] = 60000.0
    b.g[-1] = torch.inf
    b.forward()
    b.o[outside.cuda()] = torch.nan
    b.backward()
    torch.cuda.synchronize()
    for x in (b.q, b.k, b.v, b.g, b.o):
        x[outside.cuda()] = 0
    for s, m in zip(at, n):
        hold(b, slice(s, s + m))


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("size", [1.0, 30.0, 1000.0])
def test_small_dS_of_large_gradients(size, d):
    """Every element within the plain form's bounds, in which dS is rounded by 2^-25 at most where it is small, whatever the size of
    g: sentences beside long sequences, whose last queries leave little of dS for the first keys."""
    lens = [23, 294, 3, 21, 30, 6, 285, 192, 1]
    b = Batch(starts(lens), starts(lens), 1, 1, d, FP, True, seed=20, spread=2.0)
    b.g.mul_(size)
    run(b)
    b.check_forward()
    b.check_backward()


@pytest.mark.parametrize("d", [64, 128])
def test_what_does_not_fit_is_computed_again(d):
    """dP far above what the size of g lets expect (values of 2000, g along them: dP of 64 x 2000 x 2, a quarter of which
    and its power are 128000): dS times its power is infinite for some rows."""
    b = Batch([0, 300], [0, 300], 1, 1, d, FP, True, seed=7)
    b.v.mul_(2000.0)
    b.g[100:] = b.v[100:] / 1000.0
    b.g[:100].mul_(0.01)
    run(b)
    b.check_backward()


def test_workspace():
    """Larger than bf16's by the largest |g| of every 32 rows; not written behind (check_guards)."""
    for n in (1, 31, 32, 33, 1000):
        b = Batch([0, n], [0, n], 3, 1, 64, FP, True, seed=8)
        run(b)
        hold(b, what=("dv",))


def test_weak_keys():
    """dv of keys whose weights are all far below 2^-14: relative to their own values.  The weights are all alike, so their
    rounding is off by up to half a step, 2^-11, in all of them at once; results are below 2^-14 and rounded to multiples of
    2^-24."""
    n, d = 4096, 64
    b = Batch([0, 128], [0, n], 2, 1, d, FP, False, scale=1.0, seed=9)
    b.q.zero_()
    b.q[:, :, 0] = 1.0
    b.k.zero_()
    b.k[0, 0, 0] = 13.0  # 18.8 powers of two above the others
    run(b)
    torch.cuda.synchronize()
    want = b.case().backward(b.g, b.o)[2][0][1:]
    far, norm = float((b.dv.cpu().double()[1:] - want).norm()), float(want.norm())
    assert far <= 1.01 * 2.0 ** -11 * norm + 1.1 * 2.0 ** -24 / 12 ** 0.5 * want.numel() ** 0.5, far / norm
