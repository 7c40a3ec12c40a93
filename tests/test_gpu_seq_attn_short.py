"""Gradients of short sequences, whatever else is in the batch: beside long sequences, in padded batches, and where clusters
share walks they are as near the true ones as those of short sequences alone."""
import pytest

torch = pytest.importorskip("torch")
from seq_plain import check  # noqa: E402
from test_gpu_seq_attn import BF, FP, Batch, starts  # noqa: E402

pytestmark = pytest.mark.gpu


def near(b, short):
    """dq, dk and dv of the sequences in `short`: each held to its rounding as in test_gradients_of_few_keys, whose bound is
    0.7 half steps of the norm (0.56 expected: two roundings; 0.8 with D from the rounded o)."""
    b.forward()
    b.backward()
    b.check_forward()
    b.check_backward()
    case = b.case()
    for name, got, (want, _), keys in zip(("dq", "dk", "dv"), (b.dq, b.dk, b.dv), case.backward(b.g, b.o), (False, True, True)):
        rows = torch.zeros(want.shape[0], dtype=torch.bool)
        for i in short:
            q0, q1, k0, k1 = case.seqs[i]
            rows[slice(k0, k1) if keys else slice(q0, q1)] = True
        x, y = got.cpu().double()[rows], want[rows]
        far = float((x - y).norm() / y.norm())
        assert far <= 0.7 * torch.finfo(b.dtype).eps / 2, (name, far)


MIXED = [
    # lengths of queries, of keys (None: the same), the short ones among them, causal
    ([2, 3] * 16 + [2200], None, range(32), True),
    ([900] + [3, 2] * 20 + [1300], None, range(1, 41), True),
    ([2, 3, 2] * 15 + [1500], [2, 3, 2] * 15 + [2000], range(45), False),
    ([50, 30, 40, 60, 300], [3, 2, 2, 3, 4000], range(4), False),
    # few tiles and a long walk: clusters share it
    ([2, 3] * 10 + [3000], None, range(20), True),
    ([3, 2] * 10 + [40], [2, 3] * 10 + [6000], range(20), False),
]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 40, 128])
@pytest.mark.parametrize("qn,kn,short,causal", MIXED)
def test_beside_long_sequences(qn, kn, short, causal, d, dtype):
    heads = 1 if max(qn) == 3000 or kn and max(kn) == 6000 else 2
    near(Batch(starts(qn), starts(kn or qn), 2 * heads, heads, d, dtype, causal, seed=3), short)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_in_a_padded_batch(causal, d, dtype):
    """Sequences of 2 and 3 rows in slots of 160, packed queries against keys in slots, and a long one among them."""
    for n, cap, packed in [([2, 3] * 24, 160, False), ([2, 3] * 24, 160, True), ([2, 3] * 12 + [700] + [3, 2] * 12, 704, False)]:
        at = [cap * i for i in range(len(n))]
        q_at = starts(n) if packed else at
        b = Batch(q_at, at, 4, 2, d, dtype, causal, q_len=n, k_len=n, q_rows=sum(n) if packed else cap * len(n), k_rows=cap * len(n), seed=5)
        near(b, [i for i, m in enumerate(n) if m < 4])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
def test_the_same_alone_and_in_company(d, dtype):
    """A short sequence's dq does not depend on its neighbours: the same operands alone and in front of a long sequence
    give the same within the roundings of sums that are taken in another order (2^-20 of the largest before the result's
    rounding, so one step of the type at most)."""
    n = [2, 3, 5] * 10
    alone = Batch(starts(n), starts(n), 2, 2, d, dtype, True, seed=7)
    mixed = Batch(starts(n + [1900]), starts(n + [1900]), 2, 2, d, dtype, True, seed=8)
    for x, y in ((alone.q, mixed.q), (alone.k, mixed.k), (alone.v, mixed.v), (alone.g, mixed.g)):
        y[:x.shape[0]].copy_(x)
    for b in (alone, mixed):
        b.forward()
        b.backward()
    torch.cuda.synchronize()
    for x, y in ((alone.dq, mixed.dq), (alone.dk, mixed.dk), (alone.dv, mixed.dv)):
        y = y[:x.shape[0]]
        step = torch.finfo(dtype).eps * torch.maximum(x.abs(), y.abs()).double() + float(x.abs().max()) * 2.0 ** -20
        assert bool(((x.double() - y.double()).abs() <= step).all())


def test_first_rows_of_whole_tiles():
    """Short sequences whose keys fill several tiles in front of, between and behind long ones, with empty ones among them."""
    n = [1, 0, 2] * 60 + [400] + [12, 0, 1, 31, 7] * 12 + [350] + [5] * 30
    for d in (64, 128):
        b = Batch(starts(n), starts(n), 2, 1, d, BF, True, seed=9)
        near(b, [i for i, m in enumerate(n) if 2 <= m < 20])
    check("lse", b.lse, *[b.case().forward()[i] for i in (1, 3)])
