"""Sequences without rows whose start lies at another's, inside it, or behind it: lengths decide, they hide nothing."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_seq_attn import BF, FP, Batch  # noqa: E402

pytestmark = pytest.mark.gpu

CASES = [
    # starts and lengths of queries; of keys (None: the same), rows in memory
    ([0, 0, 40, 40, 40, 90], [40, 0, 0, 50, 0, 10], None, None, 100),
    ([0, 20, 40, 45], [40, 0, 10, -3], None, None, 60),
    ([0, 0], [5, 0], None, None, 5),
    ([0, 0, 0, 0, 300], [300, 0, 0, -1, 0], None, None, 300),
    # empty queries, empty keys and both, keys of the empty ones beside rows of others
    ([0, 10, 10, 80, 80], [10, 0, 70, 0, 0], [0, 30, 30, 30, 200], [30, 0, 150, 0, 20], 220),
    ([0, 50, 60], [60, 0, 0], [0, 90, 200], [120, 0, 0], 220),
]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_at,qn,k_at,kn,rows", CASES)
def test_empty_sequences(q_at, qn, k_at, kn, rows, causal, d, dtype):
    q_rows = max(a + max(n, 0) for a, n in zip(q_at, qn)) + 9
    b = Batch(q_at, k_at or q_at, 2, 1, d, dtype, causal, q_len=qn, k_len=kn or qn, q_rows=q_rows, k_rows=rows + 9, seed=3)
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("used,room", [(5, 64), (9, 10), (3, 1000), (7, 3000), (0, 50), (1, 9)])
def test_a_batch_with_room(used, room):
    """Few of many sequences in use, the others of length 0 behind the last row, at row 0, or anywhere; rows behind them."""
    n = [(17 * i) % 60 + 1 for i in range(used)]
    at = [sum(n[:i]) for i in range(used)]
    T = sum(n)
    for rest in ([T] * (room - used), [T + i // 40 for i in range(room - used)]):
        b = Batch(at + rest, at + rest, 2, 1, 64, BF, True, q_len=n + [0] * (room - used), k_len=n + [0] * (room - used), q_rows=T + 300, k_rows=T + 300, seed=5)
        b.forward()
        b.check_forward()
        b.backward()
        b.check_backward()
    if used:  # in front of all, and between
        at2, n2 = [0] * 8 + at, [0] * 8 + n
        at2[9:9], n2[9:9] = [at2[8]] * 11, [0] * 11
        b = Batch(at2, at2, 2, 1, 128, FP, False, q_len=n2, k_len=n2, q_rows=T + 300, k_rows=T + 300, seed=6)
        b.forward()
        b.check_forward()
        b.backward()
        b.check_backward()


@pytest.mark.parametrize("where", ["at", "inside", "many"])
def test_among_many(where):
    """The same where more sequences are searched than shared memory holds, and in runs of hundreds without rows."""
    at, n, row = [], [], 0
    for i in range(60):
        m = 1 + (37 * i) % 90
        at.append(row)
        n.append(m)
        for j in range(30 if where != "many" else 200 if i % 10 == 0 else 0):
            at.append(row if where == "at" else row + min(m - 1, j))
            n.append(0)
        row += m
    at, n = [list(x) for x in zip(*sorted(zip(at, range(len(n)), n)))][::2]
    b = Batch(at, at, 2, 2, 64, BF, True, q_len=n, k_len=n, q_rows=row, k_rows=row, seed=4)
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()
