"""Attention over sequences against its 64-bit plain form (tests/seq_plain.py), whose bounds were written first."""
import pytest

torch = pytest.importorskip("torch")
from paper_2306_04235_gb300 import mnmt  # noqa: E402
from seq_plain import Case, check  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {torch.bfloat16: mnmt.BF16, torch.float16: mnmt.F16}
BF, FP = torch.bfloat16, torch.float16
SENTINEL = 77.0


def starts(lens):
    s = [0]
    for n in lens:
        s.append(s[-1] + n)
    return s


def dev(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


class Batch:
    """Operands of a batch on the GPU and their calls; layout: "rows" [T][H][d], "fused" one buffer for q, k and v, "heads"
    [H][T][d], "wide" rows and heads with room between them."""

    def __init__(self, q_start, k_start, hq, hkv, d, dtype, causal=False, q_len=None, k_len=None, q_rows=None, k_rows=None, layout="rows", seed=0,
                 scale=None, spread=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.n = len(q_start) - 1 if q_len is None else len(q_len)
        self.lists = (q_start, k_start, q_len, k_len)
        Tq, Tk = q_rows if q_rows is not None else q_start[-1], k_rows if k_rows is not None else k_start[-1]
        self.scale = scale if scale is not None else d ** -0.5
        self.causal, self.dtype, self.hq, self.hkv, self.d = causal, dtype, hq, hkv, d

        def make(rows, heads, fill=True):
            if layout == "heads":
                x = torch.full((heads, max(rows, 1), d), SENTINEL, device="cuda").to(dtype).transpose(0, 1)
            elif layout == "wide":
                x = torch.full((max(rows, 1) + 1, heads + 1, d + 8), SENTINEL, device="cuda").to(dtype)[:, :heads, :d]
            else:
                x = torch.full((max(rows, 1), heads, d), SENTINEL, device="cuda").to(dtype)
            x = x[:rows]
            if fill:
                x.copy_(torch.randn((rows, heads, d), generator=g, device="cuda") * spread)
            return x

        if layout == "fused":
            x = torch.randn((Tq, hq + 2 * hkv, d), generator=g, device="cuda").to(dtype)
            self.q, self.k, self.v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
        else:
            self.q, self.k, self.v = make(Tq, hq), make(Tk, hkv), make(Tk, hkv)
        self.o, self.g = make(Tq, hq, False), make(Tq, hq)
        self.dq, self.dk, self.dv = make(Tq, hq, False), make(Tk, hkv, False), make(Tk, hkv, False)
        self.lse = torch.full((hq, Tq), SENTINEL, device="cuda")
        self.arrays = [dev(x) for x in self.lists]
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def shape(self):
        qs, ks, ql, kl = self.arrays
        return mnmt.AttentionShape(self.n, self.q.shape[0], self.k.shape[0], self.hq, self.hkv, self.d, TYPES[self.dtype], self.causal, self.scale, qs, ks,
                                   ql, kl)

    def scratch(self, size):
        """A workspace full of NaN, with a guard behind it."""
        ws = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        self.guards = getattr(self, "guards", []) + [(ws, size)]
        return ws

    def forward(self, stream=None, lse=True):
        s = self.shape()
        ws = self.scratch(mnmt.mnmt_attention_forward_workspace(s))
        mnmt.mnmt_attention_forward(s, mnmt.heads(self.q), mnmt.heads(self.k), mnmt.heads(self.v), mnmt.heads(self.o), self.lse if lse else None, ws,
                                    self.status, stream)

    def backward(self, stream=None):
        s = self.shape()
        ws = self.scratch(mnmt.mnmt_attention_backward_workspace(s))
        H = mnmt.heads
        mnmt.mnmt_attention_backward(s, H(self.q), H(self.k), H(self.v), H(self.o), self.lse, H(self.g), H(self.dq), H(self.dk), H(self.dv), ws, self.status,
                                     stream)

    def token(self, stream=None):
        s = self.shape()
        ws = self.scratch(mnmt.mnmt_attention_token_workspace(s))
        mnmt.mnmt_attention_token(s, mnmt.heads(self.q), mnmt.heads(self.k), mnmt.heads(self.v), mnmt.heads(self.o), self.lse, ws, self.status, stream)

    def case(self):
        qs, ks, ql, kl = self.lists
        return Case(self.q, self.k, self.v, self.scale, self.causal, qs, ks, ql, kl, self.n)

    def check_forward(self):
        torch.cuda.synchronize()
        assert int(self.status) == 0
        o, lse, bo, bl = self.case().forward()
        check("o", self.o, o, bo)
        check("lse", self.lse, lse, bl)
        alone = torch.isnan(o)
        assert bool((self.o.cpu().double()[alone] == float(torch.tensor(SENTINEL).to(self.dtype))).all()), "rows of no sequence were written"
        assert bool((self.lse.cpu()[torch.isnan(lse)] == SENTINEL).all())
        self.check_guards()

    def check_backward(self):
        torch.cuda.synchronize()
        assert int(self.status) == 0
        for name, got, (want, bound) in zip(("dq", "dk", "dv"), (self.dq, self.dk, self.dv), self.case().backward(self.g, self.o)):
            check(name, got, want, bound)
            alone = torch.isnan(want)
            assert bool((got.cpu().double()[alone] == float(torch.tensor(SENTINEL).to(self.dtype))).all()), f"{name}: rows of no sequence were written"
        self.check_guards()

    def check_guards(self):
        for ws, size in self.guards:
            assert bool((ws[size:] == 0xFF).all()), "written behind the workspace"


SIZES = [
    # lengths of queries, of keys (None: the same), query heads, key heads, head size, type, causal, layout
    ([1], None, 1, 1, 64, BF, True, "rows"),
    ([46], None, 4, 4, 64, BF, True, "fused"),
    ([128], None, 2, 2, 64, BF, False, "rows"),
    ([129], None, 2, 1, 64, FP, True, "rows"),
    ([127, 1, 128, 0, 130], None, 2, 2, 64, BF, True, "fused"),
    ([20, 31, 128, 64, 7, 99], None, 4, 4, 64, FP, False, "rows"),
    ([5, 0, 200, 33], [40, 17, 0, 300], 3, 1, 64, BF, False, "rows"),
    ([5, 60, 200, 33], [40, 17, 90, 300], 2, 2, 64, BF, True, "rows"),
    ([300, 77], [10, 200], 4, 2, 128, BF, True, "rows"),
    ([513], None, 4, 1, 128, BF, True, "fused"),
    ([700, 400], None, 2, 2, 128, FP, False, "fused"),
    ([257, 255], None, 6, 2, 32, BF, True, "rows"),
    ([90, 301], None, 2, 1, 96, BF, True, "heads"),
    ([333], [1], 2, 2, 8, FP, False, "rows"),
    ([1], [999], 8, 2, 40, BF, True, "wide"),
    ([100, 156, 256], None, 2, 1, 120, FP, True, "wide"),
    ([2] * 200, None, 2, 2, 64, BF, True, "rows"),
    ([1000], None, 2, 2, 64, BF, True, "rows"),
    ([640], [1400], 2, 1, 128, BF, False, "rows"),
    # few rows beside many keys: the walks are shared by clusters
    ([17], [4500], 3, 1, 64, BF, True, "rows"),
    ([200], [5000], 2, 1, 128, FP, False, "rows"),
    ([1], [2500], 2, 2, 128, BF, False, "wide"),
    ([3000], [2], 2, 2, 64, BF, True, "rows"),
    ([1500, 10], [1500, 2200], 1, 1, 40, BF, True, "heads"),
    ([2100], None, 1, 1, 64, FP, True, "fused"),
]


def batch(qn, kn, hq, hkv, d, dtype, causal, layout, **kw):
    return Batch(starts(qn), starts(kn if kn is not None else qn), hq, hkv, d, dtype, causal, layout=layout, **kw)


@pytest.mark.parametrize("qn,kn,hq,hkv,d,dtype,causal,layout", SIZES)
def test_forward(qn, kn, hq, hkv, d, dtype, causal, layout):
    b = batch(qn, kn, hq, hkv, d, dtype, causal, layout)
    b.forward()
    b.check_forward()


@pytest.mark.parametrize("qn,kn,hq,hkv,d,dtype,causal,layout", SIZES)
def test_backward(qn, kn, hq, hkv, d, dtype, causal, layout):
    b = batch(qn, kn, hq, hkv, d, dtype, causal, layout, seed=3)
    b.forward()
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("spread,scale", [(8.0, 0.125), (0.01, 0.125), (1.0, 4.0), (1.0, 1e-6)])
@pytest.mark.parametrize("d", [64, 128])
def test_sharp_and_flat(spread, scale, d):
    """Weights that are nearly one-hot (the running maximum moves far, and late rows underflow), and nearly equal ones."""
    b = batch([333, 50], None, 2, 1, d, BF, True, "rows", spread=spread, scale=scale)
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("step", [0.3, 40.0, -40.0])
def test_scores_that_rise_or_fall(step):
    """Scores that grow by `step` a key: each tile of keys moves the maximum, by little or by more than weights hold."""
    b = batch([600], None, 1, 1, 64, BF, False, "rows", scale=1.0)
    b.q.zero_()
    b.q[:, :, 0] = 1
    b.k.zero_()
    b.k[:, 0, 0] = (torch.arange(600, device="cuda") * step / 128).to(BF)
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_padded_rows(causal, dtype):
    """A padded batch: lengths apart from starts, rows between sequences that hold NaN, an empty sequence."""
    S, n = 160, [160, 3, 0, 77, 129]
    at = [S * i for i in range(5)]
    b = Batch(at, at, 2, 1, 64, dtype, causal, q_len=n, k_len=n, q_rows=5 * S, k_rows=5 * S)
    for i in range(5):
        for x in (b.q, b.k, b.v, b.g):
            x[S * i + n[i]:S * (i + 1)] = torch.nan
    b.forward()
    b.check_forward()
    b.o[torch.arange(5 * S, device="cuda") % S >= torch.tensor(n, device="cuda").repeat_interleave(S)] = torch.nan
    keep = b.o.clone()
    b.backward()
    b.o[torch.isnan(keep)] = 0
    for i in range(5):
        for x in (b.q, b.k, b.v, b.g):
            x[S * i + n[i]:S * (i + 1)] = 0
    b.check_backward()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_seen_does_not_enter(bad, d):
    """Infinities and NaN in another sequence, in later keys, and in rows behind the last sequence."""
    b = Batch([0, 100, 230], [0, 100, 230], 2, 1, d, BF, True, q_rows=300, k_rows=300)
    b.k[180:, :, 3], b.v[180:, :, 5] = bad, bad
    b.q[230:], b.g[230:] = bad, bad
    clean = Batch([0, 100, 230], [0, 100, 230], 2, 1, d, BF, True, q_rows=300, k_rows=300)
    for x in (b, clean):
        x.forward()
        x.backward()
    torch.cuda.synchronize()
    o, lse, bo, bl = clean.case().forward()
    check("o", b.o[:180], o[:180], bo[:180])
    check("lse", b.lse[:, :180], lse[:, :180], bl[:, :180])
    assert not bool(torch.isfinite(b.o[180:230, :, 5].float()).any())
    # the first sequence's gradients, and queries before the bad keys
    for name, got, (want, bound), n in zip(("dq", "dk", "dv"), (b.dq, b.dk, b.dv), clean.case().backward(clean.g, clean.o), (180, 100, 100)):
        check(name, got[:n], want[:n], bound[:n])


def test_shared_keys_and_any_order():
    """Sequences whose keys come in another order than their queries, and two that share them."""
    b = Batch([0, 40, 90, 130], [200, 0, 200], 2, 2, 64, BF, False, k_len=[150, 70, 150], k_rows=400)
    b.n = 3
    b.forward()
    b.check_forward()


def test_starts_out_of_range():
    """Rows that the arrays name beyond the operands are left out."""
    b = Batch([0, 50, 120], [0, 90, 500], 2, 2, 64, BF, True, q_rows=100, k_rows=300)
    b.forward()
    b.check_forward()
    b = Batch([-20, 50, 100], [-7, 90, 120], 2, 2, 64, BF, False, q_rows=100, k_rows=120)
    b.forward()
    b.check_forward()


def test_nothing_to_do():
    for qn, kn in [([0, 0], [3, 4]), ([4, 6], [0, 0]), ([], [])]:
        b = batch(qn, kn, 2, 1, 64, BF, False, "rows")
        b.forward()
        b.check_forward()
        b.backward()
        b.check_backward()


@pytest.mark.parametrize("lens", [[3, 0, 1, 2, 5] * 260, [0] * 40 + [70] + [0] * 100 + [1] * 3 + [0] * 33 + [90], [0] * 1500 + [40] + [0] * 70])
def test_many_sequences(lens):
    """More sequences than are looked up in shared memory, and long runs of sequences without rows."""
    b = batch(lens, None, 2, 1, 32, BF, True, "rows")
    b.forward()
    b.check_forward()
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_seen_does_not_enter_shared_walks(bad):
    """The same where clusters share a walk: the keys of one sequence, or its queries, hold what is no number."""
    for qn, kn, spoil in [([17, 30], [4000, 1000], "kv"), ([3000, 900], [20, 30], "qg")]:
        b, clean = (Batch(starts(qn), starts(kn), 2, 1, 64, BF, False, seed=4) for _ in range(2))
        for x, at in [(b.k, kn), (b.v, kn)] if spoil == "kv" else [(b.q, qn), (b.g, qn)]:
            x[at[0]:, :, 7] = bad
        for x in (b, clean):
            x.forward()
            x.backward()
        torch.cuda.synchronize()
        o, lse, bo, bl = clean.case().forward()
        check("o", b.o[:qn[0]], o[:qn[0]], bo[:qn[0]])
        check("lse", b.lse[:, :qn[0]], lse[:, :qn[0]], bl[:, :qn[0]])
        for name, got, (want, bound), n in zip(("dq", "dk", "dv"), (b.dq, b.dk, b.dv), clean.case().backward(clean.g, clean.o), (qn[0], kn[0], kn[0])):
            check(name, got[:n], want[:n], bound[:n])


@pytest.mark.parametrize("call", ["forward", "token"])
def test_offsets_past_32_bits(call):
    """Keys behind 2^32 bytes and 2^31 elements of a cache, at the end of its rows."""
    rows, d = (1 << 31) // 128 + 1000, 128
    far = rows - 600
    if call == "token":
        b = Batch([0, 1, 2], [far, 5], 2, 1, d, BF, False, k_len=[600, 300], k_rows=8)
    else:
        b = Batch([0, 70, 100], [far, 5], 2, 1, d, BF, True, k_len=[600, 300], k_rows=8)
    kv = torch.zeros((2, rows, 1, d), dtype=BF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for at, n in ((far, 600), (5, 300)):
        kv[:, at:at + n] = torch.randn((2, n, 1, d), generator=g, device="cuda").to(BF)
    b.k, b.v = kv[0], kv[1]
    getattr(b, call)()
    torch.cuda.synchronize()
    near = Case(b.q, torch.cat([b.k[far:], b.k[5:305]]), torch.cat([b.v[far:], b.v[5:305]]), b.scale, b.causal, b.lists[0], [0, 600], None, [600, 300], 2)
    o, lse, bo, bl = near.forward()
    check("o", b.o, o, bo)
    check("lse", b.lse, lse, bl)


def test_many_heads_of_short_sequences():
    """Enough tiles that a CTA takes several heads, in groups that do not divide them."""
    for d, hq, hkv in ((64, 7, 7), (128, 6, 2), (64, 10, 5)):
        b = batch([90, 128, 30, 77, 1, 50] * 24, None, hq, hkv, d, BF, True, "fused")
        b.forward()
        b.check_forward()


def test_one_key():
    """A query that sees one key has the weight 1 whatever its score: no gradient reaches q, nor k where all queries of
    a sequence are such; exactly, not within rounding.  What is not a number stays so."""
    for qn, kn, causal in [([70, 300, 5], [1, 1, 1], False), ([1] * 40, None, True), ([2000], [1], False)]:
        b = batch(qn, kn, 4, 2, 64, BF, causal, "rows")
        b.forward()
        b.backward()
        b.check_backward()
        assert not bool(b.dq.any()) and not bool(b.dk.any()) and bool(b.dv.any())
    b = batch([300], None, 2, 1, 128, FP, True, "rows")
    b.forward()
    b.backward()
    b.check_backward()
    assert not bool(b.dq[0].any()) and bool(b.dq[1].any())
    b = batch([70, 300], [1, 1], 1, 1, 64, BF, False, "rows")
    b.forward()
    b.g[10, 0, 3] = torch.nan
    b.backward()
    torch.cuda.synchronize()
    assert bool(torch.isnan(b.dq[10]).all()) and bool(torch.isnan(b.dk[0]).all()) and not bool(b.dq[11:].any()) and not bool(b.dk[1].any())


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 40, 128])
@pytest.mark.parametrize("qn,kn,causal", [([2, 3] * 60, None, True), ([3, 2, 1, 0, 4] * 30, None, False), ([12] * 50, None, True),
                                          ([40, 0, 60, 3] * 9, [2, 5, 0, 4] * 9, False)])
def test_gradients_of_few_keys(qn, kn, causal, d, dtype):
    """Few keys a row: the gradients are as near the true ones as their roundings, not as what o's rounding leaves of D."""
    b = batch(qn, kn, 4, 2, d, dtype, causal, "rows", seed=3)
    b.forward()
    b.backward()
    b.check_backward()
    for name, got, (want, _) in zip(("dq", "dk", "dv"), (b.dq, b.dk, b.dv), b.case().backward(b.g, b.o)):
        live = ~torch.isnan(want)
        # Rounding x of a binade [1, 2) is off by at most half a step h, h / sqrt 3 as a root of a mean square; that of x is
        # sqrt(3 / (2 ln 2)) = 1.47 there (as many in each part of a logarithm): 0.39 h of the norm.  A result and the P or dS that it
        # sums: 0.39 sqrt 2 = 0.56 h, over hundreds of them; 0.7 leaves room for other spreads (at most 0.58 each where all begin
        # a binade).  D from the rounded o comes on top: 0.8 h in all for sequences of 2 and 3.
        far = ((got.cpu().double() - want)[live] ** 2).sum().sqrt() / (want[live] ** 2).sum().sqrt()
        assert float(far) <= 0.7 * torch.finfo(dtype).eps / 2, (name, float(far))


def test_without_lse():
    b = batch([70, 200], None, 2, 1, 64, FP, True, "rows")
    b.forward(lse=False)
    torch.cuda.synchronize()
    o, _, bo, _ = b.case().forward()
    check("o", b.o, o, bo)
    assert bool((b.lse == SENTINEL).all())


def test_gradients_against_differences():
    """The loss sum(o w) moved by small steps of random directions of q, k and v: its differences in 64 bits are the
    gradients' products with the direction, within the gradients' rounding (2^-8 of the magnitudes that are added) and the
    step's third-order term."""
    b = batch([37, 150], None, 2, 1, 64, BF, True, "rows", seed=9)
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    g = b.g.cpu().double()
    for i, (x, grad) in enumerate([(b.q, b.dq), (b.k, b.dk), (b.v, b.dv)]):
        direction = torch.randn(x.shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64)
        loss = []
        for t in (1e-3, -1e-3):
            c = b.case()
            ops = [c.q, c.k, c.v]
            ops[i] = ops[i] + t * direction
            c.q, c.k, c.v = ops
            loss.append(float((c.forward()[0] * g).sum()))
        want = (loss[0] - loss[1]) / 2e-3
        terms = grad.cpu().double() * direction
        assert abs(float(terms.sum()) - want) <= 2.0 ** -7 * float(terms.norm()) * 4 + 1e-3, (i, float(terms.sum()), want)


def test_runs_alike():
    """Two runs give the same bits."""
    b = batch([600, 77, 300], None, 4, 1, 64, BF, True, "rows")
    b.forward()
    b.backward()
    first = [x.clone() for x in (b.o, b.lse, b.dq, b.dk, b.dv)]
    b.forward()
    b.backward()
    for x, y in zip(first, (b.o, b.lse, b.dq, b.dk, b.dv)):
        assert torch.equal(x, y)


def test_streams_and_graphs():
    """Two batches on two streams at once; a captured forward and backward pass, replayed on new values and new lengths."""
    a, b = batch([300, 200], None, 2, 2, 64, BF, True, "rows", seed=1), batch([100, 400], None, 2, 2, 64, BF, True, "rows", seed=2)
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        for x, st in ((a, s), (b, t)):
            x.forward(st)
            x.backward(st)
    torch.cuda.synchronize()
    for x in (a, b):
        x.check_forward()
        x.check_backward()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        a.forward(s)
        a.backward(s)
    for x in (a.o, a.dq, a.dk, a.dv):
        x.fill_(SENTINEL)
    for x, y in ((a.q, b.q), (a.k, b.k), (a.v, b.v), (a.g, b.g)):
        x.copy_(y)
    a.arrays[0].copy_(dev([0, 410, 500]))
    a.arrays[1].copy_(dev([0, 410, 500]))
    a.lists = ([0, 410, 500], [0, 410, 500], None, None)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    a.check_forward()
    a.check_backward()


# --------------------------------------------------------------------------- one query per sequence
TOKENS = [
    # lengths, capacity, query heads, key heads, head size, type
    ([1], 8, 1, 1, 64, BF),
    ([30, 31, 34, 32], 64, 4, 4, 64, BF),
    ([0, 5, 160, 128, 129], 160, 8, 8, 64, FP),
    ([4000, 1, 0, 2900], 4096, 8, 2, 128, BF),
    ([9000], 9000, 16, 1, 128, BF),
    ([700, 65], 1000, 6, 2, 32, FP),
    ([513, 64, 63], 600, 3, 1, 96, BF),
    ([100, 200], 256, 20, 1, 64, BF),
    ([511] * 40, 512, 4, 2, 8, FP),
    ([1777, 3], 2000, 5, 5, 120, BF),
    ([257, 300], 300, 33, 1, 128, FP),
]


def tokens(n, cap, hq, hkv, d, dtype, **kw):
    B = len(n)
    return Batch(list(range(B + 1)), [cap * i for i in range(B)], hq, hkv, d, dtype, False, k_len=n, k_rows=B * cap, **kw)


@pytest.mark.parametrize("n,cap,hq,hkv,d,dtype", TOKENS)
@pytest.mark.parametrize("layout", ["rows", "heads", "wide"])
def test_token(n, cap, hq, hkv, d, dtype, layout):
    b = tokens(n, cap, hq, hkv, d, dtype, layout=layout)
    b.token()
    b.check_forward()


@pytest.mark.parametrize("d", [64, 128])
def test_token_beside_unfilled_cache(d):
    """The part of a cache that is not filled holds NaN."""
    n, cap = [70, 0, 300, 1, 256, 128], 384
    b = tokens(n, cap, 4, 2, d, BF)
    for i, m in enumerate(n):
        b.k[cap * i + m:cap * (i + 1)] = torch.nan
        b.v[cap * i + m:cap * (i + 1)] = torch.nan
    b.token()
    b.check_forward()


def test_token_shares_keys_and_packed():
    """Beams that share their sentence's keys, and keys packed without lengths."""
    b = Batch(list(range(5)), [0, 0, 100, 100], 4, 4, 64, BF, False, k_len=[90, 90, 77, 77], k_rows=200)
    b.token()
    b.check_forward()
    b = Batch(list(range(4)), [0, 300, 310, 700], 4, 2, 64, FP, False)
    b.token()
    b.check_forward()


@pytest.mark.parametrize("spread", [10.0, 0.01])
def test_token_sharp_and_flat(spread):
    b = tokens([1500, 700], 1500, 4, 1, 64, BF, spread=spread)
    b.token()
    b.check_forward()


def test_token_is_the_last_row_of_the_prompt():
    """A prompt's last query through the single-token form is the same within both forms' roundings."""
    b = batch([200, 77], None, 4, 2, 64, BF, True, "rows")
    b.forward()
    b.check_forward()
    t = Batch([0, 1, 2], [0, 200, 277], 4, 2, 64, BF, False)
    t.q.copy_(b.q[[199, 276]])
    t.k.copy_(b.k)
    t.v.copy_(b.v)
    t.token()
    t.check_forward()
    _, _, bo, bl = t.case().forward()
    assert bool(((t.o.cpu().double() - b.o[[199, 276]].cpu().double()).abs() <= 2 * bo).all())
    assert bool(((t.lse - b.lse[:, [199, 276]]).cpu().abs() <= 2 * bl).all())


def test_token_many_sequences():
    """More units than are cut: a warp each."""
    n = [(37 * i) % 90 for i in range(700)]
    b = tokens(n, 90, 8, 4, 64, BF)
    b.token()
    b.check_forward()


def shared_cache(lens, first, q, k, v):
    """One head of 8, fp16, against a cache whose rows sequences share."""
    B, rows = len(lens), k.shape[0]
    s = mnmt.AttentionShape(B, B, rows, 1, 1, 8, mnmt.F16, False, 8 ** -0.5, None, dev(first), k_len=dev(lens))
    ws = torch.full((mnmt.mnmt_attention_token_workspace(s),), 0xFF, dtype=torch.uint8, device="cuda")
    o, lse = torch.full_like(q, SENTINEL), torch.full((1, B), SENTINEL, device="cuda")
    mnmt.mnmt_attention_token(s, mnmt.heads(q), mnmt.heads(k), mnmt.heads(v), mnmt.heads(o), lse, ws)
    torch.cuda.synchronize()
    return o[:, 0], lse[0]


def test_token_many_long_caches():
    """Room for more than 2^31 tiles of 32 keys, few of them used: units are cut into larger pieces."""
    B, rows = 2100, 1 << 25
    g, r = torch.Generator(device="cuda").manual_seed(5), torch.Generator().manual_seed(6)
    k, v = ((torch.randn((rows, 1, 8), generator=g, device="cuda") * 0.5).to(FP) for _ in range(2))
    q = torch.randn((B, 1, 8), generator=g, device="cuda").to(FP)
    lens = torch.randint(0, 9000, (B,), generator=r).tolist()
    first = torch.randint(0, rows, (B,), generator=r).tolist()
    lens[7], lens[14], first[21] = 0, 1, rows - 100  # the last ends behind the cache
    lens[21] = 500
    o, lse = shared_cache(lens, first, q, k, v)
    for b in [7, 14, 21, *range(0, B, 70)]:
        end = min(rows, first[b] + lens[b])
        if end <= first[b]:
            assert float(o[b].abs().max()) == 0.0 and float(lse[b]) == -float("inf")
            continue
        x = (k[first[b]:end, 0].double() * q[b, 0].double()).sum(1) * 8 ** -0.5
        w = torch.softmax(x, 0)[:, None] * v[first[b]:end, 0].double()
        want, mag = w.sum(0), w.abs().sum(0)
        # scores: exact products, ten fp32 steps of 2^-24 of values below 32, which a power turns into a relative 10 * 32 * 2^-24
        # < 2^-15, in numerator and denominator; a weight's rounding 2^-11; n sums in fp32 in each, truncated in one of them (2^-23);
        # the result's rounding
        n = end - first[b]
        assert bool((abs(o[b].double() - want) <= mag * (2.0 ** -14 + 2.0 ** -11 + 3 * n * 2.0 ** -24) + want.abs() * 2.0 ** -11 + 2.0 ** -25).all())
        assert abs(float(lse[b]) - float(torch.logsumexp(x, 0))) <= 2.0 ** -15 + n * 2.0 ** -24 + 32 * 2.0 ** -23


def test_token_more_than_31_bits_of_tiles():
    """Sequences that share all rows of a long cache: 2^31 tiles of 32 keys and more."""
    B, rows = 2100, 1 << 25
    g = torch.Generator(device="cuda").manual_seed(5)
    k = (torch.randn((rows, 1, 8), generator=g, device="cuda") * 0.5).to(FP)
    q = torch.randn((1, 1, 8), generator=g, device="cuda").to(FP)
    o, lse = shared_cache([rows] * B, [0] * B, q.expand(B, 1, 8).contiguous(), k, torch.ones_like(k))
    # a lane adds up to 2^22 terms (half an ulp each: 2^-2 of the sum), the tensor core 2^21 truncated ones (2^-2): a mean of ones
    # between 0.75 / 1.25 and 1.25 / 0.75, and log 0.75 in the log-sum-exp
    assert 0.59 < float(o.min()) and float(o.max()) < 1.68
    want = float(torch.logsumexp((k[:, 0].double() * q[0, 0].double()).sum(1) * 8 ** -0.5, 0))
    assert float((lse - want).abs().max()) < 0.3


def test_token_graph():
    """A captured step, replayed while the cache fills."""
    b = tokens([10, 200, 1], 512, 4, 2, 64, BF)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        b.token(s)
    for n in ([10, 200, 1], [11, 201, 2], [511, 0, 512]):
        b.arrays[3].copy_(dev(n))
        b.lists = b.lists[:3] + (n,)
        b.o.fill_(SENTINEL)
        graph.replay()
        b.check_forward()
