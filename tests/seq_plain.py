"""Attention over sequences in 64 bits, from its formulas, sequence by sequence and head by head, with bounds on how far
a kernel may be from it.

Bounds (u: half a step of the operands' type, z: half its smallest step, 2^-25 for fp16): a score is off by at most
e = (d + 4) 2^-24 scale |q| . |k| + 2^-22 |s| (fp32 sums, the power), so a weight by 2 e relative; weights (and dS) are
rounded to the type (u relative, z absolute; where the power is below 2^-126 it is zero in fp32, which moves a weight by
f = 2^-126 and dS by f (|g . v| + |D|)); sums of n terms in fp32 add n 2^-23 of the sum of magnitudes (the tensor
cores truncate); results are rounded once.  D is taken from the o that the kernel is given, which is rounded: u |g| . |o|.
Written before the kernels ran."""
import torch


FLUSH = 2.0 ** -126


def half_step(dtype):
    return torch.finfo(dtype).eps / 2, 2.0 ** -25 if dtype == torch.float16 else FLUSH


def rows_of(start, length, b, rows):
    lo = min(max(start[b], 0), rows)
    hi = start[b + 1] if length is None else start[b] + max(length[b], 0)
    return lo, max(lo, min(hi, rows))


def hidden(nq, nk, causal):
    i, j = torch.arange(nq)[:, None], torch.arange(nk)
    return (j > i + nk - nq) if causal else torch.zeros((nq, nk), dtype=torch.bool)


def _scores(q, k, scale, mask):
    """s, P, lse and the bound on the relative error of P."""
    n = q.shape[1]
    s = scale * (q @ k.t())
    e = (n + 4) * 2.0 ** -24 * scale * (q.abs() @ k.abs().t()) + 2.0 ** -22 * s.abs()
    e = e.masked_fill(mask, 0.0)
    s = s.masked_fill(mask, -torch.inf)
    m = s.amax(1) if s.shape[1] else torch.full((s.shape[0],), -torch.inf, dtype=torch.float64)
    w = torch.exp(s - torch.where(m == -torch.inf, 0.0, m)[:, None]).masked_fill(mask, 0.0)
    z = w.sum(1)
    none = mask.all(1) if s.shape[1] else torch.ones(s.shape[0], dtype=torch.bool)
    P = w / torch.where(none, 1.0, z)[:, None]
    e = e + (e.amax(1) if e.shape[1] else torch.zeros(e.shape[0], dtype=torch.float64))[:, None]
    return s, P.masked_fill(mask, 0.0), torch.where(none, -torch.inf, m + torch.log(z)), e


class Case:
    """q [Tq][Hq][d], k, v [Tk][Hkv][d] (torch, any device), starts and lengths as Python lists."""

    def __init__(self, q, k, v, scale, causal, q_start, k_start, q_len=None, k_len=None, n=None):
        self.q, self.k, self.v = (x.detach().cpu().double() for x in (q, k, v))
        self.dtype, self.scale, self.causal = q.dtype, scale, causal
        n = n if n is not None else (len(q_start) - 1 if q_len is None else len(q_len))
        self.seqs = []
        for b in range(n):
            self.seqs.append(rows_of(q_start, q_len, b, q.shape[0]) + rows_of(k_start, k_len, b, k.shape[0]))

    def _visit(self):
        group = self.q.shape[1] // max(1, self.k.shape[1])
        for q0, q1, k0, k1 in self.seqs:
            mask = hidden(q1 - q0, k1 - k0, self.causal)
            for h in range(self.q.shape[1]):
                yield slice(q0, q1), slice(k0, k1), h, h // group, mask

    def forward(self):
        """o, lse, and their bounds; rows of no sequence are NaN."""
        u, z = half_step(self.dtype)
        o = torch.full(self.q.shape, torch.nan, dtype=torch.float64)
        lse = torch.full((self.q.shape[1], self.q.shape[0]), torch.nan, dtype=torch.float64)
        bo, bl = torch.zeros_like(o), torch.zeros_like(lse)
        for r, c, h, g, mask in self._visit():
            q, k, v = self.q[r, h], self.k[c, g], self.v[c, g]
            s, P, L, e = _scores(q, k, self.scale, mask)
            n = k.shape[0]
            w = torch.where(mask, 0.0, v.abs().amax(1)[None] if n else 0.0) if n else torch.zeros((q.shape[0], 0), dtype=torch.float64)
            o[r, h], lse[h, r] = _clean(P, v, mask), L
            bo[r, h] = (P * (u + 2 * e + n * 2.0 ** -23)) @ v.abs().nan_to_num(0, 0, 0) + z * w.sum(1)[:, None]
            bo[r, h] += u * o[r, h].abs() + z
            bl[h, r] = (e.amax(1) if n else 0.0) + 2.0 ** -21 * (1 + L.abs().nan_to_num(0, 0, 0)) + n * 2.0 ** -23
        return o, lse, bo, bl

    def backward(self, g, o):
        """dq, dk, dv for the gradient g of o (rounded, as the forward pass left it), and their bounds."""
        g, o = g.detach().cpu().double(), o.detach().cpu().double()
        u, z = half_step(self.dtype)
        dq, dk, dv = (torch.full(x.shape, torch.nan, dtype=torch.float64) for x in (self.q, self.k, self.v))
        bq, bk, bv = (torch.zeros_like(x) for x in (dq, dk, dv))
        for q0, q1, k0, k1 in self.seqs:
            dk[k0:k1], dv[k0:k1], dq[q0:q1] = 0.0, 0.0, 0.0
        d = self.q.shape[2]
        for r, c, h, hk, mask in self._visit():
            if q_empty(r) or q_empty(c):
                continue
            q, k, v, gi, oi = self.q[r, h], self.k[c, hk], self.v[c, hk], g[r, h], o[r, h]
            s, P, _, e = _scores(q, k, self.scale, mask)
            dP = gi @ v.t()
            true_o = _clean(P, v, mask)
            dS = (P * (dP - (gi * true_o).sum(1, keepdim=True))).masked_fill(mask, 0.0)
            go = (gi.abs() * torch.maximum(oi.abs(), true_o.abs())).sum(1, keepdim=True)
            off = (gi * (oi - true_o)).abs().sum(1, keepdim=True)  # how far the given o is from the true one
            n, m = k.shape[0], q.shape[0]
            eS = dS.abs() * (u + 2 * e) + P * (1 + 2 * e) * (off + u * go + (d + 4) * 2.0 ** -23 * (gi.abs() @ v.abs().t() + go)) + (z + FLUSH * (dP.abs() + go)) * ~mask
            dq[r, h] = self.scale * (dS @ k)
            bq[r, h] = self.scale * ((eS + n * 2.0 ** -23 * dS.abs()) @ k.abs())
            dk[c, hk] += self.scale * (dS.t() @ q)
            bk[c, hk] += self.scale * ((eS + m * 2.0 ** -22 * dS.abs()).t() @ q.abs())
            dv[c, hk] += P.t() @ gi
            bv[c, hk] += (P * (u + 2 * e + m * 2.0 ** -22) + z * ~mask).t() @ gi.abs()
        return [(x, b + u * x.abs() + z) for x, b in ((dq, bq), (dk, bk), (dv, bv))]


def q_empty(s):
    return s.stop <= s.start


def _clean(P, v, mask):
    """P v over the keys that each row sees: a masked key's infinity or NaN does not enter."""
    if torch.isfinite(v).all():
        return P @ v
    out = torch.zeros((P.shape[0], v.shape[1]), dtype=torch.float64)
    for i in range(P.shape[0]):
        see = ~mask[i]
        out[i] = P[i, see] @ v[see]
    return out


def check(name, got, want, bound):
    """got against want within bound; NaN in want: rows that are left alone (not looked at)."""
    got = got.detach().cpu().double()
    live = ~torch.isnan(want)
    bad = live & ~((got - want).abs() <= bound) & (got != want)
    if bad.any():
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{name}: {int(bad.sum())} of {int(live.sum())} off, first at {at}: {float(got[at])} for {float(want[at])}, "
                             f"bound {float(bound[at])}")
