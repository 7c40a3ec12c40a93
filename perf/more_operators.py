"""Performance cases of attention over packed sequences and of the embedding, with their gradients.

The operators, as a user of the library calls them:

* `attention`: softmax attention of a batch of sequences of different lengths whose rows lie one after another (no
  padding), causal or not, query heads in groups that share a key head; self- or cross-attention; with the row's
  log-sum-exp that the backward pass reads;
* `attention_backward`: the gradients of queries, keys and values;
* `attention_token`: the serving form: one query per sequence against a key and value cache of a fixed capacity, of which
  each sequence has filled a part;
* `embed`: table rows times a scale, plus the row of a positional table;
* `embed_backward`: the table's gradient, dense, with a token that takes none.

`own = False` computes each operator in its plain form: elementary torch operations in 32 bits, rounded once at the end;
sequences are laid out at a common length with a mask.

Lengths and ids' sizes are the case's own (a seed in the case), so that every pass of a case does the same work.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EMB_SCALE = 22.627416997969522  # sqrt(512)


def listed():
    return [
        # one decode step of a beam search on one sentence: 4 hypotheses, caches of 64 of which about half is filled: latency
        dict(name="token_beams", kind="attention_token", dtype="bf16", B=4, Hq=4, Hkv=4, dh=64, cap=64, k_lo=30, k_hi=34, lens=1),
        # one decode step of a batch: 128 sentences with four beams
        dict(name="token_batch", kind="attention_token", dtype="f16", B=512, Hq=8, Hkv=8, dh=64, cap=160, k_lo=80, k_hi=160, lens=2),
        # one token each of a few long documents, grouped heads: the cache's bytes
        dict(name="token_long", kind="attention_token", dtype="bf16", B=12, Hq=16, Hkv=4, dh=128, cap=32768, k_lo=9000, k_hi=32768, lens=3),
        # a decoder's prompt of one sentence: latency
        dict(name="forward_sentence", kind="attention", dtype="bf16", B=1, Hq=4, Hkv=4, dh=64, causal=True, cross=False, q_lo=46, q_hi=46,
             k_lo=46, k_hi=46, lens=4, fused=True),
        # cross-attention of a training batch: 128 targets against their sources, ragged
        dict(name="forward_cross", kind="attention", dtype="f16", B=128, Hq=8, Hkv=8, dh=64, causal=False, cross=True, q_lo=20, q_hi=160,
             k_lo=20, k_hi=128, lens=5, fused=False),
        # two long documents, grouped heads
        dict(name="forward_long", kind="attention", dtype="bf16", B=2, Hq=16, Hkv=2, dh=128, causal=True, cross=False, q_lo=6000, q_hi=8192,
             k_lo=6000, k_hi=8192, lens=6, fused=True),
        # the decoder's self-attention gradients of a training batch of sentences
        dict(name="backward_batch", kind="attention_backward", dtype="bf16", B=128, Hq=8, Hkv=8, dh=64, causal=True, cross=False, q_lo=20,
             q_hi=128, k_lo=20, k_hi=128, lens=7, fused=True),
        # the gradients of a few documents of odd lengths, grouped heads: the largest
        dict(name="backward_long", kind="attention_backward", dtype="bf16", B=3, Hq=16, Hkv=2, dh=128, causal=True, cross=False, q_lo=2500,
             q_hi=4095, k_lo=2500, k_hi=4095, lens=8, fused=True),
        # the tokens of one decode step: latency
        dict(name="embed_token", kind="embed", dtype="bf16", out="f32", T=4, V=8000, d=384, P=128, pad=0),
        # a packed training batch into the fp32 residual stream
        dict(name="embed_batch", kind="embed", dtype="f32", out="f32", T=16384, V=32000, d=2048, P=160, pad=0),
        # the gradient of the table for one sentence of 46 tokens: the dense gradient's zeros
        dict(name="embed_backward_sentence", kind="embed_backward", dtype="bf16", out="f32", T=46, V=8000, d=256, pad=0),
        # the gradient of the widest table over a training batch, words as frequent as in text
        dict(name="embed_backward_batch", kind="embed_backward", dtype="bf16", out="f32", T=16384, V=32000, d=2048, pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, case):
    case["dh"] = rng.choice([32, 64, 64, 64, 128, 128, 8 * rng.randint(1, 16)])
    case["Hkv"] = rng.choice([1, 2, 3, 4, 6, 8])
    case["Hq"] = case["Hkv"] * rng.choice([1, 1, 1, 2, 4, rng.randint(1, 5)])
    case["lens"] = rng.randint(1, 10 ** 6)
    return case


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "attention_backward", "attention_backward", "attention_token",
                       "attention_token", "embed", "embed_backward", "embed_backward"])
    case = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f16"]))
    if kind == "attention_token":
        case = _heads(rng, case)
        case["B"], case["cap"] = _log(rng, 1, 512), _log(rng, 8, 32768)
        while case["B"] * case["cap"] * case["Hkv"] * case["dh"] > 12 * 32768 * 4 * 128 // 2:
            case["B"], case["cap"] = max(1, case["B"] // 2), max(8, case["cap"] * 2 // 3)
        case["k_hi"] = case["cap"]
        case["k_lo"] = rng.randint(0, case["cap"])
        return case
    if kind.startswith("attention"):
        case = _heads(rng, case)
        B, hi = _log(rng, 1, 256), _log(rng, 1, 8192)
        cross = rng.random() < 0.3
        khi = _log(rng, 1, 8192) if cross else hi
        # at most the work and the room of the largest: pairs of rows over all heads
        while B * case["Hq"] * hi * khi > 16 * 3200 ** 2 or B * max(hi, khi) > 16384:
            B, hi, khi = max(1, B * 2 // 3), max(1, hi * 5 // 6), max(1, khi * 5 // 6)
            if not cross:
                khi = hi
        lo, klo = rng.randint(0, hi), rng.randint(0, khi)
        return case | dict(B=B, causal=rng.random() < 0.6, cross=cross, q_lo=lo, q_hi=hi, k_lo=klo if cross else lo, k_hi=khi, fused=not cross and rng.random() < 0.5)
    case["dtype"] = rng.choice(["bf16", "f32", "f16"])
    T, V, d = _log(rng, 1, 32768), _log(rng, 100, 64000), _log(rng, 32, 2048)
    if rng.random() < 0.6:  # most of them in steps of 64, as the widths of layers are
        d = max(64, d // 64 * 64)
    while T * d > 16384 * 2048 or V * d > 32000 * 2048:
        d = max(32, d // 2)
    case |= dict(out=rng.choice(["f32", "f32", "bf16", "f16"]), T=T, V=V, d=d, pad=rng.choice([0, 0, 0, 8, rng.randint(1, 40)]))
    if kind == "embed":
        case["P"] = rng.choice([0, _log(rng, 8, 4096)])
    return case


def _lengths(case):
    """Lengths of queries and keys of a case's sequences."""
    rng = random.Random(case["lens"])
    k = [rng.randint(case["k_lo"], case["k_hi"]) for _ in range(case["B"])]
    if case["kind"] == "attention_token":
        return [1] * case["B"], k
    return ([rng.randint(case["q_lo"], case["q_hi"]) for _ in range(case["B"])], k) if case["cross"] else (k, k)


def _pairs(case):
    """Pairs of a query and a key that it sees, of one head."""
    n = 0
    for q, k in zip(*_lengths(case)):
        if case.get("causal"):
            m = min(q, k)  # rows that see a key: m of them, the last sees all k
            n += m * k - m * (m - 1) // 2
        else:
            n += q * k
    return n


# --------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _starts(lens):
    s = [0]
    for n in lens:
        s.append(s[-1] + n)
    return s


def _device(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _ids(g, T, V):
    """Token ids as frequent as words are: the n-th has a share of about 1 / n."""
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(V + 1)) - 1).clamp(0, V - 1).to(torch.int32)


def _strided(x, dtype, pad):
    """x in its type, as the leading columns of a buffer `pad` columns wider."""
    buf = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=dtype, device="cuda")
    buf[:, :x.shape[1]] = x
    return buf[:, :x.shape[1]]


def prepare(case, seed):
    g = _gen(seed)
    dt, kind = DTYPES[case["dtype"]], case["kind"]
    st = {"case": case}
    if kind.startswith("attention"):
        Hq, Hkv, dh, B = case["Hq"], case["Hkv"], case["dh"], case["B"]
        ql, kl = _lengths(case)
        st["scale"] = dh ** -0.5
        if kind == "attention_token":
            cap = case["cap"]
            st["q"] = _normal(g, B, Hq, dh).to(dt)
            cache = torch.empty((2, B * cap, Hkv, dh), dtype=dt, device="cuda").normal_(generator=g)
            st["k"], st["v"] = cache[0], cache[1]
            st["o"] = torch.zeros_like(st["q"])
            st["k_start"], st["k_len"] = _device([b * cap for b in range(B + 1)]), _device(kl)
            st["q_start"], st["k_rows"] = _device(list(range(B + 1))), B * cap
            return st
        qs, ks = _starts(ql), _starts(kl)
        st["q_start"] = _device(qs)
        st["k_start"] = _device(ks) if case["cross"] else st["q_start"]
        st["q_max"], st["k_max"] = max(ql), max(kl)
        Tq, Tk = qs[-1], ks[-1]
        if case["fused"]:  # heads of queries, keys and values beside each other, as one linear writes them
            qkv = _normal(g, Tq, Hq + 2 * Hkv, dh).to(dt)
            st["q"], st["k"], st["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        else:
            st["q"], st["k"], st["v"] = _normal(g, Tq, Hq, dh).to(dt), _normal(g, Tk, Hkv, dh).to(dt), _normal(g, Tk, Hkv, dh).to(dt)
        st["o"] = torch.zeros((Tq, Hq, dh), dtype=dt, device="cuda")
        st["lse"] = torch.zeros((Hq, Tq), device="cuda")
        if kind == "attention_backward":
            st["o"], st["lse"] = _attention(st)
            st["do"] = (_normal(g, Tq, Hq, dh) * 1e-2).to(dt)
            if case["fused"]:
                d = torch.zeros((Tq, Hq + 2 * Hkv, dh), dtype=dt, device="cuda")
                st["dq"], st["dk"], st["dv"] = d[:, :Hq], d[:, Hq:Hq + Hkv], d[:, Hq + Hkv:]
            else:
                st["dq"], st["dk"], st["dv"] = torch.zeros_like(st["q"]), torch.zeros_like(st["k"]), torch.zeros_like(st["v"])
        return st
    T, V, d, pad, odt = case["T"], case["V"], case["d"], case["pad"], DTYPES[case["out"]]
    st["ids"] = _ids(g, T, V)
    if kind == "embed":
        st["table"] = _strided(_normal(g, V, d) * 0.02, dt, pad)
        if case["P"]:
            st["pe"] = torch.rand((case["P"], d), generator=g, device="cuda") * 2 - 1
            st["pos"] = torch.randint(0, case["P"], (T,), generator=g, device="cuda", dtype=torch.int32)
        st["x"] = _strided(torch.zeros((T, d), device="cuda"), odt, pad)
    else:
        st["g"] = _strided(_normal(g, T, d) * 1e-2, dt, pad)
        st["table_grad"] = _strided(torch.zeros((V, d), device="cuda"), odt, pad)
    return st


# --------------------------------------------------------------------------- one pass
def _run_own(st):
    from paper_2306_04235_gb300 import mnmt

    case = st["case"]
    kind = case["kind"]
    types = {"f32": mnmt.F32, "bf16": mnmt.BF16, "f16": mnmt.F16}
    dt = types[case["dtype"]]
    if kind == "attention_token":
        a = mnmt.AttentionShape(case["B"], case["B"], st["k_rows"], case["Hq"], case["Hkv"], case["dh"], dt, False, st["scale"],
                                st["q_start"], st["k_start"], k_len=st["k_len"])
        ws = torch.empty(mnmt.mnmt_attention_token_workspace(a), dtype=torch.uint8, device="cuda")
        mnmt.mnmt_attention_token(a, mnmt.heads(st["q"]), mnmt.heads(st["k"]), mnmt.heads(st["v"]), mnmt.heads(st["o"]), None, ws)
        return st["o"]
    if kind.startswith("attention"):
        a = mnmt.AttentionShape(case["B"], st["q"].shape[0], st["k"].shape[0], case["Hq"], case["Hkv"], case["dh"], dt, case["causal"],
                                st["scale"], st["q_start"], st["k_start"])
        q, k, v, o = mnmt.heads(st["q"]), mnmt.heads(st["k"]), mnmt.heads(st["v"]), mnmt.heads(st["o"])
        if kind == "attention":
            ws = torch.empty(mnmt.mnmt_attention_forward_workspace(a), dtype=torch.uint8, device="cuda")
            mnmt.mnmt_attention_forward(a, q, k, v, o, st["lse"], ws)
            return [st["o"], st["lse"]]
        ws = torch.empty(mnmt.mnmt_attention_backward_workspace(a), dtype=torch.uint8, device="cuda")
        mnmt.mnmt_attention_backward(a, q, k, v, o, st["lse"], mnmt.heads(st["do"]), mnmt.heads(st["dq"]), mnmt.heads(st["dk"]),
                                     mnmt.heads(st["dv"]), ws)
        return [st["dq"], st["dk"], st["dv"]]
    T, V, d, pad = case["T"], case["V"], case["d"], case["pad"]
    ot = types[case["out"]]
    if kind == "embed":
        mnmt.mnmt_embed(st["ids"], T, st["table"], dt, d + pad, V, d, EMB_SCALE, st["x"], ot, d + pad, st.get("pos"), st.get("pe"), d, case["P"])
        return st["x"]
    ws = torch.empty(mnmt.mnmt_embed_backward_workspace(T, V, d), dtype=torch.uint8, device="cuda")
    mnmt.mnmt_embed_backward(st["ids"], T, st["g"], dt, d + pad, EMB_SCALE, 0, V, d, st["table_grad"], ot, d + pad, False, ws)
    return st["table_grad"]


def _padded(x, start, n):
    """Packed rows [T][H][d] as fp32 [B][H][n][d], rows past a sequence's end taken from a row in range."""
    at = (start[:-1, None] + torch.arange(n, device="cuda")).clamp_max(x.shape[0] - 1)
    return x[at].float().transpose(1, 2)


def _packed(x, start, n, rows):
    """[B][H][n][d] back to packed rows [T][H][d]."""
    length = start[1:] - start[:-1]
    t = torch.arange(n, device="cuda")
    live = t < length[:, None]
    return x.transpose(1, 2)[live].view(rows, x.shape[1], x.shape[3])


def _visible(st):
    """Which keys a query sees: [B][1][q_max][k_max]."""
    ql, kl = st["q_start"].diff(), st["k_start"].diff()
    i, j = torch.arange(st["q_max"], device="cuda")[:, None], torch.arange(st["k_max"], device="cuda")
    m = (i < ql[:, None, None]) & (j < kl[:, None, None])
    if st["case"]["causal"]:
        m = m & (j <= i + (kl - ql)[:, None, None])
    return m[:, None]


def _groups(x, Hq):
    """[B][Hkv][n][d] with each head once for every query head of its group."""
    return x.repeat_interleave(Hq // x.shape[1], 1)


def _weights(st, q, k):
    """Softmax weights [B][Hq][q][k] and log-sum-exp of fp32 q and k; no key: zeros and -inf."""
    s = ((q @ k.transpose(2, 3)) * st["scale"]).masked_fill_(~_visible(st), -math.inf)
    m = s.amax(3, keepdim=True)
    p = (s - m.masked_fill(m == -math.inf, 0)).exp_()
    z = p.sum(3, keepdim=True)
    return p / z.masked_fill(z == 0, 1), (m + z.log()).squeeze(3)


def _attention(st):
    case = st["case"]
    Tq, n = st["q"].shape[0], st["q_max"]
    if Tq == 0:
        return st["o"], st["lse"]
    if st["k"].shape[0] == 0:
        return torch.zeros_like(st["o"]), torch.full_like(st["lse"], -math.inf)
    q, k, v = _padded(st["q"], st["q_start"], n), _padded(st["k"], st["k_start"], st["k_max"]), _padded(st["v"], st["k_start"], st["k_max"])
    p, lse = _weights(st, q, _groups(k, case["Hq"]))
    o = p @ _groups(v, case["Hq"])
    return (_packed(o, st["q_start"], n, Tq).to(st["q"].dtype), _packed(lse.unsqueeze(3), st["q_start"], n, Tq)[:, :, 0].t().contiguous())


def _attention_backward(st):
    case = st["case"]
    Hq, Hkv, dt = case["Hq"], case["Hkv"], st["q"].dtype
    Tq, Tk, n, m = st["q"].shape[0], st["k"].shape[0], st["q_max"], st["k_max"]
    if Tq == 0 or Tk == 0:
        return [torch.zeros_like(st[x]) for x in ("dq", "dk", "dv")]
    q, do = _padded(st["q"], st["q_start"], n), _padded(st["do"], st["q_start"], n)
    k, v = _groups(_padded(st["k"], st["k_start"], m), Hq), _groups(_padded(st["v"], st["k_start"], m), Hq)
    p, _ = _weights(st, q, k)
    dp = do @ v.transpose(2, 3)
    dv = p.transpose(2, 3) @ do
    ds = p.mul_(dp.sub_((p * dp).sum(3, keepdim=True))).mul_(st["scale"])
    dq, dk = ds @ k, ds.transpose(2, 3) @ q
    shared = lambda x: x.view(x.shape[0], Hkv, Hq // Hkv, m, -1).sum(2)  # noqa: E731
    return [_packed(dq, st["q_start"], n, Tq).to(dt), _packed(shared(dk), st["k_start"], m, Tk).to(dt), _packed(shared(dv), st["k_start"], m, Tk).to(dt)]


def _attention_token(st):
    case = st["case"]
    B, Hq, Hkv, dh, cap = case["B"], case["Hq"], case["Hkv"], case["dh"], case["cap"]
    q = st["q"].float().view(B, Hkv, Hq // Hkv, dh)
    k, v = (st[x].view(B, cap, Hkv, dh).permute(0, 2, 1, 3).float() for x in ("k", "v"))
    live = (torch.arange(cap, device="cuda") < st["k_len"][:, None])[:, None, None]
    s = ((q @ k.transpose(2, 3)) * st["scale"]).masked_fill(~live, -math.inf)
    m = s.amax(3, keepdim=True)
    p = (s - m.masked_fill(m == -math.inf, 0)).exp()
    z = p.sum(3, keepdim=True)
    return ((p @ v) / z.masked_fill(z == 0, 1)).view(B, Hq, dh).to(st["q"].dtype)


def run(st):
    if own:
        return _run_own(st)
    case = st["case"]
    kind = case["kind"]
    if kind == "attention_token":
        return _attention_token(st)
    if kind == "attention":
        return list(_attention(st))
    if kind == "attention_backward":
        return _attention_backward(st)
    ids = st["ids"].long()
    if kind == "embed":
        x = st["table"][ids].float() * EMB_SCALE
        if case["P"]:
            x = x + st["pe"][st["pos"].long()]
        return x.to(DTYPES[case["out"]])
    g = torch.where((ids == 0)[:, None], 0.0, st["g"].float())
    grad = torch.zeros((case["V"], case["d"]), device="cuda").index_add_(0, ids, g)
    return (grad * EMB_SCALE).to(DTYPES[case["out"]])


# --------------------------------------------------------------------------- what a pass cannot do without
def _size(name):
    return 4 if name == "f32" else 2


def work(case):
    kind = case["kind"]
    if kind.startswith("attention"):
        ql, kl = _lengths(case)
        Hq, Hkv, dh = case["Hq"], case["Hkv"], case["dh"]
        q, k, pairs = 2 * sum(ql) * Hq * dh, 2 * sum(kl) * Hkv * dh, _pairs(case) * Hq
        if kind == "attention_token":
            return {"bytes": 2 * q + 2 * k, "flops": 4 * dh * pairs}
        lse = 4 * Hq * sum(ql)
        if kind == "attention":
            return {"bytes": 2 * q + 2 * k + lse, "flops": 4 * dh * pairs}
        return {"bytes": 4 * q + 4 * k + lse, "flops": 10 * dh * pairs}
    T, V, d, e, o = case["T"], case["V"], case["d"], _size(case["dtype"]), _size(case["out"])
    if kind == "embed":
        # distinct rows of the table are read once
        return {"bytes": 4 * T + min(T, V) * d * e + (4 * T + 4 * min(T, case["P"]) * d if case["P"] else 0) + T * d * o, "flops": T * d * (2 if case["P"] else 1)}
    return {"bytes": 4 * T + T * d * e + V * d * o, "flops": T * d}


# --------------------------------------------------------------------------- 64 bits
def _exact_attention(case, st, backward):
    ql, kl = _lengths(case)
    qs, ks = _starts(ql), _starts(kl)
    Hq, Hkv = case["Hq"], case["Hkv"]
    names = ("dq", "dk", "dv") if backward else ("o", "lse")
    res = {x: torch.zeros(st[x].shape, dtype=torch.float64, device="cuda") for x in names}
    if not backward:
        res["lse"].fill_(-math.inf)
    for b in range(case["B"]):
        r, c = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
        nq, nk = ql[b], kl[b]
        if nq == 0 or nk == 0:
            continue
        hidden = torch.ones((nq, nk), dtype=torch.bool, device="cuda").triu(nk - nq + 1) if case["causal"] else None
        for h in range(Hq):
            kv = h * Hkv // Hq
            q, k, v = st["q"][r, h].double(), st["k"][c, kv].double(), st["v"][c, kv].double()
            s = torch.mm(q, k.t()) * st["scale"]
            if hidden is not None:
                s[hidden] = -math.inf
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None])
            if not backward:
                res["lse"][h, r] = lse
                res["o"][r, h] = torch.mm(p, v)
                continue
            do = st["do"][r, h].double()
            dp = torch.mm(do, v.t())
            ds = p * (dp - (p * dp).sum(1, keepdim=True)) * st["scale"]
            res["dq"][r, h] = torch.mm(ds, k)
            res["dk"][c, kv] += torch.mm(ds.t(), q)
            res["dv"][c, kv] += torch.mm(p.t(), do)
    return [res[x] for x in names]


def exact(case, seed):
    kind = case["kind"]
    if kind.startswith("attention") and case["B"] * case["Hq"] > 3000 and kind != "attention_token":
        return None
    st = prepare(case, seed)
    if kind == "attention_token":
        _, kl = _lengths(case)
        Hq, Hkv, cap = case["Hq"], case["Hkv"], case["cap"]
        o = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        for b in range(case["B"]):
            if kl[b]:
                k, v = (st[x][b * cap:b * cap + kl[b]].double().repeat_interleave(Hq // Hkv, 1) for x in ("k", "v"))
                p = torch.softmax((k * st["q"][b].double()).sum(2) * st["scale"], 0)
                o[b] = (p[:, :, None] * v).sum(0)
        return o
    if kind.startswith("attention"):
        return _exact_attention(case, st, kind == "attention_backward")
    ids = st["ids"].long()
    if kind == "embed":
        x = torch.nn.functional.one_hot(ids, case["V"]).double() @ st["table"].double() if case["T"] * case["V"] < 10 ** 7 else st["table"].double()[ids]
        x = x * EMB_SCALE
        return x + st["pe"].double()[st["pos"].long()] if case["P"] else x
    order = torch.argsort(ids, stable=True)
    total = torch.cumsum(torch.cat([torch.zeros((1, case["d"]), dtype=torch.float64, device="cuda"), st["g"].double()[order]]), 0)
    count = torch.bincount(ids, minlength=case["V"])
    end = torch.cumsum(count, 0)
    grad = (total[end] - total[end - count]) * EMB_SCALE
    grad[0] = 0
    return grad
