"""Performance cases of the 4-bit floating-point operators and of dropout.

The operators, as a user of the library calls them:

* `quantize`: fake quantisation to microscaled 4-bit floating point (E2M1 codes; MX: a power-of-two scale per 32
  elements of a row, NV: an E4M3 scale per 16 and one fp32 scale per tensor), and its straight-through backward pass;
* `linear`: activations quantised in the call, multiplied with packed 4-bit weights, bias and ReLU in the epilogue;
* `linear_backward`: the gradients of input, weights and bias of that linear for bf16 output gradients;
* `dropout`: counter-based dropout (Philox4x32-10) with optional ReLU and the sublayer's residual
  `out = gamma r + D(x)`, and its backward pass, which draws the same numbers again.

`own = False` computes each operator in its plain form: elementary torch operations in 32 bits, rounded once at the end.

Packed operands are in the library's documented form.  Codes: [rows][ceil(K / 32) 16] bytes, element 2j of a row in the
low half of byte j.  Scales: tiles of 128 rows and 4 blocks, 512 bytes each, tile (row / 128, block / 4) row-major,
byte 16 (row % 32) + 4 (row % 128 / 32) + block % 4 of its tile.  Padding is zero.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = {"mx": 32, "nv": 16}
GAMMA = 0.75


def listed():
    return [
        # the activations of one decode step (the four beams of one sentence), in front of any product: latency
        dict(name="quantize_token", kind="quantize", format="mx", dtype="bf16", M=4, K=512, pad=0),
        # the hidden activations of a training batch of 128 sentences of 128 tokens
        dict(name="quantize_batch", kind="quantize", format="mx", dtype="bf16", M=16384, K=2048, pad=0),
        # straight-through gradient of an fp32 master embedding whose width is no multiple of a block
        dict(name="quantize_backward", kind="quantize_backward", format="nv", dtype="f32", M=8000, K=509, pad=3),
        # serving one sentence, greedy: the first FFN layer for one token
        dict(name="linear_token", kind="linear", format="mx", dtype="bf16", out="bf16", relu=True, M=1, N=2048, K=512, pad=0),
        # serving a batch: logits of 128 sentences with four beams over the vocabulary
        dict(name="linear_vocab", kind="linear", format="nv", dtype="bf16", out="f32", relu=False, M=512, N=32000, K=512, pad=0),
        # a layer of odd widths on a ragged batch, rows inside a wider buffer
        dict(name="linear_ragged", kind="linear", format="nv", dtype="f16", out="f16", relu=False, M=1001, N=771, K=389, pad=11),
        # the largest product: an FFN layer of the widest model over a training batch
        dict(name="linear_batch", kind="linear", format="mx", dtype="bf16", out="bf16", relu=True, M=16384, N=8192, K=2048, pad=0),
        # training on one sentence (fine-tuning): the gradients of an FFN layer for 46 tokens
        dict(name="backward_sentence", kind="linear_backward", format="nv", dtype="bf16", M=46, N=1024, K=256, pad=0),
        # the gradients of the largest product
        dict(name="backward_batch", kind="linear_backward", format="mx", dtype="bf16", M=16384, N=8192, K=2048, pad=0),
        # the hidden units of one sentence of 30 tokens: ReLU, then dropout
        dict(name="dropout_sentence", kind="dropout", dtype="bf16", relu=True, residual=False, p=0.1, M=30, K=768, pad=0),
        # the end of a sublayer over a training batch: dropout onto the fp32 residual stream
        dict(name="dropout_residual", kind="dropout", dtype="bf16", relu=False, residual=True, p=0.1, M=16384, K=2048, pad=0),
        # the same backward, ragged rows, with the gradients of the residual and of its learned gain
        dict(name="dropout_backward", kind="dropout_backward", dtype="f16", relu=True, residual=True, p=0.3, M=5003, K=1001, pad=7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "quantize_backward", "linear", "linear", "linear", "linear_backward", "linear_backward",
                       "dropout", "dropout_backward"])
    case = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), pad=rng.choice([0, 0, 0, 8, rng.randint(1, 40)]))
    if kind.startswith("linear"):
        backward = kind == "linear_backward"
        M, N, K = _log(rng, 1, 16384), _log(rng, 64, 32000), _log(rng, 64, 8192)
        if rng.random() < 0.5:  # half of them in steps of 32, as the widths of layers are
            N, K = max(64, N // 160 * 160), max(64, K // 160 * 160)
        while M * N * K > 16384 * 8192 * 2048 or (M * N > 16384 * 8192):
            M = max(1, M // 2)
        case |= dict(format=rng.choice(["mx", "nv"]), M=M, N=N, K=K)
        if not backward:
            case |= dict(out=rng.choice(["bf16", "f32", "f16"]), relu=rng.random() < 0.5)
        return case
    M, K = _log(rng, 1, 16384), _log(rng, 16, 8192)
    while M * K > 16384 * 2048:
        M = max(1, M // 2)
    if kind.startswith("quantize"):
        return case | dict(format=rng.choice(["mx", "nv"]), M=M, K=K)
    residual = rng.random() < 0.6
    return case | dict(relu=rng.random() < 0.5, residual=residual, p=rng.choice([0.0, 0.1, 0.1, 0.3, round(rng.random(), 3)]), M=M, K=K)


# --------------------------------------------------------------------------- formats
_tables = {}


def _table(name):
    """fp32 values of a byte: "mx" scales, their inverses "mx_inv", "nv" scales, and the 16 codes "e2m1"."""
    if name not in _tables:
        b = np.arange(256)
        if name == "e2m1":
            v = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
            v = np.concatenate([v, -v])
        elif name == "nv":
            e, m = (b >> 3) & 15, b & 7
            v = np.where(e == 0, np.ldexp(m / 8, -6), np.ldexp(1 + m / 8, e - 7)) * np.where(b & 128, -1, 1)
            v = np.where((b & 127) == 127, np.nan, v)
        else:
            v = np.where(b == 255, np.nan, np.ldexp(1.0, 127 - b if name == "mx_inv" else b - 127))
        _tables[name] = torch.from_numpy(v.astype(np.float32)).cuda()
    return _tables[name]


def _blocks(x, block):
    """[rows][K] as [rows][blocks][block], zeros at the end."""
    rows, K = x.shape
    pad = -K % block
    if pad:
        x = torch.nn.functional.pad(x, (0, pad))
    return x.view(rows, -1, block)


def _e2m1(t):
    """fp32 values of the nearest 4-bit codes, ties to even, beyond 6 held at 6."""
    a = t.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign(((a / step).round() * step).clamp_max(6), t)


def _scales(x, format, g):
    """Scale byte, fp32 scale S and its inverse r of every block of fp32 x [rows][blocks][block]."""
    a = x.abs().amax(2)
    bad = ~torch.isfinite(a)
    a = torch.where(bad, torch.ones_like(a), a)
    if format == "mx":
        byte = torch.where(a > 0, (torch.frexp(a)[1] - 3).clamp(-127, 127), -127) + 127
        byte = torch.where(bad, 255, byte)
        return byte, _table("mx")[byte], _table("mx_inv")[byte]
    c = float(np.float32(1) / (np.float32(6) * np.float32(g)))
    v = (a * c).clamp_max(448)
    e = torch.frexp(v)[1].clamp_min(-5)  # v in [2^(e-1), 2^e): three bits after the first, from 2^-9 on
    step = torch.ldexp(torch.ones_like(v), e - 4)
    n = (v / step).round() * step
    m, e = torch.frexp(n)
    normal = n >= 2.0 ** -6
    byte = torch.where(normal, ((e + 6) << 3) + (m * 16 - 8).to(torch.int32), (n * 512).to(torch.int32))
    byte = torch.where(bad, 127, byte)
    s = _table("nv")[byte] * float(np.float32(g))
    return byte, s, torch.where(s == 0, torch.zeros_like(s), 1 / s)


def _quantized(x, format, g):
    """Scale bytes [rows][blocks], codes as fp32 [rows][blocks][block], and values [rows][K] of fp32 x."""
    b = _blocks(x, BLOCK[format])
    byte, s, r = _scales(b, format, g)
    t = torch.where(torch.isfinite(s)[:, :, None], b * r[:, :, None], torch.zeros_like(b))
    q = _e2m1(t)
    return byte, q, (q * s[:, :, None]).view(x.shape[0], -1)[:, :x.shape[1]]


def _pack(x, format, g):
    """The packed form of fp32 x: codes and scales, as the library documents them."""
    rows, K = x.shape
    byte, q, _ = _quantized(x, format, g)
    mag = torch.bucketize(q.abs(), _table("e2m1")[:8].contiguous())
    code = (mag + 8 * (torch.signbit(q) & (mag > 0))).to(torch.uint8).view(rows, -1)
    code = torch.nn.functional.pad(code, (0, -(-K // 32) * 32 - code.shape[1]))
    nb = byte.shape[1]
    rt, bt = -(-rows // 128), -(-nb // 4)
    s = torch.nn.functional.pad(byte.to(torch.uint8), (0, bt * 4 - nb, 0, rt * 128 - rows))
    s = s.view(rt, 4, 32, bt, 4).permute(0, 3, 2, 1, 4).contiguous()
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), s.view(-1)


def _scale_bytes(scales, rows, nb):
    rt, bt = -(-rows // 128), -(-nb // 4)
    return scales.view(rt, bt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, bt * 4)[:rows, :nb].to(torch.int32)


def _unpack(codes, scales, rows, K, format, g):
    """Values [rows][K] and inverse scales [rows][blocks] of a packed matrix, fp32."""
    block = BLOCK[format]
    nb = -(-K // block)
    q = torch.stack([codes & 15, codes >> 4], 2).view(rows, -1)[:, :nb * block].to(torch.int32)
    byte = _scale_bytes(scales, rows, nb)
    if format == "mx":
        s, r = _table("mx")[byte], _table("mx_inv")[byte]
    else:
        s = _table("nv")[byte] * float(np.float32(g))
        r = torch.where(s == 0, torch.zeros_like(s), 1 / s)
    v = _table("e2m1")[q].view(rows, nb, block) * s[:, :, None]
    return v.view(rows, -1)[:, :K], r


def _inside(x, r, block):
    """Whether fp32 x [rows][K] lies within its block's range: the straight-through mask."""
    t = _blocks(x, block) * r[:, :, None]
    return (t.abs() <= 6).view(x.shape[0], -1)[:, :x.shape[1]]


# --------------------------------------------------------------------------- counter-based generator
_M32 = 0xFFFFFFFF


def _mulhilo(a, b):
    """High and low word of the product of 32-bit numbers held in int64."""
    h, l = a * (b >> 16), a * (b & 0xFFFF)
    return (h + (l >> 16)) >> 16, (((h & 0xFFFF) << 16) + l) & _M32


def _fields(rows, K, seed, offset):
    """16-bit numbers [rows][K] of Philox4x32-10: counter {c / 8, row, offset}, key seed."""
    c0 = torch.arange(-(-K // 8), device="cuda").expand(rows, -1)
    c1 = torch.arange(rows, device="cuda")[:, None].expand_as(c0)
    c2 = torch.full_like(c0, offset & _M32)
    c3 = torch.full_like(c0, offset >> 32)
    k0, k1 = seed & _M32, seed >> 32
    for _ in range(10):  # the rounds of the generator
        h0, l0 = _mulhilo(0xD2511F53, c0)
        h1, l1 = _mulhilo(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    w = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], 2)
    return w.view(rows, -1)[:, :K]


def _threshold(p):
    """p in units of 2^-16, and the fp32 factor of what is kept."""
    thr = int(np.rint(np.float32(p) * np.float32(65536)))
    return thr, float(np.float32(65536) / np.float32(65536 - thr)) if thr < 65536 else 0.0


# --------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _strided(x, dtype, pad):
    """x in its type, as the leading columns of a buffer `pad` columns wider."""
    buf = torch.empty((x.shape[0], x.shape[1] + pad), dtype=dtype, device="cuda")
    buf[:, :x.shape[1]] = x
    return buf[:, :x.shape[1]]


def _activations(g, M, K):
    """Outputs of a LayerNorm: unit normals with gains of their own, a few channels much larger than the rest."""
    gain = 1 + 0.2 * _normal(g, K)
    gain = torch.where(torch.rand(K, generator=g, device="cuda") < 0.01, gain * 12, gain)
    return _normal(g, M, K) * gain


G_X = float(np.float32(48 / 2688))   # tensor scales as a calibration run leaves them
G_W = float(np.float32(0.1 / 2688))


def prepare(case, seed):
    g = _gen(seed)
    dt, M, K, pad = DTYPES[case["dtype"]], case["M"], case["K"], case["pad"]
    st = {"case": case, "ldx": K + pad}
    kind = case["kind"]
    if kind in ("quantize", "quantize_backward"):
        st["x"] = _strided(_activations(g, M, K), dt, pad)
        if kind == "quantize_backward":
            st["g"] = _strided(_normal(g, M, K) * 1e-3, dt, pad)
        st["y"] = _strided(torch.zeros((M, K), device="cuda"), dt, pad)
        # room for the packed form, which the forward pass writes beside the values
        st["codes"] = torch.empty((M, -(-K // 32) * 16), dtype=torch.uint8, device="cuda")
        st["scales"] = torch.empty(-(-M // 128) * -(-(-(-K // BLOCK[case["format"]])) // 4) * 512, dtype=torch.uint8, device="cuda")
        return st
    if kind in ("linear", "linear_backward"):
        N, f = case["N"], case["format"]
        w = _normal(g, N, K) * 0.02
        st["w_codes"], st["w_scales"] = _pack(w, f, G_W)
        st["x"] = _strided(_activations(g, M, K), dt, pad)
        if kind == "linear":
            st["bias"] = _normal(g, N) * 0.02
            st["x_codes"] = torch.empty((M, -(-K // 32) * 16), dtype=torch.uint8, device="cuda")
            st["x_scales"] = torch.empty(-(-M // 128) * -(-(-(-K // BLOCK[f])) // 4) * 512, dtype=torch.uint8, device="cuda")
            st["y"] = _strided(torch.zeros((M, N), device="cuda"), DTYPES[case["out"]], pad)
        else:
            st["w"] = w
            st["x_codes"], st["x_scales"] = _pack(st["x"].float(), f, G_X)
            st["g"] = _strided(_normal(g, M, N) * (torch.rand((M, 1), generator=g, device="cuda") * 1e-3 + 1e-4), torch.bfloat16, pad)
            st["gx"] = _strided(torch.zeros((M, K), device="cuda"), dt, pad)
            st["gw"], st["gb"] = torch.empty((N, K), device="cuda"), torch.empty(N, device="cuda")
        return st
    st["seed"], st["offset"] = (int(seed) * 0x9E3779B97F4A7C15 + 12345) & (2 ** 64 - 1), (int(seed) * 7919 + 5) & (2 ** 40 - 1)
    st["x"] = _strided(_normal(g, M, K), dt, pad)
    if case["residual"]:
        st["r"] = _normal(g, M, K) + 0.5
    # with a residual the output (and its gradient) is the fp32 residual stream, else it has the input's type
    odt = torch.float32 if case["residual"] else dt
    opad = 0 if case["residual"] else pad
    if kind == "dropout":
        st["out"] = _strided(torch.zeros((M, K), device="cuda"), odt, opad)
    else:
        st["g"] = _strided(_normal(g, M, K) * 1e-2 + (st["r"] * 1e-3 if case["residual"] else 0), odt, opad)
        st["gx"] = _strided(torch.zeros((M, K), device="cuda"), dt, pad)
        if case["residual"]:
            st["gr"], st["ggamma"] = torch.empty((M, K), device="cuda"), torch.empty(1, device="cuda")
    return st


# --------------------------------------------------------------------------- one pass
def _run_own(st):
    from paper_2306_04235_gb300 import mnmt

    case = st["case"]
    kind, M, K, ldx = case["kind"], case["M"], case["K"], st["ldx"]
    types = {"f32": mnmt.F32, "bf16": mnmt.BF16, "f16": mnmt.F16}
    dt = types[case["dtype"]]
    if kind in ("quantize", "quantize_backward"):
        f = mnmt.FP4_MX if case["format"] == "mx" else mnmt.FP4_NV
        q = mnmt.Fp4(M, K, f, G_X, st["codes"], st["scales"])
        if kind == "quantize":
            mnmt.mnmt_fp4_quantize(q, st["x"], dt, ldx, st["y"], ldx)
        else:
            mnmt.mnmt_fp4_quantize_backward(q, st["x"], dt, ldx, st["g"], ldx, st["y"], ldx)
        return st["y"]
    if kind in ("linear", "linear_backward"):
        N = case["N"]
        f = mnmt.FP4_MX if case["format"] == "mx" else mnmt.FP4_NV
        xq = mnmt.Fp4(M, K, f, G_X, st["x_codes"], st["x_scales"])
        wq = mnmt.Fp4(N, K, f, G_W, st["w_codes"], st["w_scales"])
        if kind == "linear":
            mnmt.mnmt_fp4_linear(xq, wq, st["x"], dt, ldx, st["bias"], case["relu"], st["y"], types[case["out"]], N + case["pad"])
            return st["y"]
        ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(M, N, K), dtype=torch.uint8, device="cuda")
        mnmt.mnmt_fp4_linear_backward(xq, wq, st["g"], N + case["pad"], st["x"], dt, ldx, st["w"], mnmt.F32, K, ws,
                                      st["gx"], ldx, st["gw"], K, st["gb"])
        return [st["gx"], st["gw"], st["gb"]]
    res = case["residual"]
    rdt, ldo = (mnmt.F32, K) if res else (dt, ldx)
    if kind == "dropout":
        mnmt.mnmt_dropout(st["x"], dt, ldx, st["r"] if res else None, K, GAMMA, case["p"], st["seed"], st["offset"], case["relu"],
                          M, K, st["out"], rdt, ldo)
        return st["out"]
    ws = torch.empty(mnmt.DROPOUT_WORKSPACE, dtype=torch.uint8, device="cuda") if res else None
    mnmt.mnmt_dropout_backward(st["g"], rdt, ldo, st["x"], dt, ldx, st["r"] if res else None, K, GAMMA, case["p"], st["seed"],
                               st["offset"], case["relu"], M, K, st["gx"], ldx, st["gr"] if res else None, K,
                               st["ggamma"] if res else None, ws)
    return [st["gx"], st["gr"], st["ggamma"]] if res else [st["gx"]]


def run(st):
    if own:
        return _run_own(st)
    case = st["case"]
    kind, M, K = case["kind"], case["M"], case["K"]
    dt = DTYPES[case["dtype"]]
    x = st["x"].float()
    if kind == "quantize":
        return _quantized(x, case["format"], G_X)[2].to(dt)
    if kind == "quantize_backward":
        block = BLOCK[case["format"]]
        _, _, r = _scales(_blocks(x, block), case["format"], G_X)
        return torch.where(_inside(x, r, block), st["g"], torch.zeros_like(st["g"]))
    if kind == "linear":
        xv = _quantized(x, case["format"], G_X)[2]
        wv, _ = _unpack(st["w_codes"], st["w_scales"], case["N"], K, case["format"], G_W)
        y = xv @ wv.t() + st["bias"]
        return (torch.relu(y) if case["relu"] else y).to(DTYPES[case["out"]])
    if kind == "linear_backward":
        block = BLOCK[case["format"]]
        xv, xr = _unpack(st["x_codes"], st["x_scales"], M, K, case["format"], G_X)
        wv, wr = _unpack(st["w_codes"], st["w_scales"], case["N"], K, case["format"], G_W)
        g = st["g"].float()
        gx = torch.where(_inside(x, xr, block), g @ wv, 0.0)
        gw = torch.where(_inside(st["w"], wr, block), g.t() @ xv, 0.0)
        return [gx.to(dt), gw, g.sum(0)]
    thr, s = _threshold(case["p"])
    keep = _fields(M, K, st["seed"], st["offset"]) >= thr
    if kind == "dropout":
        v = torch.relu(x) if case["relu"] else x
        v = torch.where(keep, v * s, torch.zeros_like(v))
        return st["r"] * GAMMA + v if case["residual"] else v.to(dt)
    if case["relu"]:
        keep = keep & (x > 0)
    g = st["g"].float()
    gx = torch.where(keep, g * s, torch.zeros_like(g)).to(dt)
    return [gx, g * GAMMA, (g * st["r"]).sum().view(1)] if case["residual"] else [gx]


# --------------------------------------------------------------------------- what a pass cannot do without
def _size(name):
    return 4 if name == "f32" else 2


def work(case):
    M, K, e = case["M"], case["K"], _size(case["dtype"])
    kind = case["kind"]
    if kind == "quantize":
        return {"bytes": M * K * (2 * e + 0.5 + 1 / BLOCK[case["format"]]), "flops": 3 * M * K}
    if kind == "quantize_backward":
        return {"bytes": M * K * 3 * e, "flops": 3 * M * K}
    if kind in ("linear", "linear_backward"):
        N, packed = case["N"], 0.5 + 1 / BLOCK[case["format"]]
        if kind == "linear":
            return {"bytes": M * K * (e + packed) + N * K * packed + 4 * N + M * N * _size(case["out"]), "flops": 2 * M * N * K}
        return {"bytes": 2 * M * N + M * K * (packed + 2 * e) + N * K * (packed + 8) + 4 * N, "flops": 4 * M * N * K}
    r = 4 if case["residual"] else 0
    if kind == "dropout":
        return {"bytes": M * K * (e + r + (4 if r else e)), "flops": 4 * M * K}
    return {"bytes": M * K * ((e if case["relu"] else 0) + (4 if r else e) + 2 * r + e), "flops": 5 * M * K}


# --------------------------------------------------------------------------- 64 bits
def _exact_scale(x, format, g):
    """Block scale in float64, inverse as the definition rounds it to fp32, of float64 x [rows][blocks][block]."""
    a = x.abs().amax(2)
    if format == "mx":
        # floor(log2 a) from the exponent field; every fp32, bf16 and fp16 number is a normal float64
        e = ((a.view(torch.int64) >> 52) - 1023 - 2).clamp(-127, 127)
        s = (torch.where(a > 0, e, -127) + 1023 << 52).view(torch.float64)
        return s, 1 / s
    g32 = np.float32(g)
    inv = float(np.float32(1.0 / float(np.float32(6.0 * float(g32)))))
    v = (a * inv).float().double()
    lattice = torch.from_numpy(np.concatenate([np.arange(8) / 512, np.ldexp((8 + np.arange(119) % 8) / 8, np.arange(119) // 8 - 6)[:119]])).cuda()
    lattice = lattice[lattice <= 448]
    mid = (lattice[1:] + lattice[:-1]) / 2
    # index of the nearest number of the lattice; a tie goes to the even index (the even mantissa)
    lo, hi = torch.bucketize(v, mid), torch.bucketize(v, mid, right=True)
    s = (lattice[torch.where(lo % 2 == 0, lo, hi)] * float(g32)).float().double()
    return s, torch.where(s > 0, 1 / s, 0).float().double()


def _exact_quantized(x, format, g):
    rows, K = x.shape
    block = BLOCK[format]
    nb = -(-K // block)
    b = torch.zeros((rows, nb * block), dtype=torch.float64, device=x.device)
    b[:, :K] = x
    b = b.view(rows, nb, block)
    s, r = _exact_scale(b, format, g)
    t = (b * r[:, :, None]).float().double()
    a = t.abs()
    idx = sum((a > m).to(torch.int8) for m in (0.25, 1.25, 2.5, 5.0)) + sum((a >= m).to(torch.int8) for m in (0.75, 1.75, 3.5))
    mag = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)[idx.long()]
    v = torch.sign(t) * mag * s[:, :, None]
    return v.reshape(rows, -1)[:, :K], (a <= 6).reshape(rows, -1)[:, :K]


def _exact_fields(rows, K, seed, offset):
    """The generator in unsigned 64-bit integers of numpy: [rows][K] of 16-bit numbers."""
    n = -(-K // 8)
    u, m = np.uint64, np.uint64(_M32)
    c = [np.tile(np.arange(n, dtype=u), (rows, 1)), np.tile(np.arange(rows, dtype=u)[:, None], (1, n)),
         np.full((rows, n), offset & _M32, u), np.full((rows, n), offset >> 32, u)]
    for i in range(10):
        k0, k1 = u(((seed & _M32) + i * 0x9E3779B9) & _M32), u(((seed >> 32) + i * 0xBB67AE85) & _M32)
        p0, p1 = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(p1 >> u(32)) ^ c[1] ^ k0, p1 & m, (p0 >> u(32)) ^ c[3] ^ k1, p0 & m]
    out = np.empty((rows, n, 8), np.uint16)
    for i in range(4):
        out[:, :, 2 * i] = c[i] & u(0xFFFF)
        out[:, :, 2 * i + 1] = c[i] >> u(16)
    return torch.from_numpy(out.reshape(rows, -1)[:, :K].astype(np.int32)).cuda()


def exact(case, seed):
    st = prepare(case, seed)
    kind, M, K = case["kind"], case["M"], case["K"]
    x = st["x"].double()
    if kind == "quantize":
        return _exact_quantized(x, case["format"], G_X)[0]
    if kind == "quantize_backward":
        return st["g"].double() * _exact_quantized(x, case["format"], G_X)[1]
    if kind in ("linear", "linear_backward"):
        # the float weights again, from the same generator
        w = (_normal(_gen(seed), case["N"], K) * 0.02).double()
        (xv, xin), (wv, win) = _exact_quantized(x, case["format"], G_X), _exact_quantized(w, case["format"], G_W)
        if kind == "linear":
            y = torch.addmm(st["bias"].double(), xv, wv.t())
            return y.clamp_min(0) if case["relu"] else y
        g = st["g"].double()
        return [(g @ wv) * xin, (g.t() @ xv) * win, g.sum(0)]
    f = _exact_fields(M, K, st["seed"], st["offset"])
    thr = int(np.rint(float(np.float32(case["p"])) * 65536))
    scale = float(np.float32(65536 / (65536 - thr))) if thr < 65536 else 0.0
    live = f >= thr
    if case["relu"]:
        live &= x > 0
    if kind == "dropout":
        v = x * scale * live
        return st["r"].double() * GAMMA + v if case["residual"] else v
    g = st["g"].double()
    gx = g * scale * live
    return [gx, g * GAMMA, (g * st["r"].double()).sum().view(1)] if case["residual"] else [gx]
