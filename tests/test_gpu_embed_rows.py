"""The floating-point embedding and its gradient against plain forms in 64 bits."""
import pytest

torch = pytest.importorskip("torch")
from paper_2306_04235_gb300 import mnmt  # noqa: E402

pytestmark = pytest.mark.gpu
CODE = {torch.float32: mnmt.F32, torch.bfloat16: mnmt.BF16, torch.float16: mnmt.F16}
F32, BF, FP = CODE
SENTINEL = 5.0
SCALE = 16.0 * 2 ** 0.5


def matrix(rows, cols, dtype, pad=0, seed=0, spread=1.0, shift=0):
    """Random values as the leading columns of a buffer, `shift` elements after its start."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((rows * (cols + pad) + shift + 64,), SENTINEL, dtype=dtype, device="cuda")
    x = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)
    x[:, :cols] = (torch.randn((rows, cols), generator=g, device="cuda") * spread).to(dtype)
    return buf, x


def half_step(dtype):
    return torch.finfo(dtype).eps / 2, torch.finfo(dtype).tiny * torch.finfo(dtype).eps / 2


SIZES = [(1, 10, 8, 0, 0), (4, 8000, 384, 0, 0), (46, 300, 256, 8, 0), (300, 1000, 2048, 0, 0), (77, 50, 37, 3, 1), (1000, 7, 130, 0, 0), (513, 4000, 515, 5, 3),
         (2000, 100, 1024, 0, 0), (64, 64, 1, 0, 0)]


@pytest.mark.parametrize("T,V,d,pad,shift", SIZES)
@pytest.mark.parametrize("dtype,otype", [(F32, F32), (BF, F32), (FP, BF), (BF, BF), (F32, FP)])
@pytest.mark.parametrize("positions", ["none", "given", "row"])
def test_embed(T, V, d, pad, shift, dtype, otype, positions):
    _, table = matrix(V, d, dtype, pad, 1, shift=shift)
    P = T + 5
    _, pe = matrix(P, d, F32, pad, 2)
    g = torch.Generator(device="cuda").manual_seed(3)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    pos = torch.randint(0, P, (T,), generator=g, device="cuda", dtype=torch.int32)
    buf, out = matrix(T, d, otype, pad, 4, shift=shift)
    before = buf.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = {} if positions == "none" else dict(pe=pe, ldpe=d + pad, P=P, pos=pos if positions == "given" else None)
    mnmt.mnmt_embed(ids, T, table, CODE[dtype], d + pad, V, d, SCALE, out, CODE[otype], d + pad, status=status, **kw)
    torch.cuda.synchronize()
    assert int(status) == 0
    # two fp32 roundings of 2^-24 each, then the output's
    want = (table[ids.long(), :d].double() * torch.tensor(SCALE, dtype=F32).double()).float()
    if positions != "none":
        want = want + pe[pos.long() if positions == "given" else torch.arange(T, device="cuda"), :d]
    assert torch.equal(out[:, :d], want.to(otype)), "not the formula's own roundings"
    keep = torch.ones_like(buf, dtype=torch.bool)
    keep[shift:shift + T * (d + pad)].view(T, d + pad)[:, :d] = False
    assert torch.equal(buf[keep], before[keep]), "written beside the output"


def test_embed_bad_ids():
    _, table = matrix(50, 64, BF)
    _, pe = matrix(9, 64, F32, seed=5)
    ids = torch.tensor([3, -1, 49, 50, 2 ** 31 - 1, -2 ** 31, 0, 1], dtype=torch.int32, device="cuda")
    pos = torch.tensor([0, 1, 2, 3, 4, 5, 9, -1], dtype=torch.int32, device="cuda")
    _, out = matrix(8, 64, F32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mnmt.mnmt_embed(ids, 8, table, mnmt.BF16, 64, 50, 64, 2.0, out, mnmt.F32, 64, pos, pe, 64, 9, status)
    assert int(status) == mnmt.EINVAL
    want = torch.zeros((8, 64), device="cuda")
    for t in (0, 2):
        want[t] = table[ids[t]].float() * 2.0 + pe[pos[t]]
    assert torch.equal(out, want)


def test_embed_offsets_past_32_bits():
    """A table of more than 2^32 bytes, and 2^31 elements."""
    V, d = (1 << 31) // 4096 + 3, 4096
    table = torch.zeros((V, d), dtype=BF, device="cuda")
    ids = torch.tensor([V - 1, 0, V - 2], dtype=torch.int32, device="cuda")
    table[V - 1], table[V - 2] = 3.0, 2.0
    out = torch.empty((3, d), dtype=BF, device="cuda")
    mnmt.mnmt_embed(ids, 3, table, mnmt.BF16, d, V, d, 1.0, out, mnmt.BF16, d)
    torch.cuda.synchronize()
    assert [float(x) for x in out.float().mean(1)] == [3.0, 0.0, 2.0]


def plain_gradient(ids, g, V, scale, pad_id, out, accumulate, otype):
    """The gradient in 64 bits, and its bound: additions of n terms in fp32 (2^-24 each of the sum of magnitudes, in chains
    that are no longer than n), the scale's rounding, the addition to what was there, and the output's."""
    ids = ids.cpu().long()
    use = (ids >= 0) & (ids < V) & (ids != pad_id)
    g = g.cpu().double()[use]
    want, mag = (torch.zeros((V, g.shape[1]), dtype=torch.float64) for _ in range(2))
    n = torch.bincount(ids[use], minlength=V)[:, None]
    want.index_add_(0, ids[use], g)
    mag.index_add_(0, ids[use], g.abs())
    s = float(torch.tensor(scale, dtype=F32))
    base = out.cpu().double() if accumulate else 0.0
    total = base + s * want
    u, z = half_step(otype)
    return total, s * mag * (n + 2) * 2.0 ** -24 + 2.0 ** -24 * (total.abs() + (s * want).abs()) + u * total.abs() * (1 + 2.0 ** -20) + z


@pytest.mark.parametrize("T,V,d,pad,shift", SIZES + [(20000, 3000, 64, 0, 0), (5000, 2, 96, 0, 0), (40000, 70000, 16, 0, 0), (0, 30, 40, 2, 0)])
@pytest.mark.parametrize("dtype,otype", [(F32, F32), (BF, F32), (FP, BF), (BF, FP)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_backward(T, V, d, pad, shift, dtype, otype, accumulate):
    gen = torch.Generator(device="cuda").manual_seed(3)
    u = torch.rand(T, generator=gen, device="cuda")
    ids = (torch.exp(u * float(torch.log(torch.tensor(V + 1.0)))) - 1).clamp(0, V - 1).to(torch.int32)  # a few tokens are very frequent
    _, g = matrix(T, d, dtype, pad, 5, shift=shift)
    buf, out = matrix(V, d, otype, pad, 6, shift=shift)
    before = buf.clone()
    pad_id = 1 if V > 8 else -1
    want, bound = plain_gradient(ids, g[:, :d], V, SCALE, pad_id, out[:, :d], accumulate, otype)
    ws_size = mnmt.mnmt_embed_backward_workspace(T, V, d)
    ws = torch.full((ws_size + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mnmt.mnmt_embed_backward(ids, T, g, CODE[dtype], d + pad, SCALE, pad_id, V, d, out, CODE[otype], d + pad, accumulate, ws, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    err = (out[:, :d].cpu().double() - want).abs()
    assert bool((err <= bound).all()), f"{int((err > bound).sum())} off, worst {float((err / bound.clamp_min(1e-300)).max())} bounds"
    keep = torch.ones_like(buf, dtype=torch.bool)
    keep[shift:shift + V * (d + pad)].view(V, d + pad)[:, :d] = False
    assert torch.equal(buf[keep], before[keep]), "written beside the gradient"
    assert bool((ws[ws_size:] == 0xFF).all()), "written behind the workspace"
    if accumulate and T:
        untouched = torch.ones(V, dtype=torch.bool)
        untouched[ids.cpu().long()] = False
        if pad_id >= 0:
            untouched[pad_id] = True
        assert torch.equal(out.cpu()[untouched], before[shift:shift + V * (d + pad)].view(V, d + pad).cpu()[untouched])


def test_embed_backward_one_token_everywhere():
    """Every token the same: one long sum."""
    T, V, d = 30000, 100, 72
    ids = torch.full((T,), 42, dtype=torch.int32, device="cuda")
    _, g = matrix(T, d, BF, seed=8)
    out = torch.empty((V, d), device="cuda")
    ws = torch.empty(mnmt.mnmt_embed_backward_workspace(T, V, d), dtype=torch.uint8, device="cuda")
    mnmt.mnmt_embed_backward(ids, T, g, mnmt.BF16, d, 1.0, -1, V, d, out, mnmt.F32, d, False, ws)
    torch.cuda.synchronize()
    want, bound = plain_gradient(ids, g, V, 1.0, -1, out, False, F32)
    assert bool(((out.cpu().double() - want).abs() <= bound).all())


def test_embed_backward_large_numbers():
    """Numbers of tokens that take four passes of the sort, rows behind 2^32 bytes, added to what is there."""
    V, d, T = (1 << 28) + 77, 8, 9000
    gen = torch.Generator(device="cuda").manual_seed(2)
    ids = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    ids[::50] = V - 1
    ids[1::70] = 3
    _, g = matrix(T, d, F32, seed=9)
    out = torch.zeros((V, d), dtype=BF, device="cuda")
    ws = torch.empty(mnmt.mnmt_embed_backward_workspace(T, V, d), dtype=torch.uint8, device="cuda")
    mnmt.mnmt_embed_backward(ids, T, g, mnmt.F32, d, 1.0, -1, V, d, out, mnmt.BF16, d, True, ws)
    torch.cuda.synchronize()
    names, back = torch.unique(ids.long(), return_inverse=True)
    want = torch.zeros((len(names), d), dtype=torch.float64, device="cuda").index_add_(0, back, g.double())
    mag = torch.zeros_like(want).index_add_(0, back, g.double().abs())
    got = out[names].double()
    assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + T * 2.0 ** -24 * mag).all())
    out[names] = 0
    assert not bool(out.any())


def test_embed_backward_bad_ids():
    ids = torch.tensor([3, -1, 49, 50, 2 ** 31 - 1, -2 ** 31, 3, 0], dtype=torch.int32, device="cuda")
    _, g = matrix(8, 64, F32, seed=7)
    out = torch.full((50, 64), SENTINEL, device="cuda")
    ws = torch.empty(mnmt.mnmt_embed_backward_workspace(8, 50, 64), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mnmt.mnmt_embed_backward(ids, 8, g, mnmt.F32, 64, 1.0, 0, 50, 64, out, mnmt.F32, 64, False, ws, status)
    assert int(status) == mnmt.EINVAL
    want = torch.zeros((50, 64), device="cuda")
    want[3], want[49] = g[0] + g[6], g[2]
    assert torch.equal(out, want)


def test_embed_backward_runs_alike_and_replays():
    """The same bits twice, on two streams at once with a workspace each, and from a graph on new ids."""
    T, V, d = 6000, 500, 256
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids = [torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32) // 7 for _ in range(2)]
    _, g = matrix(T, d, BF, seed=2)
    outs, wss = [torch.empty((V, d), device="cuda") for _ in range(2)], [
        torch.empty(mnmt.mnmt_embed_backward_workspace(T, V, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()

    def go(i, st):
        mnmt.mnmt_embed_backward(ids[i], T, g, mnmt.BF16, d, 1.0, -1, V, d, outs[i], mnmt.F32, d, False, wss[i], None, st)

    for _ in range(4):
        for i in range(2):
            go(i, streams[i])
    torch.cuda.synchronize()
    first = [x.clone() for x in outs]
    for i in range(2):
        go(i, streams[0])
    torch.cuda.synchronize()
    assert torch.equal(first[0], outs[0]) and torch.equal(first[1], outs[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=streams[0]):
        go(0, streams[0])
    ids[0].copy_(ids[1])
    for _ in range(2):
        outs[0].fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], first[1])
