"""The table gradient without tokens, and into tables of more rows than a block of the zeroing kernel marks at a time."""
import pytest

torch = pytest.importorskip("torch")
from paper_2306_04235_gb300 import mnmt  # noqa: E402

pytestmark = pytest.mark.gpu
CODE = {torch.float32: mnmt.F32, torch.bfloat16: mnmt.BF16, torch.float16: mnmt.F16}
SENTINEL = 5.0
# 4 x 152 sets of rows and 4096 rows a block are what one launch takes with up to 256 columns
FEW_ROWS = 4 * 152 * 4096


def backward(ids, T, g, V, d, out, accumulate, ld=None, pad_id=-1):
    ws = torch.empty(mnmt.mnmt_embed_backward_workspace(T, V, d), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mnmt.mnmt_embed_backward(ids, T, g, mnmt.BF16, d, 1.0, pad_id, V, d, out, CODE[out.dtype], ld or d, accumulate, ws, status)
    return status


@pytest.mark.parametrize("V,d,pad", [(30, 40, 2), (FEW_ROWS, 8, 0), (FEW_ROWS + 1, 8, 0), (FEW_ROWS + 1, 5, 3), (FEW_ROWS + 700, 3, 0), (13000, 70000, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("accumulate", [False, True])
def test_no_tokens(V, d, pad, dtype, accumulate):
    """Zeros, or what was there; nothing between the rows is written."""
    buf = torch.full((V, d + pad), SENTINEL, dtype=dtype, device="cuda")
    status = backward(None, 0, None, V, d, buf, accumulate, d + pad)
    assert int(status) == 0
    assert bool((buf[:, :d] == (SENTINEL if accumulate else 0.0)).all()) and bool((buf[:, d:] == SENTINEL).all())


def test_no_tokens_behind_other_calls():
    """The zeros come after what the calls before them in the stream read and wrote there."""
    V, d, T = FEW_ROWS + 1, 8, 5000
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    g = torch.ones((T, d), dtype=torch.bfloat16, device="cuda")
    table, x = torch.full((V, d), SENTINEL, dtype=torch.bfloat16, device="cuda"), torch.empty((T, d), device="cuda")
    ws = [torch.empty(mnmt.mnmt_embed_backward_workspace(t, V, d), dtype=torch.uint8, device="cuda") for t in (T, 0)]
    for _ in range(5):
        table.fill_(SENTINEL)
        mnmt.mnmt_embed_backward(ids, T, g, mnmt.BF16, d, 1.0, -1, V, d, table, mnmt.BF16, d, True, ws[0])
        mnmt.mnmt_embed(ids, T, table, mnmt.BF16, d, V, d, 1.0, x, mnmt.F32, d)
        mnmt.mnmt_embed_backward(None, 0, None, mnmt.BF16, d, 1.0, -1, V, d, table, mnmt.BF16, d, False, ws[1])
        torch.cuda.synchronize()
        n = torch.bincount(ids.long(), minlength=V)[ids.long()].float()  # at most 3 or so of 5000 in 2.5 million: exact in bf16
        assert torch.equal(x, (SENTINEL + n)[:, None].expand(T, d)) and not bool(table.any())


@pytest.mark.parametrize("T", [0, 4999])
def test_rows_past_one_round_of_marks(T):
    """More than 65536 rows a block, into a buffer that is not zero before: rows that no token names are zero, the others
    the sums (small whole numbers: exact)."""
    V, d = 65536 * 4 * 152 + 1300, 8
    gen = torch.Generator(device="cuda").manual_seed(4)
    ids = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    if T:
        ids[:5] = torch.tensor([0, V - 1, 65536 * 4 * 152, 65536 * 4 * 152 - 1, 7], device="cuda")
        ids[5:9] = V - 1
    g = torch.randint(1, 4, (max(T, 1), d), generator=gen, device="cuda").to(torch.bfloat16)
    out = torch.full((V, d), SENTINEL, dtype=torch.bfloat16, device="cuda")
    status = backward(ids, T, g, V, d, out, False, pad_id=7)
    assert int(status) == 0
    use = ids.long()[ids != 7]
    names, back = torch.unique(use, return_inverse=True)
    want = torch.zeros((len(names), d), device="cuda").index_add_(0, back, g[:T][ids != 7].float())
    assert torch.equal(out[names].float(), want)
    out[names] = 0
    assert not bool(out.any())
