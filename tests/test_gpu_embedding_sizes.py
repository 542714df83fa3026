"""The embedding's gradient at the sizes that change how it is formed: keys of one, two and
three digits of the sort on both sides of 8192 tokens, more than 2^20 tokens, pieces of
8, 16, 32 and 64 tokens, and runs of one row over many pieces.

Gradients are differences: a row's n-th token brings a[n] - a[n - 1], a small whole numbers,
so that every sum of neighbouring tokens of a row, and their total a[last], is exact in
any order, and a token left out, taken twice or put into another row shows."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def ids_of(kind, N, rows, g):
    u = torch.rand((N,), generator=g, device="cuda", dtype=torch.float64)
    i = torch.arange(N, device="cuda")
    if kind == "one":
        return torch.full((N,), rows // 2, device="cuda")
    if kind == "even":
        return (u * rows).long()
    if kind == "skewed":  # half of the tokens one row, the n-th row as often as 1 / n else
        ids = (torch.exp(u * torch.log(torch.tensor(rows + 1.0))) - 1).long().clamp(max=rows - 1)
        return torch.where(i % 2 == 0, rows - 1, ids)
    if kind == "runs":    # sorted: runs of 1, 8, 16, 63, 64, 65, 128, 4500 tokens, and again
        sizes = torch.tensor([1, 8, 16, 63, 64, 65, 128, 4500], device="cuda")
        ends = sizes.repeat(N // int(sizes.sum()) + 1).cumsum(0)
        return torch.searchsorted(ends, i, right=True) % rows
    if kind == "edges":   # both sides of every power of two, and the last rows
        k = torch.arange(1, rows.bit_length(), device="cuda")
        at = torch.cat([2 ** k - 1, 2 ** k, 2 ** k + 1, torch.tensor([0, rows - 2, rows - 1], device="cuda")])
        at = at.clamp(max=rows - 1)
        return at[(u * at.numel()).long()]
    raise ValueError(kind)


CASES = [
    # keys 0 .. rows: 10, 11, 20, 21, 23 and 28 bits in digits of at most 10
    (3000, 8, 1023, "even"), (3000, 8, 1024, "edges"), (8192, 16, (1 << 20) - 1, "edges"),
    (5000, 8, 1 << 20, "edges"), (8192, 16, 1100000, "even"), (700, 8, (1 << 22) + 5, "edges"),
    (8193, 8, 1023, "skewed"), (9000, 16, (1 << 20) - 1, "edges"), (9000, 8, 1 << 20, "edges"),
    (70001, 16, 1100000, "even"), (100000, 8, (1 << 22) + 5, "edges"), (40000, 8, (1 << 27) + 3, "edges"),
    (4000, 8, (1 << 27) + 3, "edges"),
    # more than 2^20 tokens, and a last block that is short
    ((1 << 20) + 1, 8, 5000, "skewed"), (3000003, 8, 1200000, "even"), (2500001, 16, 70000, "runs"),
    # a wave over 512 columns: pieces of 16, 32 and 64 tokens
    (2100, 4096, 300, "skewed"), (2100, 4096, 5, "one"), (5000, 4096, 90, "runs"), (5000, 4096, 2000, "skewed"),
    (16001, 4096, 700, "skewed"), (16001, 4096, 3, "one"), (16001, 4096, 40, "runs"), (40000, 520, 1000, "runs"),
    (20000, 264, 100, "skewed"), (33000, 264, 7, "runs"), (70001, 264, 30000, "skewed"),
    # several pieces a wave: 16, 32 and 64 tokens
    (33000, 256, 500, "skewed"), (70000, 256, 60, "runs"), (140001, 256, 4000, "skewed"), (140001, 256, 9, "one"),
    (600001, 16, 3000, "skewed"), (600001, 16, 2, "one"), (2200001, 16, 500, "skewed"), (2200001, 16, 9, "one"),
    (2200001, 16, 300, "runs"),
]


@pytest.mark.parametrize("N,H,rows,kind", CASES, ids=lambda c: str(c))
@pytest.mark.parametrize("outside", [False, True], ids=["", "outside"])
def test_every_token_once_in_its_row(N, H, rows, kind, outside):
    from paper_2607_01844_amd import moe
    print(N, H, rows, kind, outside, flush=True)
    g = torch.Generator(device="cuda").manual_seed(N + H)
    ids = ids_of(kind, N, rows, g)
    begin = 0
    if outside:  # a tenth of the tokens is another rank's, or padding
        begin = 77
        r = torch.rand((N,), generator=g, device="cuda")
        ids = torch.where(r < 0.05, -begin - 1, torch.where(r < 0.1, rows + 3, ids))
    mine = (ids >= 0) & (ids < rows)
    order = torch.argsort(torch.where(mine, ids, rows), stable=True)
    row = ids[order]
    a = torch.randint(-40, 41, (N, H), generator=g, device="cuda", dtype=torch.int16)
    d = a.clone()
    again = row[1:] == row[:-1]
    d[1:] -= torch.where(again[:, None], a[:-1], torch.zeros((), dtype=torch.int16, device="cuda"))
    dy = torch.empty((N, H), dtype=torch.bfloat16, device="cuda")
    dy[order] = d.bfloat16()  # 80 at most: exact
    want = torch.zeros((rows, H), dtype=torch.bfloat16, device="cuda")
    last = mine[order]
    last[:-1] &= ~again
    want[row[last]] = (a[last] * 2).bfloat16()
    dw = torch.full((rows, H), float("nan"), dtype=torch.bfloat16, device="cuda")
    moe.moe_embedding_bwd((ids + begin).int(), dy, rows, 2.0, begin, dw=dw)
    assert torch.equal(dw, want)
