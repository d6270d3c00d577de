"""argus_embedding and argus_embedding_bwd against the definition in 64 bits.

The lookup is one product rounded once: the exact bits are expected. The
gradient's tolerance, per element: n additions of 32-bit floats are off by at
most n 2^-24 of the sum of magnitudes, the product with the scale by 2^-24 of
the result, and the output's rounding by half a unit of its type."""
import pytest
import torch

import paper_2606_20374_amd as pa
from paper_2606_20374_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
UNIT = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
TINY = {torch.float32: 2.0**-149, torch.bfloat16: 2.0**-133, torch.float16: 2.0**-24}


def _ids(n, vocab, kind, seed, dtype=torch.int64):
    g = torch.Generator().manual_seed(seed)
    if kind == "uniform":
        ids = torch.randint(0, vocab, (n,), generator=g)
    elif kind == "one":  # every token the same
        ids = torch.full((n,), vocab // 2)
    elif kind == "hot":  # one id has half of the tokens, the rest are spread; some padding
        ids = torch.randint(0, vocab, (n,), generator=g)
        ids[torch.rand(n, generator=g) < 0.5] = vocab - 1
        ids[torch.rand(n, generator=g) < 0.1] = -1
    elif kind == "ends":  # the first and the last row of the table only
        ids = torch.randint(0, 2, (n,), generator=g) * (vocab - 1)
    else:
        ids = torch.full((n,), -1)
    return ids.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,vocab,dim,pad", [(1, 1, 1, 0), (3, 7, 33, 0), (130, 100, 64, 0), (1000, 51, 257, 3),
                                             (37, 1000, 2048, 8), (5, 9, 5001, 1), (0, 4, 16, 0)])
def test_lookup(n, vocab, dim, pad, dtype):
    g = torch.Generator().manual_seed(n + dim)
    table = torch.randn(vocab, dim + pad, generator=g).to(dtype)
    ids = _ids(n, vocab, "hot", 1, torch.int32 if n % 2 else torch.int64)
    got = pa.embedding(ids.to(DEV), table.to(DEV)[:, :dim], scale=1.7)
    want = (table[:, :dim][ids.clamp(min=0).long()].float() * torch.tensor(1.7)).to(dtype)
    want[ids < 0] = 0
    assert torch.equal(got["out"].cpu(), want)
    assert int(got["dev_status"]) == 0


def test_lookup_out_of_range_and_bad_rows():
    table = torch.randn(10, 24)
    table[0] = float("nan")  # a row that no token names
    ids = torch.tensor([1, 10, -5, 2**40, 9])
    got = pa.embedding(ids.to(DEV), table.to(DEV))
    want = torch.zeros(5, 24)
    want[0], want[4] = table[1], table[9]
    assert torch.equal(got["out"].cpu(), want)
    assert int(got["dev_status"]) == ops.DEV_TOKEN_RANGE


def _check_bwd(ids, dout, vocab, scale, got, dtype):
    keep = (ids >= 0) & (ids < vocab)
    at = ids[keep].long()
    d = dout[keep].double()
    ref = torch.zeros(vocab, dout.shape[1], dtype=torch.float64).index_add_(0, at, d) * scale
    mag = torch.zeros(vocab, dout.shape[1], dtype=torch.float64).index_add_(0, at, d.abs()) * abs(scale)
    n = torch.zeros(vocab, dtype=torch.float64).index_add_(0, at, torch.ones(len(at), dtype=torch.float64))
    tol = n[:, None] * 2.0**-24 * mag + (2.0**-23 + UNIT[dtype]) * ref.abs() + TINY[dtype]
    g = got["dtable"].cpu().double()
    bad = (g - ref).abs() > tol
    assert not bad.any(), (int(bad.sum()), (g - ref).abs().max())
    assert torch.all(g[n == 0] == 0)


@pytest.mark.parametrize("kind", ["uniform", "one", "hot", "ends", "none"])
@pytest.mark.parametrize("n,vocab,dim", [(1, 3, 8), (64, 5, 40), (129, 300, 33), (1000, 50, 128), (1024, 2000, 16),
                                         (1025, 70_000, 24), (5000, 300, 100), (20_011, 257, 64), (9000, 65_536, 8)])
def test_gradient(n, vocab, dim, kind):
    g = torch.Generator().manual_seed(n)
    ids = _ids(n, vocab, kind, 2, torch.int32 if dim % 3 else torch.int64)
    dout = torch.randn(n, dim, generator=g)
    got = pa.embedding_bwd(ids.to(DEV), dout.to(DEV), vocab, scale=0.5)
    _check_bwd(ids, dout, vocab, 0.5, got, torch.float32)
    assert int(got["dev_status"]) == 0


@pytest.mark.parametrize("dtype,grad", [(torch.bfloat16, None), (torch.float16, None), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("n,vocab,dim,pad", [(700, 90, 200, 0), (3000, 1000, 333, 5), (300, 20, 4104, 0)])
def test_gradient_types_and_strides(n, vocab, dim, pad, dtype, grad):
    g = torch.Generator().manual_seed(n)
    ids = _ids(n, vocab, "hot", 3)
    dout = torch.randn(n, dim + pad, generator=g).to(dtype)
    got = pa.embedding_bwd(ids.to(DEV), dout.to(DEV)[:, :dim], vocab, scale=0.125, dtype=grad)
    assert got["dtable"].dtype == (grad or dtype)
    _check_bwd(ids, dout[:, :dim], vocab, 0.125, got, grad or dtype)


def test_gradient_of_a_broadcast_input_and_out_of_range():
    ids = torch.tensor([4, 4, 5, 9, 100, -1, 4] * 300)
    row = torch.randn(1, 48)
    got = pa.embedding_bwd(ids.to(DEV), row.to(DEV).expand(len(ids), 48), 10)
    _check_bwd(ids, row.expand(len(ids), 48), 10, 1.0, got, torch.float32)
    assert int(got["dev_status"]) == ops.DEV_TOKEN_RANGE


def test_empty_batch_clears_the_gradient():
    out = pa.alloc_embedding_bwd(33, 20, torch.float32)
    out["dtable"].fill_(7)
    pa.embedding_bwd(torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, 20, device=DEV), 33, out=out)
    assert torch.all(out["dtable"] == 0)


def test_gradient_against_differences():
    # the lookup is linear in the table: a difference has no truncation, only
    # the rounding of its products (2^-24 of each) and of the two sums here
    g = torch.Generator().manual_seed(9)
    ids = _ids(2000, 37, "hot", 5)
    table, step, dout = (torch.randn(s, generator=g) for s in ((37, 19), (37, 19), (2000, 19)))
    up = pa.embedding(ids.to(DEV), (table + step).to(DEV), scale=3.0)["out"].cpu().double()
    dn = pa.embedding(ids.to(DEV), table.to(DEV), scale=3.0)["out"].cpu().double()
    d = pa.embedding_bwd(ids.to(DEV), dout.to(DEV), 37, scale=3.0)["dtable"].cpu().double()
    moved = ((table + step).double() - table.double())
    lhs, rhs = ((up - dn) * dout.double()).sum(), (d * moved).sum()
    tol = 2.0**-23 * ((up.abs() + dn.abs()) * dout.abs()).sum() + 2000 * 2.0**-24 * (
        3 * torch.zeros(37, 19, dtype=torch.float64).index_add_(0, ids[ids >= 0], dout[ids >= 0].double().abs()) * moved.abs()).sum()
    assert abs(lhs - rhs) <= tol, (lhs, rhs, tol)


def test_same_bits_each_time_and_on_another_stream():
    ids = _ids(30_000, 4000, "hot", 8).to(DEV)
    dout = torch.randn(30_000, 72, device=DEV)
    first = pa.embedding_bwd(ids, dout, 4000)["dtable"].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = pa.embedding_bwd(ids, dout, 4000)["dtable"]
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(first, again)


@pytest.mark.parametrize("n,pad", [(1, 1), (5, 2), (10, 1), (33, 1), (40, 40), (100, 3), (130, 2), (1030, 5), (5001, 1)])
@pytest.mark.parametrize("dim", [8, 40, 600, 2056])
def test_gradient_of_padding_writes_no_row(n, pad, dim):
    # padding that begins and ends among the last sorted positions: what lies
    # behind the table keeps its values
    vocab = 77
    ids = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(n))
    ids[:pad] = -1
    ids[0] = vocab
    dout = torch.randn(n, dim, generator=torch.Generator().manual_seed(dim))
    rows = torch.full((vocab + 2, dim), 7.0, device=DEV)
    got = pa.embedding_bwd(ids.to(DEV), dout.to(DEV), vocab,
                           out={"dtable": rows[:vocab], "dev_status": torch.zeros(1, dtype=torch.int32, device=DEV)})
    _check_bwd(ids, dout, vocab, 1.0, got, torch.float32)
    assert torch.all(rows[vocab:] == 7.0)
    assert int(got["dev_status"]) == ops.DEV_TOKEN_RANGE


@pytest.mark.parametrize("kind", ["uniform", "one", "hot", "ends", "none"])
@pytest.mark.parametrize("n,vocab,dim", [(70_001, 300, 24), (140_000, 50_000, 8), (5000, 262_144, 8), (70_001, 300_007, 9)])
def test_gradient_of_many_tokens_and_ids(n, vocab, dim, kind):
    # past 65,536 tokens a workgroup sorts several rounds of them, and ids from
    # 262,144 on take a third pass
    test_gradient(n, vocab, dim, kind)
