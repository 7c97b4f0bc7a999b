"""Token embedding: the lookup bit for bit, the table gradient against a 64-bit sum, over id distributions, widths and types.

The gradient's bound: a sum of m terms in 32 bits is off by at most (m + 2) 2^-24 times the sum A of their absolute values (two more
roundings: the scale, the store), and a 16-bit table by its unit roundoff."""
import numpy as np
import pytest
import torch

from paper_2411_17887_b200 import api
from tests.lm_reference import U, assert_within, f64

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def ids_of(kind, n, rows, dtype=torch.int64, seed=0):
    rng = np.random.default_rng(seed + n)
    if kind == "uniform":
        x = rng.integers(0, rows, n)
    elif kind == "one":
        x = np.full(n, rows - 1)
    elif kind == "skewed":
        x = np.minimum((rows ** rng.random(n) - 1).astype(np.int64), rows - 1)
    elif kind == "distinct":
        x = rng.permutation(rows)[:n]
    elif kind == "outside":
        x = rng.integers(-3, rows + 3, n)
        x[0] = -2 ** 31
    return torch.from_numpy(x.astype(np.int64)).to(dtype).cuda()


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("id_type", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,rows,d", [(1, 1, 1), (7, 100, 64), (33, 1000, 500), (5, 10, 3), (300, 50, 1030), (1, 5, 4096), (2050, 700, 24)])
def test_lookup(n, rows, d, id_type, dtype):
    table = torch.randn((rows, d), device="cuda").to(dtype)
    ids = ids_of("outside" if n > 4 else "uniform", n, rows, id_type)
    got = api.embedding(ids, table, scale=1.7)
    ok = (ids >= 0) & (ids < rows)
    want = (table[ids.long().clamp(0, rows - 1)].float() * 1.7).to(dtype)
    assert torch.equal(got, torch.where(ok[:, None], want, torch.zeros_like(want)))


def test_lookup_shapes_and_strides():
    table = torch.randn((50, 96), device="cuda").to(torch.bfloat16)
    ids = ids_of("uniform", 30, 50).view(2, 3, 5)
    want = table[ids]
    assert torch.equal(api.embedding(ids, table), want)
    wide = torch.zeros((50, 101), dtype=table.dtype, device="cuda")
    wide[:, 1:97] = table
    assert torch.equal(api.embedding(ids, wide[:, 1:97]), want)               # rows off every boundary but their own
    assert torch.equal(api.embedding(ids.transpose(0, 2), table), table[ids.transpose(0, 2)])
    assert torch.equal(api.embedding(ids, table.t().contiguous().t()), want)
    assert api.embedding(ids[:0], table).shape == (0, 3, 5, 96)


def gradient(ids, d_out, rows, scale):
    want, size, count = np.zeros((rows, d_out.shape[1])), np.zeros((rows, d_out.shape[1])), np.zeros(rows)
    x, at = f64(d_out), ids.cpu().numpy()
    ok = (at >= 0) & (at < rows)
    np.add.at(want, at[ok], x[ok])
    np.add.at(size, at[ok], np.abs(x[ok]))
    np.add.at(count, at[ok], 1)
    return want * scale, (count + 2)[:, None] * 2.0 ** -24 * size * scale + 1e-30


@pytest.mark.parametrize("dtype,table_type", [(torch.float32, torch.float32), (torch.float16, torch.float32), (torch.bfloat16, torch.float32),
                                              (torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16)], ids=str)
@pytest.mark.parametrize("kind,n,rows,d", [
    ("uniform", 1, 1, 1), ("uniform", 5, 3, 7), ("uniform", 64, 64, 64), ("one", 5000, 40, 32), ("distinct", 900, 1000, 100),
    ("skewed", 4097, 3000, 500), ("skewed", 70000, 600, 16), ("outside", 3000, 100, 65), ("uniform", 100, 300000, 8),
    ("uniform", 2500, 511, 1032), ("one", 300, 512, 4104), ("uniform", 128, 513, 12)])
def test_table_gradient(kind, n, rows, d, dtype, table_type):
    ids = ids_of(kind, n, rows, torch.int32 if d % 2 else torch.int64)
    d_out = torch.randn((n, d), device="cuda").to(dtype)
    want, bound = gradient(ids, d_out, rows, 1.3)
    if table_type != torch.float32:
        bound = bound + U[table_type] * np.abs(want) + (2.0 ** -25 if table_type == torch.float16 else 0.0)
    got = api.embedding_backward(d_out, ids, rows, scale=1.3, dtype=table_type)
    assert got.dtype == table_type
    assert_within(got, want, bound, "gradient")
    assert torch.equal(got, api.embedding_backward(d_out, ids, rows, scale=1.3, dtype=table_type))       # the same bits again


@pytest.mark.parametrize("dtype,table_type", [(torch.bfloat16, torch.float32), (torch.float16, torch.float16)], ids=str)
@pytest.mark.parametrize("kind,n,rows,d", [
    ("uniform", 1024, 4000, 40), ("one", 8192, 300, 16), ("outside", 8191, 520, 12), ("skewed", 2000, 300000, 8), ("uniform", 8193, 30000, 12), ("uniform", 1025, 900, 264), ("one", 4096, 300, 16), ("skewed", 30, 70000, 240), ("outside", 4097, 511, 33), ("uniform", 8193, 20, 8), ("skewed", 12289, 30000, 136), ("one", 9000, 70000, 1100),
    ("uniform", 5000, 300000, 4), ("skewed", 270000, 5000, 6), ("outside", 300001, 600, 3)])
def test_table_gradient_of_many_tokens(kind, n, rows, d, dtype, table_type):
    """Either side of the tokens that one launch takes; one, two and three passes of the sort; counts added and scanned."""
    test_table_gradient(kind, n, rows, d, dtype, table_type)


@pytest.mark.parametrize("kind,n,rows,d", [("skewed", 9001, 5000, 72), ("one", 6000, 9, 130), ("outside", 5000, 50, 33), ("uniform", 4500, 100000, 16)])
def test_sums_of_many_tokens_added_to_another(kind, n, rows, d):
    test_table_gradient_added_to_another(kind, n, rows, d)


@pytest.mark.parametrize("kind,n,rows,d", [("skewed", 3000, 500, 64), ("one", 1000, 9, 130), ("outside", 200, 50, 33), ("uniform", 3, 100000, 16)])
def test_table_gradient_added_to_another(kind, n, rows, d):
    ids = ids_of(kind, n, rows)
    d_out = torch.randn((n, d), device="cuda").to(torch.bfloat16)
    held = torch.randn((rows, d), device="cuda")
    untouched = torch.ones(rows, dtype=torch.bool, device="cuda")
    untouched[ids[(ids >= 0) & (ids < rows)].long()] = False
    want, bound = gradient(ids, d_out, rows, 0.5)
    out = held.clone()
    assert api.embedding_backward(d_out, ids, rows, scale=0.5, out=out) is out
    assert torch.equal(out[untouched], held[untouched])
    assert_within(out, want + f64(held), bound + 2.0 ** -23 * np.abs(f64(held)) + 2.0 ** -23 * np.abs(want), "gradient")


def test_infinities_stay_in_their_rows():
    ids = ids_of("uniform", 500, 40)
    d_out = torch.randn((500, 48), device="cuda").to(torch.bfloat16)
    want, bound = gradient(ids, d_out, 40, 1.0)
    row = int(ids[17])
    d_out[17] = float("inf")
    outside = ids.clone()
    outside[3] = 40                                     # a token that belongs to no row may hold anything
    d_out[3] = float("nan")
    got = api.embedding_backward(d_out, outside, 40)
    assert torch.isinf(got[row]).all()
    keep = np.arange(40) != row
    keep[int(ids[3])] = False
    assert_within(f64(got)[keep], want[keep], bound[keep], "gradient")


def test_empty_gradient_and_side_stream_and_graph():
    none = torch.empty((0, 16), device="cuda")
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    assert torch.equal(api.embedding_backward(none, ids, 5), torch.zeros((5, 16), device="cuda"))
    held = torch.ones((5, 16), device="cuda")
    api.embedding_backward(none, ids, 5, out=held)
    assert torch.equal(held, torch.ones_like(held))

    ids = ids_of("skewed", 3000, 700)
    d_out = torch.randn((3000, 64), device="cuda").to(torch.float16)
    table = torch.randn((700, 64), device="cuda")
    want, looked = api.embedding_backward(d_out, ids, 700), api.embedding(ids, table, 2.0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = d_out * 0
        torch.cuda._sleep(2_000_000)
        late += d_out
        got = api.embedding_backward(late, ids, 700)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g1, g2 = api.embedding_backward(d_out, ids, 700), api.embedding(ids, table, 2.0)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(g1, want) and torch.equal(g2, looked)


def test_autograd():
    table = torch.randn((300, 40), device="cuda").to(torch.bfloat16).requires_grad_()
    ids = ids_of("skewed", 200, 300).view(10, 20)
    out = api.embedding(ids, table, scale=3.0)
    d_out = torch.randn_like(out)
    out.backward(d_out)
    assert torch.equal(table.grad, api.embedding_backward(d_out, ids, 300, scale=3.0, dtype=torch.bfloat16))
