"""Layer norm: values and gradients against 64 bits with derived bounds, over widths, rows, types, strides and rows that are hard to normalise."""
import numpy as np
import pytest
import torch

from paper_2411_17887_b200 import api
from tests import norm_reference as ref
from tests.lm_reference import assert_within, f64

pytestmark = pytest.mark.gpu
TYPES = [(torch.float32, torch.float32), (torch.float16, torch.float32), (torch.float16, torch.float16), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16)]


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def draw(rows, d, dtype, param_type, seed=0, shift=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    return (normal(rows, d) * 2.0 + shift).to(dtype), normal(rows, d).to(dtype), (1.0 + 0.5 * normal(d)).to(param_type), normal(d).to(param_type)


def check(x, d_y, weight, bias, eps=1e-5):
    d = x.shape[-1]
    w = np.ones(d) if weight is None else f64(weight)
    b = np.zeros(d) if bias is None else f64(bias)
    kind = torch.float32 if weight is None else weight.dtype
    y = api.layer_norm(x, weight, bias, eps)
    d_x, d_w, d_b = api.layer_norm_backward(d_y, x, weight, eps)
    assert y.shape == d_x.shape == x.shape and y.dtype == d_x.dtype == x.dtype and d_w.dtype == d_b.dtype == kind
    flat = lambda z: f64(z).reshape(-1, d)  # noqa: E731
    value, bound = ref.forward(flat(x), w, b, eps, x.dtype)
    assert_within(flat(y), value, bound, "y")
    for name, got, (value, bound) in zip(("d_x", "d_weight", "d_bias"), (flat(d_x), d_w, d_b), ref.backward(flat(d_y), flat(x), w, eps, x.dtype, kind)):
        assert_within(got, value, bound, name)
    again = api.layer_norm_backward(d_y, x, weight, eps)
    assert all(torch.equal(p, q) for p, q in zip(again, (d_x, d_w, d_b)))                 # the same bits again
    alone = api.layer_norm_backward(d_y, x, weight, eps, params=False)
    assert torch.equal(alone[0], d_x) and alone[1] is None and alone[2] is None


@pytest.mark.parametrize("dtype,param_type", TYPES, ids=str)
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 2), (7, 64), (9, 255), (33, 256), (5, 257), (100, 501), (17, 512), (6, 513), (40, 1024), (3, 2056), (11, 4097), (2, 8192), (3, 8200),
                                    (2, 16383), (1, 16384), (2, 10000), (30, 40), (1000, 128), (65, 130), (77, 8), (5, 12002), (64, 62)])
def test_sizes(rows, d, dtype, param_type):
    check(*draw(rows, d, dtype, param_type, rows + d))


@pytest.mark.parametrize("rows,d", [(20000, 64), (12000, 300), (5000, 1000), (700, 1537)])
def test_many_rows(rows, d):
    """More rows than a grid holds at once: sums of the parameters' gradients over several rows a block."""
    check(*draw(rows, d, torch.bfloat16, torch.float32, d))


def test_without_parameters():
    x, d_y, weight, bias = draw(30, 96, torch.bfloat16, torch.float32)
    check(x, d_y, None, None)
    check(x, d_y, weight, None)
    check(x, d_y, None, bias)
    check(x, d_y, weight, bias, eps=0.0)
    check(x, d_y, weight, bias, eps=1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("d", [96, 101, 1040])
def test_strides(d, dtype):
    wide, other, weight, bias = draw(50, d + 24, dtype, torch.float32)
    weight, bias = weight[:d].clone(), bias[:d].clone()
    for x, d_y in ((wide[:, :d], other[:, 8:d + 8]), (wide[:, 1:d + 1], other[:, :d]), (wide[::2, 16:d + 16], other[:25, 3:d + 3]), (wide[:1, :d].expand(50, d), other[:, :d]),
                   (wide[:, :d].t().contiguous().t(), other[:, :d])):
        check(x, d_y, weight, bias)
    x = wide[:, :d].reshape(2, 5, 5, d)
    check(x.transpose(0, 2), other[:, :d].reshape(5, 5, 2, d), weight, bias)
    assert torch.equal(api.layer_norm(x[0, 0, 0], weight, bias), api.layer_norm(x, weight, bias)[0, 0, 0])


@pytest.mark.parametrize("d", [100, 512, 3001])
def test_rows_far_from_zero(d):
    """A mean of a thousand deviations, and rows of one value: the deviations are still those of the values."""
    x, d_y, weight, bias = draw(12, d, torch.float32, torch.float32, 1, shift=2000.0)
    x[3] = 1234.5678
    x[4] = 0.0
    check(x, d_y, weight, bias)
    assert (api.layer_norm(x, None, None)[4] == 0).all()


def test_what_is_not_finite_stays_in_its_row():
    x, d_y, weight, bias = draw(20, 300, torch.float16, torch.float32)
    clean, clean_x = api.layer_norm(x, weight, bias), api.layer_norm_backward(d_y, x, weight)[0]
    x[3, 7], x[11, 299] = float("inf"), float("nan")
    y, d_x = api.layer_norm(x, weight, bias), api.layer_norm_backward(d_y, x, weight)[0]
    rest = torch.ones(20, dtype=torch.bool, device="cuda")
    rest[3] = rest[11] = False
    assert torch.equal(y[rest], clean[rest]) and torch.equal(d_x[rest], clean_x[rest])
    assert not torch.isfinite(y[~rest]).all(1).any()


def test_no_rows():
    x = torch.empty((0, 40), device="cuda", dtype=torch.bfloat16)
    weight = torch.ones(40, device="cuda")
    assert api.layer_norm(x, weight, weight).shape == (0, 40)
    d_x, d_w, d_b = api.layer_norm_backward(x, x, weight)
    assert d_x.shape == (0, 40) and not d_w.any() and not d_b.any()


def test_in_place():
    """From C, y may be x and d_x may be d_y."""
    from paper_2411_17887_b200 import binding as B
    stream = torch.cuda.current_stream().cuda_stream
    for d in (200, 2000):
        x, d_y, weight, bias = draw(37, d, torch.bfloat16, torch.float32)
        want, want_x = api.layer_norm(x, weight, bias), api.layer_norm_backward(d_y, x, weight)[0]
        assert B.tcu_layer_norm_backward(d_y, d, x, d, 37, d, B.TCU_BF16, weight, B.TCU_F32, 1e-5, d_y, None, None, None, 0, stream) == B.TCU_OK
        assert B.tcu_layer_norm_forward(x, 37, d, d, B.TCU_BF16, weight, bias, B.TCU_F32, 1e-5, x, stream) == B.TCU_OK
        assert torch.equal(x, want) and torch.equal(d_y, want_x)


def test_differences():
    """The kernel's gradients against differences of the 64-bit formula."""
    x, d_y, weight, bias = draw(2, 7, torch.float32, torch.float32, 3)
    got = api.layer_norm_backward(d_y, x, weight)
    args = [f64(x), f64(weight), f64(bias)]
    loss = lambda x, w, b: (ref.forward(x, w, b, 1e-5, torch.float32)[0] * f64(d_y)).sum()  # noqa: E731
    for which in range(3):
        for at in np.ndindex(args[which].shape):
            moved = []
            for step in (1e-5, -1e-5):
                some = [a.copy() for a in args]
                some[which][at] += step
                moved.append(loss(*some))
            # second order of the difference and cancellation (1e-9), then 32 bits of values of a few units
            assert abs((moved[0] - moved[1]) / 2e-5 - float(got[which][at])) < 1e-5


def test_autograd():
    x, d_y, weight, bias = draw(60, 130, torch.bfloat16, torch.float32)
    want = api.layer_norm_backward(d_y, x, weight)
    leaves = [z.clone().requires_grad_() for z in (x, weight, bias)]
    api.layer_norm(*leaves).backward(d_y)
    assert all(torch.equal(leaf.grad, w) for leaf, w in zip(leaves, want))
    for which in range(3):                                                                  # one alone
        args = [x, weight, bias]
        args[which] = args[which].clone().requires_grad_()
        api.layer_norm(*args).backward(d_y)
        assert torch.equal(args[which].grad, want[which])
    api.layer_norm(leaves[0]).sum().backward()                                              # a gradient with strides of zero
    root = torch.ones_like(x).requires_grad_()
    g, = torch.autograd.grad(api.layer_norm(x * root ** 2, weight).float().square().sum(), root, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.float().sum().backward()
    with torch.autograd.forward_ad.dual_level():
        dual = lambda z: torch.autograd.forward_ad.make_dual(z, torch.ones_like(z))  # noqa: E731
        for call in (lambda: api.layer_norm(dual(x)), lambda: api.layer_norm(x, dual(weight)), lambda: api.layer_norm(x, weight, dual(bias)),
                     lambda: api.layer_norm_backward(dual(d_y), x, weight), lambda: api.layer_norm_backward(d_y, x, dual(weight))):
            with pytest.raises(NotImplementedError):
                call()


def test_graph():
    sets = [draw(300, 700, torch.bfloat16, torch.float32, s) for s in range(3)]
    both = lambda x, d_y, weight, bias: (api.layer_norm(x, weight, bias), *api.layer_norm_backward(d_y, x, weight))  # noqa: E731
    want = [both(*s) for s in sets]
    held = [z.clone() for z in sets[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(*held)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = both(*held)
    for i in (1, 2, 0):
        for z, new in zip(held, sets[i]):
            z.copy_(new)
        graph.replay()
        assert all(torch.equal(p, q) for p, q in zip(outs, want[i]))
