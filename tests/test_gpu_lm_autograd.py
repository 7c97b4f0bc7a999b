"""The language-model operators under autograd: what they cannot differentiate they refuse, and what they write in place they say."""
import pytest
import torch

from paper_2411_17887_b200 import api
from tests.test_gpu_linattn import draw

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")


def test_second_derivatives_are_refused():
    """A penalty on gradients reaches the parameters by way of the gradients themselves: without an error it would lose that part."""
    q, k, v, _, decay, s0, _ = draw(1, 1, 50, 2, 16, 16, torch.bfloat16, True)
    for which in range(4):
        args = [q, k, v, s0]
        root = torch.ones_like(args[which]).requires_grad_()
        args[which] = args[which] * root ** 2
        o, last = api.linear_attention(*args[:3], decay, initial_state=args[3], output_final_state=True)
        g, = torch.autograd.grad(o.float().square().sum() + last.square().sum(), root, create_graph=True)
        assert torch.isfinite(g).all() and g.abs().sum() > 0
        with pytest.raises(RuntimeError, match="once_differentiable"):
            g.float().square().sum().backward()
    root = torch.randn((9, 8), device="cuda").requires_grad_()
    out = api.embedding(torch.arange(9, device="cuda"), root ** 2)
    g, = torch.autograd.grad(out.square().sum(), root, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.square().sum().backward()


def test_tangents_are_refused():
    """Forward-mode derivatives: an output without its tangent would read as one that does not depend on the input."""
    q, k, v, d_o, decay, s0, _ = draw(2, 1, 50, 2, 16, 16, torch.bfloat16, True)
    table, ids, grad = torch.randn((9, 8), device="cuda"), torch.arange(9, device="cuda"), torch.zeros((9, 8), device="cuda")
    plain = api.linear_attention(q, k, v, decay, initial_state=s0)[0], api.embedding(ids, table)
    step = lambda q, k, v, decay, s0: api.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, s0.clone())  # noqa: E731
    calls = [lambda q, k, v, decay, s0: api.linear_attention(q, k, v, decay, initial_state=s0), step,
             lambda q, k, v, decay, s0: api.linear_attention_backward(d_o, q, k, v, decay, initial_state=s0)]
    with torch.autograd.forward_ad.dual_level():
        dual = lambda x: torch.autograd.forward_ad.make_dual(x, torch.ones_like(x))  # noqa: E731
        for which in range(5):
            args = [q, k, v, decay, s0]
            args[which] = dual(args[which])
            for call in calls:
                with pytest.raises(NotImplementedError):
                    call(*args)
        with pytest.raises(NotImplementedError):
            api.linear_attention_backward(dual(d_o), q, k, v, decay)
        with pytest.raises(NotImplementedError):
            api.embedding(ids, dual(table))
        with pytest.raises(NotImplementedError):
            api.embedding_backward(dual(table), ids, 9)
        with pytest.raises(NotImplementedError):
            api.embedding_backward(table, ids, 9, out=dual(grad))
        # without one the calls are as ever
        assert torch.equal(api.linear_attention(q, k, v, decay, initial_state=s0)[0], plain[0])
        assert torch.equal(api.embedding(ids, table), plain[1])


def test_what_is_written_in_place_is_known():
    """A state, or a sum, that a backward pass has saved and that is then written to: torch raises, as for its own operators."""
    q, k, v, d_o, decay, s0, _ = draw(3, 1, 50, 2, 16, 16, torch.bfloat16, True)
    token = [x[:, 0].clone() for x in (q, k, v)]
    q.requires_grad_()
    o, _ = api.linear_attention(q, k, v, decay, initial_state=s0)
    api.linear_attention_step(*token, decay, s0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.backward(d_o)
    ids, held, x = torch.arange(9, device="cuda"), torch.randn((9, 8), device="cuda"), torch.randn((9, 8), device="cuda", requires_grad=True)
    y = (x * held).sum()
    api.embedding_backward(torch.ones((9, 8), device="cuda"), ids, 9, out=held)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    # a state that has been through nothing but steps, made where versions are not kept
    with torch.inference_mode():
        pool = torch.zeros((1, 2, 16, 16), device="cuda")
    api.linear_attention_step(*token, decay, pool)
    with torch.inference_mode():
        api.linear_attention_step(*token, decay, pool)
        api.embedding_backward(torch.ones((9, 8), device="cuda"), ids, 9, out=held)


def test_steps_do_not_lose_gradients():
    """Single tokens have no backward pass: inputs that want one are refused, unless gradients are off."""
    q, k, v, _, decay, s0, _ = draw(4, 1, 1, 2, 16, 16, torch.bfloat16, True)
    args = [x[:, 0] for x in (q, k, v)] + [decay, s0]
    want_state = s0.clone()
    want = api.linear_attention_step(*args[:4], want_state)
    for which in (0, 1, 2, 4):
        some = list(args)
        some[which] = some[which].clone().requires_grad_()
        with pytest.raises(RuntimeError, match="no_grad"):
            api.linear_attention_step(*some)
    assert torch.equal(s0, args[4])
    with torch.no_grad():
        state = s0.clone().requires_grad_()
        assert torch.equal(api.linear_attention_step(args[0].clone().requires_grad_(), *args[1:4], state), want)
        assert torch.equal(state, want_state)
    grad = torch.zeros((9, 8), device="cuda", requires_grad=True)
    with pytest.raises(RuntimeError, match="no_grad"):
        api.embedding_backward(torch.ones((9, 8), device="cuda"), torch.arange(9, device="cuda"), 9, out=grad)
