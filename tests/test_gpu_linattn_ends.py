"""Linear attention where calls end: blocks leave nothing under way, and waits that run out are given up in good order."""
import pytest
import torch

from paper_2411_17887_b200 import api
from paper_2411_17887_b200 import binding as B
from tests.test_gpu_linattn import draw

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    yield
    assert api.linear_attention_status() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 64, 64), (1, 37, 4, 64, 64), (2, 129, 3, 128, 128), (1, 2100, 1, 128, 128), (1, 300, 160, 16, 16), (300, 5, 1, 16, 72)], ids=str)
def test_short_calls_one_after_another(shape, dtype):
    """Nobody but the block itself waits for the commits of a walk's last group, least of all where no state is wanted.  The blocks of
    the next call, and of a scan with barriers in other places, take over the shared memory at once."""
    b, t, h, dk, dv = shape
    q, k, v, d_o, decay, _, _ = draw(t + h, b, t, h, dk, dv, dtype)
    x = torch.ones(40 * 16384, dtype=torch.int8, device="cuda")
    o, grads = api.linear_attention(q, k, v, decay)[0], api.linear_attention_backward(d_o, q, k, v, decay)[:3]
    want = api.scan(x)
    got = []
    for _ in range(30):
        got.append((api.linear_attention(q, k, v, decay)[0], api.linear_attention(q, k, v, decay)[0], api.scan(x), *api.linear_attention_backward(d_o, q, k, v, decay)[:3]))
    torch.cuda.synchronize()
    for one in got:
        for a, w in zip(one, (o, o, want, *grads)):
            assert torch.equal(a, w)


def raw(q, k, v, decay, d_o=None, offsets=None):
    """Arguments of a call on these arrays with fresh outputs (packed: one axis less), with scratch memory where it is of use; and what has to stay alive."""
    t, h, dk = q.shape[-3:]
    dv, b = v.shape[-1], q.shape[0] if offsets is None else offsets.numel() - 1
    held = [torch.zeros_like(v), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)]
    at = lambda x: api._tokens(x)[1]  # noqa: E731
    more = {} if d_o is None else dict(d_o=at(d_o), d_q=at(held[1]), d_k=at(held[2]), d_v=at(held[3]))
    args = B.tcu_linattn_args(api._FLOAT[q.dtype], b, t, h, dk, dv, dk ** -0.5, decay.data_ptr(), at(q), at(k), at(v), at(held[0]),
                              d_offsets=0 if offsets is None else offsets.data_ptr(), **more)
    size = B.tcu_linattn_scratch_bytes(args, int(d_o is not None))
    if size:
        held.append(torch.empty((size + 255) // 4, device="cuda"))
        args = B.tcu_linattn_with_scratch(args, held[-1].data_ptr(), size)
    return args, held, size


# (batch, tokens, heads, dk, dv), lengths of packed sequences, the silent group: a walk of one group, a group within, the last one
# (for which only the block's own end waits); parts of a walk in a cluster, in their first phase and in their second; cut walks;
# packed sequences in order, most of them without such a group
GIVE_UP = [((1, 100, 2, 64, 64), None, 0), ((2, 500, 3, 128, 128), None, 1), ((2, 300, 3, 64, 128), None, 2),
           ((1, 2100, 1, 128, 128), None, 0), ((1, 2100, 1, 64, 64), None, 1), ((1, 2100, 1, 128, 72), None, 4), ((1, 2100, 2, 32, 64), None, 5),
           ((2, 700, 80, 16, 24), None, 0), ((2, 700, 80, 64, 128), None, 3), ((1, 520, 60, 24, 72), None, 4),
           ((1, 4630, 9, 24, 16), [0, 1, 128, 40, 300, 129, 500] * 4 + [238], 2)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("backward", [False, True], ids=["forward", "backward"])
@pytest.mark.parametrize("shape,lens,silent", GIVE_UP, ids=str)
def test_waits_that_run_out(shape, lens, silent, backward, dtype):
    """One group of every walk never reports its state: what waits for it gives up, the kernel returns, the host reads
    TCU_ERR_TIMEOUT, and the same call is right afterwards.  Nothing faults."""
    b, t, h, dk, dv = shape
    q, k, v, d_o, decay, _, _ = draw(t + silent, b, t, h, dk, dv, dtype)
    offsets = None
    if lens:
        offsets = torch.tensor([0] + lens, device="cuda").cumsum(0)
        assert int(offsets[-1]) == t
        q, k, v, d_o = (x[0] for x in (q, k, v, d_o))
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    fn = B.tcu_linattn_backward if backward else B.tcu_linattn_forward
    args, held, scratch = raw(q, k, v, decay, d_o if backward else None, offsets)
    assert scratch > 0 or not (lens or b * h > 148)
    stream = torch.cuda.current_stream().cuda_stream
    assert B.tcu_linattn_selftest_timeout(args, backward, silent, 0, ws, 256, stream) == B.TCU_ERR_INVALID_ARG
    assert B.tcu_linattn_selftest_timeout(args, backward, silent, 1001, ws, 256, stream) == B.TCU_ERR_INVALID_ARG
    B.check(fn(args, ws, 256, stream))
    assert B.tcu_scan_device_status(ws.data_ptr(), stream) == B.TCU_OK
    want = [x.clone() for x in held[:4]]
    B.check(B.tcu_linattn_selftest_timeout(args, backward, silent, 20, ws, 256, stream))
    assert B.tcu_scan_device_status(ws.data_ptr(), stream) == B.TCU_ERR_TIMEOUT
    ws.zero_()
    for x in held[:4]:
        x.zero_()
    B.check(fn(args, ws, 256, stream))
    assert B.tcu_scan_device_status(ws.data_ptr(), stream) == B.TCU_OK
    assert all(torch.equal(a, w) for a, w in zip(held[:4], want))
    # a group that no walk has
    B.check(B.tcu_linattn_selftest_timeout(args, backward, 1000, 500, ws, 256, stream))
    assert B.tcu_scan_device_status(ws.data_ptr(), stream) == B.TCU_OK
    assert all(torch.equal(a, w) for a, w in zip(held[:4], want))
