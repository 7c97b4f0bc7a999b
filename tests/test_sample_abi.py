"""Host-only checks of sampling: argument errors are found before any launch, the Python layer refuses what the library does not take, and the
reference that the GPU tests compare with gives what can be worked out by hand."""
import math

import numpy as np
import pytest
import torch

from tests.sample_reference import kept_tokens, token_of


@pytest.fixture(scope="module")
def B():
    from paper_2411_17887_b200 import build
    build.build()
    from paper_2411_17887_b200 import binding
    return binding


X, U, T, K, P, M, OUT, LP = (0x1000_0000 * i for i in range(1, 9))


def test_refusals(B):
    def f(dtype=B.TCU_BF16, rows=10, vocabulary=100, logits=X, stride=100, uniform=U, f64=0, tokens=OUT, log_probs=LP, **more):
        return B.tcu_sample(B.tcu_sample_args(dtype, rows, vocabulary, logits, stride, uniform, f64, tokens, log_probs, **more))
    assert f(rows=0) == B.TCU_OK
    good = B.tcu_sample_args(B.TCU_BF16, 0, 100, X, 100, U, 0, OUT)
    assert B.tcu_sample((4).to_bytes(4, "little") + good[4:]) == B.TCU_ERR_INVALID_ARG
    assert B.tcu_sample(None) == B.TCU_ERR_INVALID_ARG
    nan, inf = math.nan, math.inf
    for bad in (dict(dtype=3), dict(vocabulary=0), dict(logits=0), dict(uniform=0), dict(tokens=0), dict(logits=X + 1), dict(uniform=U + 2), dict(uniform=U + 4, f64=1), dict(f64=2),
                dict(tokens=OUT + 4), dict(log_probs=LP + 2), dict(stride=(1 << 38) + 1), dict(temperature=-1.0), dict(temperature=nan), dict(temperature=inf), dict(top_p=nan),
                dict(min_p=nan), dict(d_temperature=T + 1), dict(d_top_k=K + 2), dict(d_top_p=P + 3), dict(d_min_p=M + 1), dict(tokens=X), dict(tokens=U), dict(log_probs=X + 1996),
                dict(log_probs=U), dict(log_probs=OUT + 76), dict(d_temperature=OUT), dict(d_top_k=LP), dict(d_top_p=OUT + 40), dict(d_min_p=LP + 36),
                dict(rows=(1 << 28) - 2, stride=1 << 38, dtype=B.TCU_F32)):
        assert f(**bad) == B.TCU_ERR_INVALID_ARG, bad
    assert f(vocabulary=(1 << 18) + 1) == B.TCU_ERR_UNSUPPORTED
    assert f(rows=1 << 28) == B.TCU_ERR_UNSUPPORTED


def test_python_layer_refuses(B):
    from paper_2411_17887_b200 import api
    x, u = torch.zeros((4, 6)), torch.zeros(4)
    for error, call in ((TypeError, lambda: api.sample(x.double(), u)), (ValueError, lambda: api.sample(x[0], u)), (ValueError, lambda: api.sample(x[:, :0], u)),
                        (ValueError, lambda: api.sample(x, u[:3])), (ValueError, lambda: api.sample(x, u.half())), (ValueError, lambda: api.sample(x, u, temperature=-0.1)),
                        (ValueError, lambda: api.sample(x, u, temperature=math.inf)), (ValueError, lambda: api.sample(x, u, temperature=math.nan)),
                        (ValueError, lambda: api.sample(x, u, temperature=u[:2])), (ValueError, lambda: api.sample(x, u, top_k=u)), (ValueError, lambda: api.sample(x, u, top_p=math.nan)),
                        (ValueError, lambda: api.sample(x, u, top_p=u.double())), (ValueError, lambda: api.sample(x, u, min_p=math.nan)), (ValueError, lambda: api.sample(x, u))):
        with pytest.raises(error):
            call()


def test_reference_by_hand():
    logits = np.log(np.array([1.0, 4.0, 2.0, 4.0, 0.5]))                # weights 1/4, 1, 1/2, 1, 1/8
    assert kept_tokens(logits, 1.0)[0].tolist() == [1, 3, 2, 0, 4]
    assert kept_tokens(logits, 1.0, 3)[0].tolist() == [1, 3, 2]
    assert kept_tokens(logits, 1.0, 0, 1.0, 0.3)[0].tolist() == [1, 3, 2]
    assert kept_tokens(logits, 1.0, 0, 0.6)[0].tolist() == [1, 3]       # 2 of 2.875
    assert kept_tokens(logits, 1.0, 0, 0.7)[0].tolist() == [1, 3, 2]
    assert kept_tokens(logits, 1.0, 1)[0].tolist() == [1] and kept_tokens(logits, 0.0)[0].tolist() == [1] and kept_tokens(logits, 1.0, 0, 0.0)[0].tolist() == [1]
    assert kept_tokens(logits, 1.0, 3, 0.79)[0].tolist() == [1, 3]      # 2 of 2.5
    for u, token, weight in ((0.0, 0, 0.25), (0.08, 0, 0.25), (0.1, 1, 1.0), (0.5, 2, 0.5), (0.95, 3, 1.0), (0.97, 4, 0.125)):
        got, log_prob = token_of(logits, u, 1.0)
        assert got == token and abs(log_prob - math.log(weight / 2.875)) < 1e-14
    assert token_of(logits, 0.99, 1.0, 2) == (3, math.log(0.5))
    assert token_of(np.full(3, -np.inf), 0.5, 1.0) == (-1, -math.inf)
    assert token_of(np.array([np.nan, 0.0, np.inf, np.inf]), 0.6, 1.0) == (3, math.log(0.5))
