"""Which device linear_attention_status() asks, without a GPU."""
from types import SimpleNamespace

import pytest
import torch


@pytest.fixture()
def api(monkeypatch):
    from paper_2411_17887_b200 import build
    build.build()
    from paper_2411_17887_b200 import api
    status = {i: SimpleNamespace(error=SimpleNamespace(value=0)) for i in range(2)}
    waited = []
    monkeypatch.setattr(api, "_status", status)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index=None: SimpleNamespace(synchronize=lambda: waited.append(0 if index is None else index)))
    api.waited = waited
    return api


@pytest.mark.parametrize("asked,index", [(None, 0), ("cuda", 0), (torch.device("cuda"), 0), ("cuda:0", 0), (0, 0), ("cuda:1", 1), (torch.device("cuda", 1), 1), (1, 1)])
def test_status_of_a_device(api, asked, index):
    assert api.linear_attention_status(asked) == api.B.TCU_OK
    api._status[index].error.value = 5
    assert api.linear_attention_status(asked) == api.B.TCU_ERR_TIMEOUT
    api._status[index].error.value = 0
    api._status[1 - index].error.value = 5
    assert api.linear_attention_status(asked) == api.B.TCU_OK
    assert api.waited == [index] * 3
    api._status.clear()
    assert api.linear_attention_status(asked) == api.B.TCU_OK              # no call was made there


def test_status_of_something_else(api):
    with pytest.raises(ValueError):
        api.linear_attention_status("cpu")
