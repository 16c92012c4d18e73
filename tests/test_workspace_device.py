"""A workspace that is not device memory is refused before any launch: its
address would reach a kernel."""
import pytest
import torch


def test_host_workspace_is_refused():
    from paper_2606_11867_amd import api
    ws = torch.zeros(512, dtype=torch.uint8)
    with pytest.raises(ValueError):
        api._ws(ws, torch.device("cuda:0"))
    with pytest.raises(ValueError):
        api._ws(ws, ws.device)
    assert api._ws(None, torch.device("cuda:0")) == (None, 0)


@pytest.mark.gpu
def test_calls_refuse_a_host_workspace(gpu):
    from paper_2606_11867_amd import api
    x = torch.randn(3, 40000, device=gpu)
    with pytest.raises(ValueError):
        api.token_logprobs(x, n_top=2, ws=api.logprobs_workspace("cpu"))
    x = torch.randn(5, 16, device=gpu)
    with pytest.raises(ValueError):
        api.router_fwd(x, 2, ws=api.router_workspace(16, "cpu"))
    with pytest.raises(ValueError):  # every other byte of one
        api.router_fwd(x, 2, ws=torch.zeros(2 * api.router_workspace(16, gpu).numel(), dtype=torch.uint8, device=gpu)[::2])
    offset = torch.zeros(2, dtype=torch.int32, device=gpu)
    w = torch.zeros(1, 256, 128, device=gpu, dtype=torch.bfloat16)
    down = torch.zeros(1, 128, 128, device=gpu, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        api.grouped_ffn_fwd(torch.zeros(8, 128, device=gpu, dtype=torch.bfloat16), offset, offset[:1], w, down,
                            ws=torch.zeros(1 << 20, dtype=torch.uint8))
