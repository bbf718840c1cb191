"""A call of the library may be the first thing that a host thread does with CUDA: layers and adapters whose tensor maps are made then."""
import threading

import pytest
import torch

import paper_2503_13565_b200 as mxq

pytestmark = pytest.mark.gpu


def in_a_thread(f):
    result = []

    def work():
        try:
            result.append(f())
        except BaseException as e:  # noqa: BLE001
            result.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    if isinstance(result[0], BaseException):
        raise result[0]
    return result[0]


@pytest.mark.parametrize("m", [9, 600])
def test_adapters(m):
    x, a, b = (torch.randn(*s, device="cuda").bfloat16() for s in ((m, 256), (2, 16, 256), (2, 40, 16)))
    ids, out = (torch.arange(m, device="cuda") % 2).int(), torch.empty(m, 40, device="cuda")
    ws = torch.zeros(mxq.mxq_lora_workspace_bytes(m, 40, 256, 16, 2), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    in_a_thread(lambda: mxq.mxq_lora(x, a, b, ids, out=out, workspace=ws, stream=stream))
    torch.cuda.synchronize()
    assert torch.equal(out, mxq.mxq_lora(x, a, b, ids))


@pytest.mark.parametrize("m", [1, 8])
def test_a_layer_with_new_weights(m):
    codes, scales = mxq.mxq_quantize(torch.randn(512, 4096, device="cuda").bfloat16())
    x, out = torch.randn(m, 4096, device="cuda").bfloat16(), torch.empty(m, 512, device="cuda")
    ws = mxq.new_workspace(mxq.mxq_linear_workspace_bytes(m, 512, 4096))
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    in_a_thread(lambda: mxq.mxq_linear(x, codes, scales, out=out, workspace=ws, stream=stream))
    torch.cuda.synchronize()
    assert torch.equal(out, mxq.mxq_linear(x, codes, scales, workspace=mxq.new_workspace(mxq.mxq_linear_workspace_bytes(m, 512, 4096))))
