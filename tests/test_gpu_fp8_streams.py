"""New outputs of a call on a given stream belong to that stream: memory that the
current stream has freed and is still to write is not theirs."""
import pytest
import torch

from paper_2608_01784_gb300 import api
from tests.test_gpu_fp8 import BF16, F32, experts_layer, normal, routing

pytestmark = pytest.mark.gpu
ROWS = 300


def quantize():
    x = normal(1, ROWS, 1024)
    return lambda stream: api.quantize_fp8(x, stream=stream)


def matmul():
    a, b = api.quantize_fp8(normal(1, ROWS, 256)), api.quantize_fp8(normal(2, 2048, 256), 128)
    return lambda stream: (api.matmul_fp8(*a, *b, stream=stream),)


def linear():
    op = api.LinearFp8(*api.quantize_fp8(normal(2, 2048, 256), 128), max_rows=ROWS)
    x = normal(1, ROWS, 256, dtype=BF16)
    return lambda stream: (op.forward(x, stream=stream),)


def experts():
    w = experts_layer(1, 1024, 4, 64)
    op = api.ExpertsFp8(w, d=1024, E=4, inter=64, k_max=2, max_tokens=ROWS)
    h = normal(1, ROWS, 1024, dtype=BF16)
    ids, alpha, k = routing(1, ROWS, 4, 2)
    return lambda stream: (op.forward(h, ids, alpha, k, stream=stream),)


def weights():
    up, down = normal(1, 1, 128, 2048), normal(2, 1, 2048, 64)
    return lambda stream: tuple(api.quantize_experts(up, down, stream).values())


def sample():
    z = normal(1, 70000, 8)
    u = torch.rand(70000, generator=torch.Generator().manual_seed(1)).cuda()
    return lambda stream: api.sample(z, u, stream=stream)


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("call", [quantize, matmul, linear, experts, weights, sample])
def test_new_outputs_belong_to_the_stream(call, handle):
    run = call()
    want = [t.clone() for t in run(None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # blocks of the outputs' sizes, freed before the current stream has written them
    blocks = [torch.empty_like(t) for t in want for _ in range(3)]
    torch.cuda._sleep(100_000_000)
    for t in blocks:
        t.view(torch.uint8).fill_(0x55)
    del blocks, t
    got = run(side.cuda_stream if handle else side)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
