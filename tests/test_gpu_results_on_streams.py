"""Results that a call makes for itself while it runs on another stream than the current one: their memory may not be what the
current stream has freed but not yet written to the end."""
import pytest

pytestmark = pytest.mark.gpu
M, K, N, G = 40, 512, 4096, 64                                       # y: 640 KB of fp32


@pytest.fixture(scope="module")
def gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2508_06753_b200 import binding, build
    build.build()
    binding.lib()
    return torch, binding


def _calls(torch, b):
    """name -> call(stream) that makes its results itself"""
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(0, 4, (N, K), generator=g, device="cuda", dtype=torch.uint8)
    scale = 0.02 * torch.exp(0.5 * torch.randn((N, K // G), generator=g, device="cuda"))
    packed = b.w2_pack(codes)
    x = torch.randn((M, K), generator=g, device="cuda").to(torch.bfloat16)
    a, s = b.a8_quantize(x)
    ws = b.new_workspace(max(b.w2a8_workspace_bytes(M, N, K, G), b.w2a8_grouped_workspace_bytes([N], M, K, G)))
    lora = b.LoraGroup([torch.randn((2, 8, K), generator=g, device="cuda").to(torch.bfloat16)],
                       [torch.randn((2, N, 8), generator=g, device="cuda").to(torch.bfloat16)])
    owner = (torch.arange(M, device="cuda") % 3 - 1).to(torch.int32)
    h16 = scale.half()
    return {
        "w2a8_lora_grouped": lambda st: b.w2a8_lora_grouped(x, owner, lora, stream=st)[0],
        "w2a8_gemm": lambda st: b.w2a8_gemm(a, s, packed, scale, G, ws, stream=st),
        "w2a8_gemm_h16": lambda st: b.w2a8_gemm_h16(a, s, packed, h16, G, ws, stream=st),
        "w2a16_gemm": lambda st: b.w2a16_gemm(x, packed, scale, G, ws, stream=st),
        "w2a8_linear": lambda st: b.w2a8_linear(x, packed, scale, G, ws, stream=st)[0],
        "w2a8_gemm_grouped": lambda st: b.w2a8_gemm_grouped(a, s, b.Group([packed], [scale]), G, ws, stream=st)[0],
        "w2a8_linear_grouped": lambda st: b.w2a8_linear_grouped(x, b.Group([packed], [scale]), G, ws, a=a, a_scale=s, stream=st)[0],
        "w2_pack": lambda st: b.w2_pack(codes, stream=st),
        "a8_quantize": lambda st: b.a8_quantize(x, stream=st)[0],
    }


@pytest.mark.parametrize("name", ["w2a8_lora_grouped", "w2a8_gemm", "w2a8_gemm_h16", "w2a16_gemm", "w2a8_linear", "w2a8_gemm_grouped",
                                  "w2a8_linear_grouped", "w2_pack", "a8_quantize"])
def test_memory_that_the_current_stream_still_writes(gpu, name):
    torch, b = gpu
    call = _calls(torch, b)[name]
    side = torch.cuda.Stream()
    want = call(None).clone()
    like = call(None)
    shape, dtype = like.shape, like.dtype
    del like
    torch.cuda.synchronize()
    late = [torch.empty(shape, dtype=dtype, device="cuda") for _ in range(32)]       # all that is free of this size
    late[0].fill_(1)                                                 # a kernel that is loaded first would outlast the sleep
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)                                    # some ten milliseconds
    for t in late:
        t.fill_(77)
    del late, t                                                      # free, and written once the sleep is over
    y = call(side)
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_result_freed_while_the_current_stream_reads_it(gpu):
    """The other end: what the side stream takes next is not memory that the current stream still reads."""
    torch, b = gpu
    call = _calls(torch, b)["w2a8_lora_grouped"]
    side = torch.cuda.Stream()
    want = call(None).clone()
    torch.cuda.synchronize()
    y = call(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(20_000_000)
    copy = y.clone()
    del y
    with torch.cuda.stream(side):
        others = [torch.full((M, N), 5.0, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(copy, want) and len(others) == 4
