"""8-bit integer rows and products against 64-bit forms.

Tolerances.  Codes and scales are the definition's own float32 numbers: equal.  A product's sum is an exact integer; turning it
into fp32 and two multiplications round three times (2^-24 each), the output once more to bf16 (2^-8).  1.01: second order."""
import pytest
import torch

from tests import lowbit_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dllm():
    from paper_2506_06295_b200 import build as build_mod
    build_mod.build()
    from paper_2506_06295_b200 import dllm as d
    return d


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def pitched(t, pitch):
    """The same matrix with rows `pitch` elements apart, the gaps filled with something."""
    store = torch.full((t.shape[0], pitch), 77, dtype=t.dtype, device=t.device)
    store[:, :t.shape[1]] = t
    return store[:, :t.shape[1]]


def check(y, want, dtype):
    tol = (2.0 ** -8 if dtype is torch.bfloat16 else 0.0) + 3 * 2.0 ** -24
    err = (y.double() - want).abs()
    assert bool((err <= 1.01 * tol * want.abs() + 1e-37).all()), float((err - tol * want.abs()).max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,pitch", [(1, 1, 1), (3, 7, 9), (5, 200, 200), (17, 448, 456), (64, 4096, 4096), (2, 18944, 18944),
                                             (3, 33001, 33003), (2, 40000, 40000)])
def test_quantize_rows(dllm, rows, cols, pitch, dtype):
    x = torch.randn((rows, cols), generator=gen(1), device="cuda").to(dtype)
    if rows > 2:
        x[1] = 0
        x[2, cols // 2] = 1e4
    q, s = dllm.quantize_rows_s8(pitched(x, pitch))
    codes, scale = ref.quantize_rows_s8(x)
    assert torch.equal(q.double(), codes) and torch.equal(s.double(), scale)
    assert q.stride(0) % 16 == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_rows_at_ties(dllm, dtype):
    """Rows whose maximum is a short number meet ties, and quotients next to ties, in every other element."""
    g = gen(3)
    top = torch.cat([torch.arange(128, 256, device="cuda"), torch.tensor([127.0, 254.0, 1.0], device="cuda")]).float()
    top = top * 2.0 ** torch.randint(-60, 60, top.shape, generator=g, device="cuda").float()
    half = (torch.randint(-253, 254, (top.numel(), 4096), generator=g, device="cuda").float() * 0.5)
    x = (half.double() * (top.double() / 127)[:, None]).float()
    x = x * (1 + torch.randint(-2, 3, x.shape, generator=g, device="cuda").float() * 2.0 ** -23)
    x[:, 0] = top
    x = x.to(dtype)
    q, s = dllm.quantize_rows_s8(x)
    codes, scale = ref.quantize_rows_s8(x)
    assert torch.equal(q.double(), codes) and torch.equal(s.double(), scale)


def test_quantize_rows_special_values(dllm):
    x = torch.randn((6, 64), generator=gen(2), device="cuda")
    x[0, 3], x[1, 5], x[2, 63] = float("nan"), float("inf"), -float("inf")
    x[3] *= 1e-43 / x[3].abs().max()                # denormal, with a scale of a few units of the last place
    x[4] = 3e38 * torch.sign(x[4])
    q, s = dllm.quantize_rows_s8(x)
    assert not torch.isfinite(s[:3]).any() and not q[:3].any()
    codes, scale = ref.quantize_rows_s8(x[3:])
    assert torch.equal(q[3:].double(), codes) and torch.equal(s[3:].double(), scale)
    w = torch.ones((5, 64), dtype=torch.int8, device="cuda")
    y = dllm.gemm_s8(q, s, w, torch.ones(5, device="cuda"))
    assert y[:3].isnan().all() and y[3:].isfinite().all()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 128, 64), (3, 4096, 4096), (17, 300, 130), (32, 129, 128), (33, 1000, 515), (64, 2560, 448),
                                   (65, 512, 2048), (96, 257, 333), (128, 1792, 4097), (129, 100, 200), (144, 2560, 448),
                                   (200, 3584, 2000), (256, 4096, 1024), (300, 777, 9000), (513, 130, 777), (1024, 1792, 1024),
                                   (777, 2051, 4096), (2050, 900, 516)])
def test_product(dllm, M, N, K, out):
    g = gen(M * 7 + N + K)
    A = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    W = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    sa, sw = (torch.randn(n, generator=g, device="cuda") for n in (M, N))
    up = lambda c: -(-c // 16) * 16                                          # noqa: E731
    y = dllm.gemm_s8(pitched(A, up(K) + 16), sa, pitched(W, up(K)), sw, out_dtype=out)
    check(y, (A.double() @ W.double().t()) * sa.double()[:, None] * sw.double()[None, :], out)
    dllm.kernel_status()


def test_sums_of_the_largest_k(dllm):
    """-128 * -128 * 131071 is the largest sum there is."""
    K = 131071
    A = torch.full((2, K + 1), -128, dtype=torch.int8, device="cuda")[:, :K]
    W = torch.full((3, K + 1), -128, dtype=torch.int8, device="cuda")[:, :K]
    one = torch.ones(3, device="cuda")
    y = dllm.gemm_s8(A, one[:2].contiguous(), W, one)
    check(y, torch.full((2, 3), 16384.0 * K, dtype=torch.float64, device="cuda"), torch.float32)


@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("M,N,K", [(1, 64, 200), (3, 4096, 4096), (128, 3584, 1895), (500, 1000, 2048), (8, 5, 18944)])
def test_linear(dllm, M, N, K, dtype, out):
    g = gen(M + N * 3 + K)
    x = torch.randn((M, K), generator=g, device="cuda").to(dtype)
    W, sw = dllm.quantize_rows_s8(0.02 * torch.randn((N, K), generator=g, device="cuda"))
    codes, scale = ref.quantize_rows_s8(x)
    want = (codes @ W.double().t()) * scale[:, None] * sw.double()[None, :]
    check(dllm.linear_s8(pitched(x, K + 5), W, sw, out_dtype=out), want, out)
    # the caller's output and scratch, another stream, a captured call replayed on new rows
    y = torch.empty((M, N), dtype=out, device="cuda")
    scratch = torch.empty(dllm.lib.dllm_linear_s8_scratch_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert dllm.linear_s8(x, W, sw, out=y, scratch=scratch, stream=side) is y
    side.synchronize()
    check(y, want, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dllm.linear_s8(x, W, sw, out=y, scratch=scratch)
    x.copy_(torch.randn((M, K), generator=g, device="cuda").to(dtype))
    for _ in range(2):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        codes, scale = ref.quantize_rows_s8(x)
        check(y, (codes @ W.double().t()) * scale[:, None] * sw.double()[None, :], out)
    dllm.kernel_status()


def test_two_calls_on_two_streams(dllm):
    g = gen(9)
    jobs = []
    for M, N, K in ((3, 4096, 4096), (200, 3584, 2000)):
        x = torch.randn((M, K), generator=g, device="cuda").bfloat16()
        W, sw = dllm.quantize_rows_s8(0.02 * torch.randn((N, K), generator=g, device="cuda"))
        codes, scale = ref.quantize_rows_s8(x)
        jobs.append((x, W, sw, (codes @ W.double().t()) * scale[:, None] * sw.double()[None, :], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        ys = [dllm.linear_s8(x, W, sw, stream=s) for x, W, sw, _, s in jobs]
        torch.cuda.synchronize()
        for y, (_, _, _, want, _) in zip(ys, jobs):
            check(y, want, torch.float32)
