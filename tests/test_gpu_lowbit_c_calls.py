"""Calls of the 8-bit and 4-bit entry points that the header allows and the Python binding does not make: outputs that are left out,
off every 16-byte boundary, or wider apart than their rows."""
import pytest
import torch

from tests import lowbit_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dllm():
    from paper_2506_06295_b200 import build as build_mod
    build_mod.build()
    from paper_2506_06295_b200 import dllm as d
    yield d
    d.debug_kv4_plan()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def stream():
    return torch.cuda.current_stream().cuda_stream


def behind(n, dtype, off):
    """n elements of `dtype` that start `off` elements behind a 16-byte boundary, between guards."""
    store = torch.full((n + off + 64,), -77.0, device="cuda").to(dtype)
    return store, store[off:off + n]


def guarded(store, off, n):
    return bool((store[:off] == -77).all()) and bool((store[off + n:] == -77).all())


@pytest.mark.parametrize("kernel,splits", [(1, 1), (1, 4), (1, 11), (2, 1), (2, 3)])
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_without_lse(dllm, kernel, splits, hd):
    g = gen(31)
    a, n, H, Hkv = 40, 1500, 4, 2
    cache = ref.random_cache(dllm, g, 1, Hkv, 1536, hd)
    q = torch.randn((a, H * hd), generator=g, device="cuda").bfloat16()
    dllm.debug_kv4_plan(kernel, splits)
    want, _ = dllm.attention_kv4(q, cache, a, n, H)
    o = torch.zeros_like(want)
    need = dllm.lib.dllm_attention_kv4_scratch_bytes(1, a, n, H, Hkv, hd)
    scratch = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    dllm._check(dllm.lib.dllm_attention_kv4(q.data_ptr(), H * hd, cache.ref, o.data_ptr(), None, a, n, H, None, scratch.data_ptr(), need,
                                            stream()))
    assert torch.equal(o, want)
    dllm.debug_kv4_plan()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off", [0, 1, 2, 4])
def test_load_of_one_tensor_and_off_alignment(dllm, dtype, off):
    g = gen(32)
    B, Hkv, hd, n = 2, 3, 64, 77
    cache = ref.random_cache(dllm, g, B, Hkv, 128, hd)
    want = dllm.kv4_load(cache, n, dtype=dtype)
    size = B * n * Hkv * hd
    code = dllm.BF16 if dtype is torch.bfloat16 else dllm.FP32
    for which in (0, 1, 2):
        (sk, k), (sv, v) = behind(size, dtype, off), behind(size, dtype, off)
        dllm._check(dllm.lib.dllm_kv4_load(cache.ref, n, None, k.data_ptr() if which != 1 else None, v.data_ptr() if which != 0 else None, code,
                                           stream()))
        for skip, s, t, w in ((1, sk, k, want[0]), (0, sv, v, want[1])):
            assert guarded(s, off, size)
            assert bool((t == -77).all()) if which == skip else torch.equal(t, w.flatten())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols,ldq", [(1, 16), (7, 32), (100, 112), (104, 144), (4096, 4112)])
def test_the_gap_behind_rows_of_codes_stays(dllm, dtype, cols, ldq):
    x = torch.randn((5, cols), generator=gen(33), device="cuda").to(dtype)
    q = torch.full((5, ldq), 99, dtype=torch.int8, device="cuda")
    scale = torch.empty(5, device="cuda")
    dllm._check(dllm.lib.dllm_quantize_rows_s8(x.data_ptr(), cols, dllm.BF16 if dtype is torch.bfloat16 else dllm.FP32, q.data_ptr(), ldq,
                                               scale.data_ptr(), 5, cols, stream()))
    codes, s = ref.quantize_rows_s8(x)
    assert torch.equal(q[:, :cols].double(), codes) and torch.equal(scale.double(), s) and bool((q[:, cols:] == 99).all())


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("off", [0, 1, 2, 3])
@pytest.mark.parametrize("M,N,K", [(3, 256, 4096), (60, 130, 300), (150, 300, 200), (300, 777, 9000), (513, 256, 128)])
def test_product_into_an_output_off_alignment(dllm, M, N, K, off, out):
    g = gen(M + off)
    pitch = -(-K // 16) * 16
    A = torch.randint(-128, 128, (M, pitch), generator=g, device="cuda", dtype=torch.int8)[:, :K]
    W = torch.randint(-128, 128, (N, pitch), generator=g, device="cuda", dtype=torch.int8)[:, :K]
    sa, sw = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    want = dllm.gemm_s8(A, sa, W, sw, out_dtype=out)
    store, y = behind(M * N, out, off)
    dllm.gemm_s8(A, sa, W, sw, out=y.view(M, N))
    assert torch.equal(y.view(M, N), want) and guarded(store, off, M * N)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_store_of_keys_and_values_of_different_pitch(dllm, dtype):
    g = gen(34)
    k, v = (torch.randn((2, 9, w), generator=g, device="cuda").to(dtype) for w in (256, 391))
    a, b = (dllm.KV4Cache(2, 2, 64, 128) for _ in range(2))
    dllm.kv4_store(a, k, v[..., 3:259], start=50)
    dllm.kv4_store(b, k.contiguous(), v[..., 3:259].contiguous(), start=50)
    for x, y in zip(a.tensors(), b.tensors()):
        assert torch.equal(x, y)


def test_a_row_whose_step_has_no_number_of_codes(dllm):
    """fp32 rows far from zero: their offset rounds to bf16 by many steps, and codes stay within 0 .. 15."""
    g = gen(35)
    x = 1000 + torch.randn((1, 64, 128), generator=g, device="cuda")
    cache = dllm.KV4Cache(1, 1, 64, 128)
    dllm.kv4_store(cache, x, -x)
    for which, t in ((0, x), (2, -x)):
        code, step, lo = ref.encode4(t.reshape(1, 64, 1, 128))
        assert torch.equal(cache.tensors()[which][0, 0], ref.pack4(code)[0, :, 0])
        assert torch.equal(cache.tensors()[which + 1][0, 0], torch.stack([step, lo], -1).bfloat16()[0, :, 0])
