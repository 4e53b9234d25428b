"""The bounded waits of the 8-bit and 4-bit kernels, made to run out without faulting or hanging anything: a host-set flag makes
one CTA of a launch leave out one copy or one arrival, and a limit of a few milliseconds ends the waits for it.  The call reports
DLLM_TIMEOUT once, what it could not finish stays unwritten, and the next call works as if nothing had happened."""
import pytest
import torch

from tests import lowbit_ref as ref

pytestmark = pytest.mark.gpu
LIMIT_NS = 3_000_000      # 3 ms per wait


@pytest.fixture(scope="module")
def dllm():
    from paper_2506_06295_b200 import build as build_mod
    build_mod.build()
    from paper_2506_06295_b200 import dllm as d
    yield d
    d.debug_skip_one_load(False)          # whatever a failing test left behind
    d.debug_set_wait_limit_ns(0)
    d.debug_kv4_plan()


def run_out(dllm, call):
    """`call` with one of its CTAs' waits running out: it must report that, at its limit, and once."""
    dllm.kernel_status()                  # clean to start with
    dllm.debug_set_wait_limit_ns(LIMIT_NS)
    dllm.debug_skip_one_load(True)
    try:
        t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        t0.record()
        call()
        t1.record()
        with pytest.raises(dllm.DllmError) as e:
            dllm.kernel_status()
        assert e.value.status == dllm.TIMEOUT
        assert 0.5 * LIMIT_NS / 1e6 < t0.elapsed_time(t1) < 1000.0
    finally:
        dllm.debug_skip_one_load(False)
        dllm.debug_set_wait_limit_ns(0)
    dllm.kernel_status()                  # the word was cleared by the read


@pytest.mark.parametrize("a,n,hd", [(512, 512, 128), (512, 512, 64), (256, 40000, 128)])
def test_weights_are_added_whole_or_not_at_all(dllm, a, n, hd):
    """512 rows of two heads over 512 keys: four units of 256 keys, their rows in eight shares of one tile of 128 each, the last
    of which gives up.  40000 keys: a CTA for each of several units.  The keys of the unit that gave up keep their weights to the
    bit; every other key gets all of its sum or nothing."""
    g = torch.Generator(device="cuda")
    g.manual_seed(a + n + hd)
    Hkv, H, cap = 2, 4, -(-n // 64) * 64
    cache = ref.random_cache(dllm, g, 1, Hkv, cap, hd)
    q = torch.randn((a, H * hd), generator=g, device="cuda").bfloat16()
    _, lse = dllm.attention_kv4(q, cache, a, n, H)
    had = torch.rand((1, Hkv, cap), generator=g, device="cuda")
    want = had.clone()
    dllm.attention_weights_kv4(q, cache, lse, want, a, n, H)
    w = had.clone()
    run_out(dllm, lambda: dllm.attention_weights_kv4(q, cache, lse, w, a, n, H))
    assert torch.equal(w[0, 0, :256], had[0, 0, :256])
    assert bool(((w == had) | (w == want)).all())
    assert n > 1000 or torch.equal(w[0, 1], want[0, 1]) and torch.equal(w[0, 0, 256:], want[0, 0, 256:])
    w = had.clone()
    dllm.attention_weights_kv4(q, cache, lse, w, a, n, H)
    assert torch.equal(w, want)
    dllm.kernel_status()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", [(3, 300, 4096), (60, 300, 2048), (40, 300, 200), (200, 513, 4096)])
def test_a_tile_of_a_product_is_written_whole_or_not_at_all(dllm, M, N, K, out):
    """Few rows: the first tile of 128 columns is cut into ranges of k (eight, four, one and eight of them) whose last one gives up.
    The tile keeps what stood there; the others are right."""
    g = torch.Generator(device="cuda")
    g.manual_seed(M + K)
    A = torch.randint(-128, 128, (M, -(-K // 16) * 16), generator=g, device="cuda", dtype=torch.int8)[:, :K]
    W = torch.randint(-128, 128, (N, -(-K // 16) * 16), generator=g, device="cuda", dtype=torch.int8)[:, :K]
    sa, sw = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    want = dllm.gemm_s8(A, sa, W, sw, out_dtype=out)
    y = torch.full((M, N), -77.0, dtype=out, device="cuda")
    run_out(dllm, lambda: dllm.gemm_s8(A, sa, W, sw, out=y))
    rows = min(M, 128)                   # of a tile
    part = want.clone()
    part[:rows, :128] = -77.0
    assert torch.equal(y, part)
    assert dllm.gemm_s8(A, sa, W, sw, out=y) is y
    dllm.kernel_status()
    assert torch.equal(y, want)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("splits", [1, 3])
def test_attention_of_many_rows_gives_up_and_goes_on(dllm, hd, splits):
    """300 rows of two heads over 700 keys: the CTA of the first 256 rows of the first head (and of the first range of keys, where
    there are several) gives up.  Its rows stay as they were (with one range); all others are right."""
    g = torch.Generator(device="cuda")
    g.manual_seed(hd + splits)
    a, n, H = 300, 700, 2
    cache = ref.random_cache(dllm, g, 1, H, 704, hd)
    q = torch.randn((a, H * hd), generator=g, device="cuda").bfloat16()
    dllm.debug_kv4_plan(2, splits)
    try:
        want, want_lse = dllm.attention_kv4(q, cache, a, n, H)
        o, lse = torch.full_like(want, -77.0), torch.full_like(want_lse, -77.0)
        need = dllm.lib.dllm_attention_kv4_scratch_bytes(1, a, n, H, H, hd)
        assert (need > 0) == (splits > 1)
        scratch = torch.zeros(max(need, 16), dtype=torch.uint8, device="cuda")
        run_out(dllm, lambda: dllm._check(dllm.lib.dllm_attention_kv4(
            q.data_ptr(), H * hd, cache.ref, o.data_ptr(), lse.data_ptr(), a, n, H, None, scratch.data_ptr(), need,
            torch.cuda.current_stream().cuda_stream)))
        lost = torch.zeros((a, H), dtype=torch.bool, device="cuda")
        lost[:256, 0] = True
        if splits == 1:
            assert bool((o.reshape(a, H, hd)[lost] == -77.0).all()) and bool((lse[lost] == -77.0).all())
        assert torch.equal(o.reshape(a, H, hd)[~lost], want.reshape(a, H, hd)[~lost]) and torch.equal(lse[~lost], want_lse[~lost])
        o, lse = dllm.attention_kv4(q, cache, a, n, H, scratch=scratch if need else None)
        assert torch.equal(o, want) and torch.equal(lse, want_lse)
        dllm.kernel_status()
    finally:
        dllm.debug_kv4_plan()
