"""What the 8-bit products and the 4-bit cache's entry points refuse, on the host: no call here reaches a kernel."""
import ctypes as C

import pytest

from paper_2506_06295_b200 import build as build_mod

P = 0x100000          # an aligned address that nothing dereferences: every call below is refused first


@pytest.fixture(scope="module")
def dllm():
    build_mod.build()
    from paper_2506_06295_b200 import dllm as d
    return d


def refused(dllm, fn, *args, status=None):
    st = getattr(dllm.lib, fn)(*args)
    assert st == (dllm.INVALID_ARG if status is None else status), (fn, args, st)
    assert dllm.last_error()


def cache(dllm, B=2, Hkv=4, cap=128, hd=128, at=P, step=1 << 24, **over):
    f = dict(k_codes=at, k_params=at + step, v_codes=at + 2 * step, v_params=at + 3 * step, B=B, n_kv_heads=Hkv, capacity=cap,
             head_dim=hd)
    f.update(over)
    return C.byref(dllm.Kv4CacheStruct(*(f[k] for k, _ in dllm.Kv4CacheStruct._fields_)))


def test_quantize_rows(dllm):
    good = dict(x=P, ldx=100, dt=1, q=P, ldq=112, s=P, rows=3, cols=100)
    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(rows=0), dict(cols=0), dict(rows=-1), dict(ldx=99), dict(ldq=96),
                dict(ldq=120), dict(dt=2), dict(x=P + 1), dict(q=P + 8)):
        a = {**good, **bad}
        refused(dllm, "dllm_quantize_rows_s8", a["x"], a["ldx"], a["dt"], a["q"], a["ldq"], a["s"], a["rows"], a["cols"], None)


def test_gemm(dllm):
    need = dllm.lib.dllm_gemm_s8_scratch_bytes(384, 1024, 18944)
    assert need > 0 and dllm.lib.dllm_gemm_s8_scratch_bytes(0, 256, 4096) == 0 == dllm.lib.dllm_gemm_s8_scratch_bytes(3, 256, 4096)
    good = dict(A=P, lda=18944, sa=P, W=P, ldw=18944, sw=P, C=P, dt=0, M=384, N=1024, K=18944, s=P, sb=need)
    for bad in (dict(A=None), dict(sa=None), dict(W=None), dict(sw=None), dict(C=None), dict(M=0), dict(N=0), dict(K=0),
                dict(lda=18952), dict(lda=18928), dict(ldw=18952), dict(ldw=18928), dict(A=P + 8), dict(W=P + 4), dict(dt=3), dict(s=None),
                dict(sb=need - 1), dict(s=P + 8), dict(C=P + 2)):
        a = {**good, **bad}
        refused(dllm, "dllm_gemm_s8", a["A"], a["lda"], a["sa"], a["W"], a["ldw"], a["sw"], a["C"], a["dt"], a["M"], a["N"], a["K"],
                a["s"], a["sb"], None)
    refused(dllm, "dllm_gemm_s8", P, 131072, P, P, 131072, P, P, 0, 3, 256, 131072, P, 1 << 40, None, status=dllm.UNSUPPORTED)
    refused(dllm, "dllm_gemm_s8", P, 16, P, P, 16, P, P, 0, (1 << 30) + 1, 1, 16, P, 1 << 40, None, status=dllm.UNSUPPORTED)
    refused(dllm, "dllm_quantize_rows_s8", P, 1 << 31, 1, P, 1 << 31, P, 1, (1 << 30) + 1, None, status=dllm.UNSUPPORTED)
    assert dllm.lib.dllm_gemm_s8_scratch_bytes((1 << 30) + 1, 1, 16) == 0


def test_linear(dllm):
    need = dllm.lib.dllm_linear_s8_scratch_bytes(3, 256, 4096)
    good = dict(x=P, ldx=4096, dt=1, W=P, ldw=4096, sw=P, y=P, out=1, M=3, N=256, K=4096, s=P, sb=need)
    for bad in (dict(x=None), dict(ldx=4095), dict(dt=5), dict(W=None), dict(y=None), dict(out=-1), dict(M=0), dict(s=None),
                dict(sb=need - 1), dict(x=P + 1), dict(y=P + 1)):
        a = {**good, **bad}
        refused(dllm, "dllm_linear_s8", a["x"], a["ldx"], a["dt"], a["W"], a["ldw"], a["sw"], a["y"], a["out"], a["M"], a["N"], a["K"],
                a["s"], a["sb"], None)


def test_caches(dllm):
    for over, status in ((dict(k_codes=None), None), (dict(v_params=None), None), (dict(B=0), None), (dict(n_kv_heads=0), None),
                         (dict(capacity=100), None), (dict(capacity=0), None), (dict(head_dim=96), dllm.UNSUPPORTED),
                         (dict(k_codes=P + 8), None), (dict(B=70000), dllm.UNSUPPORTED),
                         (dict(capacity=(1 << 24) + 64), dllm.UNSUPPORTED)):
        refused(dllm, "dllm_kv4_load", cache(dllm, **over), 10, None, P, P, 0, None, status=status)
    refused(dllm, "dllm_kv4_load", None, 10, None, P, P, 0, None)


def test_store_and_load(dllm):
    c = cache(dllm)
    good = dict(k=P, ldk=512, v=P, ldv=512, dt=1, a=4, pos=None, start=0)
    for bad in (dict(k=None), dict(v=None), dict(ldk=511), dict(ldv=511), dict(dt=2), dict(a=0), dict(start=-1), dict(start=125),
                dict(a=129), dict(k=P + 1)):
        a = {**good, **bad}
        refused(dllm, "dllm_kv4_store", c, a["k"], a["ldk"], a["v"], a["ldv"], a["dt"], a["a"], a["pos"], a["start"], None)
    for n, k, v, dt in ((0, P, P, 0), (129, P, P, 0), (5, None, None, 0), (5, P, P, 2), (5, P + 1, P, 1)):
        refused(dllm, "dllm_kv4_load", c, n, None, k, v, dt, None)


def test_attention_and_weights(dllm):
    c = cache(dllm)
    need = dllm.lib.dllm_attention_kv4_scratch_bytes(2, 3, 128, 8, 4, 128)
    good = dict(q=P, ldq=1024, o=P, lse=P, a=3, n=128, H=8, s=P, sb=need)
    for bad in (dict(q=None), dict(q=P + 8), dict(ldq=1023), dict(ldq=1016), dict(a=0), dict(n=0), dict(n=129), dict(H=6), dict(H=0)):
        a = {**good, **bad}
        refused(dllm, "dllm_attention_kv4", a["q"], a["ldq"], c, a["o"], a["lse"], a["a"], a["n"], a["H"], None, a["s"], a["sb"], None)
        refused(dllm, "dllm_attention_weights_kv4", a["q"], a["ldq"], c, P, P, a["a"], a["n"], a["H"], None, P, 1 << 40, None)
    for o in (None, P + 8):
        refused(dllm, "dllm_attention_kv4", P, 1024, c, o, P, 3, 128, 8, None, P, need, None)
    for lse, w in ((None, P), (P, None)):
        refused(dllm, "dllm_attention_weights_kv4", P, 1024, c, lse, w, 3, 128, 8, None, P, 1 << 40, None)
    need = dllm.lib.dllm_attention_weights_kv4_scratch_bytes(2, 100, 8, 4)
    assert need > 0
    for s, sb in ((None, need), (P, need - 1), (P + 8, need)):
        refused(dllm, "dllm_attention_weights_kv4", P, 1024, c, P, P, 100, 128, 8, None, s, sb, None)
    big = cache(dllm, B=1, Hkv=1, cap=8192)
    need = dllm.lib.dllm_attention_kv4_scratch_bytes(1, 1, 8192, 1, 1, 128)
    assert need > 0
    for s, sb in ((None, need), (P, need - 4), (P + 8, need)):
        refused(dllm, "dllm_attention_kv4", P, 128, big, P, P, 1, 8192, 1, None, s, sb, None)
    refused(dllm, "dllm_attention_kv4", P, 1024, c, P, P, 1 << 27, 128, 8, None, P, 1 << 50, None, status=dllm.UNSUPPORTED)


def test_evict(dllm):
    src, far = cache(dllm, cap=256), P + (1 << 30)
    dst = cache(dllm, cap=64, at=far)
    good = dict(src=src, w=P + (1 << 28), n=200, keep=50, first=3, last=5, lens=None, dst=dst, dw=far + (1 << 28), idx=far + (1 << 29), nl=far + (3 << 28))
    for bad in (dict(src=None), dict(dst=None), dict(w=None), dict(dw=None), dict(idx=None), dict(nl=None), dict(n=0), dict(n=257),
                dict(keep=0), dict(keep=65), dict(first=-1), dict(last=-1), dict(first=30, last=21), dict(w=P + (1 << 28) + 4),
                dict(dst=cache(dllm, cap=64, at=far, hd=64)), dict(dst=cache(dllm, cap=64, at=far, Hkv=2)),
                dict(lens=far + (3 << 28)), dict(lens=far + (3 << 28) - 4),
                dict(dst=cache(dllm, cap=64, at=P)), dict(dst=src), dict(dw=P + (1 << 28)), dict(idx=P), dict(nl=P + 64)):
        a = {**good, **bad}
        refused(dllm, "dllm_kv4_evict", a["src"], a["w"], a["n"], a["keep"], a["first"], a["last"], a["lens"], a["dst"], a["dw"], a["idx"],
                a["nl"], None)


def test_evict_into_outputs_that_overlap(dllm):
    """The index is read back to move the rows: another output over it would send the reads anywhere."""
    src, far = cache(dllm, cap=256), P + (1 << 30)
    dst = cache(dllm, cap=64, at=far)
    good = dict(dw=far + (1 << 28), idx=far + (1 << 29), nl=far + (3 << 28))
    at = dict(k=far, kp=far + (1 << 24), v=far + (2 << 24), vp=far + (3 << 24))   # of 2 * 4 * 64 rows
    for bad in (dict(idx=good["dw"]), dict(idx=good["dw"] + 2 * 4 * 64 * 4 - 4), dict(dw=good["idx"] + 2 * 4 * 50 * 4 - 16), dict(nl=good["idx"]),
                dict(nl=good["dw"] + 16), dict(idx=at["k"]), dict(idx=at["vp"] + 16), dict(dw=at["v"]), dict(nl=at["kp"])):
        a = {**good, **bad}
        refused(dllm, "dllm_kv4_evict", src, P + (1 << 28), 200, 50, 3, 5, None, dst, a["dw"], a["idx"], a["nl"], None)
        assert "outputs overlap" in dllm.last_error()
    refused(dllm, "dllm_kv4_evict", src, P + (1 << 28), 200, 50, 3, 5, None, cache(dllm, cap=64, at=far, v_params=at["k"]), *good.values(), None)


def test_arrays_of_words_off_alignment(dllm):
    """A load from such an address would fault; NULL where it is allowed is none."""
    c, big = cache(dllm), cache(dllm, at=P + (1 << 30))
    calls = [("dllm_quantize_rows_s8", (P, 100, 1, P, 112, P, 3, 100, None), (5,)),
             ("dllm_gemm_s8", (P, 4096, P, P, 4096, P, P, 1, 3, 256, 4096, P, 1 << 30, None), (2, 5)),
             ("dllm_linear_s8", (P, 4096, 1, P, 4096, P, P, 1, 3, 256, 4096, P, 1 << 30, None), (5,)),
             ("dllm_kv4_store", (c, P, 512, P, 512, 1, 4, P, 0, None), (7,)),
             ("dllm_kv4_load", (c, 10, P, P, P, 0, None), (2,)),
             ("dllm_attention_kv4", (P, 1024, c, P, P, 3, 128, 8, P, P, 1 << 40, None), (4, 8)),
             ("dllm_attention_weights_kv4", (P, 1024, c, P, P, 3, 128, 8, P, P, 1 << 40, None), (3, 4, 8)),
             ("dllm_kv4_evict", (c, P + (1 << 28), 100, 50, 0, 0, P + (1 << 29), big, P + (5 << 28), P + (6 << 28), P + (7 << 28), None),
              (6, 8, 9, 10))]
    for name, args, words in calls:
        for w in words:
            for off in (1, 2):
                refused(dllm, name, *(x + off if k == w else x for k, x in enumerate(args)))
                assert "aligned" in dllm.last_error()


def test_binding_refuses_what_the_library_cannot_see(dllm):
    import torch
    with pytest.raises(dllm.DllmError):        # no CUDA tensors
        dllm.quantize_rows_s8(torch.zeros(3, 16))
    with pytest.raises(dllm.DllmError):
        dllm.gemm_s8(torch.zeros(3, 16, dtype=torch.int8), torch.zeros(3), torch.zeros(4, 16, dtype=torch.int8), torch.zeros(4))
    with pytest.raises(dllm.DllmError):
        dllm.KV4Cache.from_tensors(*(torch.zeros((1, 1, 64, w), dtype=torch.uint8) for w in (64, 2, 64, 2)))
    c = dllm.KV4Cache(1, 2, 64, 64, device="cpu")
    assert c.capacity == 64 and dllm.KV4Cache(1, 2, 65, 64, device="cpu").capacity == 128
    with pytest.raises(dllm.DllmError):
        dllm.kv4_load(c, 10)          # on the CPU
    with pytest.raises(dllm.DllmError):
        dllm.kv4_store(c, torch.zeros(1, 3, 128), torch.zeros(1, 4, 128))
    # rows that no single pitch describes
    with pytest.raises(dllm.DllmError):
        dllm._row_pitch(torch.zeros(2, 4, 8)[:, :3], 8, "x")
    assert dllm._row_pitch(torch.zeros(2, 3, 24)[:, :, 8:16], 8, "x") == 24
    assert dllm._row_pitch(torch.zeros(1, 1, 24)[:, :, 8:16], 8, "x") == 16


def test_binding_refuses_a_stream_of_another_device(dllm):
    """Which would otherwise be left aside for the current one of the tensors' device."""
    import types

    import torch
    on = lambda i, **more: types.SimpleNamespace(device=torch.device("cuda", i), is_cuda=True, get_device=lambda: i, **more)  # noqa: E731
    x, stream = on(0), on(1)
    cache = types.SimpleNamespace(_base=x, tensors=lambda: (x, x, x, x))
    for call in (lambda: dllm.quantize_rows_s8(x, stream=stream), lambda: dllm.gemm_s8(x, x, x, x, stream=stream),
                 lambda: dllm.linear_s8(x, x, x, stream=stream), lambda: dllm.kv4_store(cache, x, x, stream=stream),
                 lambda: dllm.kv4_load(cache, 1, stream=stream), lambda: dllm.attention_kv4(x, cache, 1, 1, 1, stream=stream),
                 lambda: dllm.attention_weights_kv4(x, cache, x, x, 1, 1, 1, stream=stream),
                 lambda: dllm.kv4_evict(cache, x, 1, 1, stream=stream)):
        with pytest.raises(dllm.DllmError, match="stream of cuda:1"):
            call()
