"""A call over the 4-bit cache decides once which kernel it takes and how many ranges of keys: what its scratch was checked
against is what is launched, whatever another host thread does to the tuning hook meanwhile."""
import os
import re
import threading

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2506_06295_b200", "csrc")


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def body(text, name):
    """Of the function `name` (its definition's braces)."""
    at = re.search(re.escape(name) + r"\([^;{]*\)\s*\{", text).end()
    depth, i = 1, at
    while depth:
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        i += 1
    return text[at:i]


def test_a_call_makes_one_plan():
    text, entries = source("kv4_attention.cu"), source("lowbit.cu")
    hook = re.search(r"std::atomic<int>\s+(\w+)", text).group(1)          # one word, read as a whole
    for name in ("plan_kv4", "plan_kv4_weights"):
        assert len(re.findall(hook + r"\.load", body(text, name))) == 1
    assert len(re.findall(hook, text)) == 4                               # its definition, the two plans, the setter
    for name in ("launch_kv4_attention", "launch_kv4_weights", "attention_as", "kv4_attention_scratch_bytes", "kv4_weights_scratch_bytes"):
        assert "plan_kv4" not in body(text, name)
    for name in ("dllm_attention_kv4", "dllm_attention_weights_kv4"):
        b = body(entries, name)
        assert len(re.findall(r"plan_kv4\w*\(", b)) == 1 and "_scratch_bytes(" in b


@pytest.mark.gpu
def test_the_hook_changes_while_calls_run():
    """Scratch for the largest plan, another thread that goes through the plans: every call is right and none is refused."""
    import torch

    from paper_2506_06295_b200 import build as build_mod
    build_mod.build()
    from paper_2506_06295_b200 import dllm
    from tests import lowbit_ref as ref
    g = torch.Generator(device="cuda")
    g.manual_seed(18)
    a, n, H, Hkv, hd = 20, 1000, 4, 2, 64
    cache = ref.random_cache(dllm, g, 1, Hkv, 1024, hd)
    q = torch.randn((a, H * hd), generator=g, device="cuda").bfloat16()
    plans = [(0, 0), (1, 4), (1, 11), (2, 1), (2, 3)]
    need = 0
    for p in plans:
        dllm.debug_kv4_plan(*p)
        need = max(need, dllm.lib.dllm_attention_kv4_scratch_bytes(1, a, n, H, Hkv, hd),
                   dllm.lib.dllm_attention_weights_kv4_scratch_bytes(1, a, H, Hkv))
    scratch = torch.empty(need, dtype=torch.uint8, device="cuda")
    dllm.debug_kv4_plan()
    want, wl, oe, se = ref.attention(q, cache, a, n, H)
    stop = threading.Event()

    def turn():
        while not stop.is_set():
            for p in plans:
                dllm.debug_kv4_plan(*p)

    other = threading.Thread(target=turn)
    other.start()
    try:
        for _ in range(200):
            o, lse = dllm.attention_kv4(q, cache, a, n, H, scratch=scratch)
            w = torch.zeros((1, Hkv, 1024), device="cuda")
            dllm.attention_weights_kv4(q, cache, lse, w, a, n, H, scratch=scratch)
            bound = oe + 2.0 ** -8 * want.abs() * 1.01
            assert bool(((o.double().reshape(want.shape) - want).abs() <= bound).all())
            assert bool(((lse.double().reshape(wl.shape) - wl).abs() <= se + 2.0 ** -23 * wl.abs()).all())
            got, err = ref.weights(q, cache, lse, a, n, H)
            assert bool(((w.double() - got).abs() <= err + 2.0 ** -23 * got).all())
    finally:
        stop.set()
        other.join()
        dllm.debug_kv4_plan()
    dllm.kernel_status()
