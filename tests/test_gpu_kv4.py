"""The 4-bit K / V cache: rows in and out, attention over it, weights and eviction, against 64-bit forms.

Tolerances.  What is stored, read back, chosen and moved is defined in float32 arithmetic and compared for equality; a number
read back is lo + step * code rounded once.  Attention and weights: see lowbit_ref."""
import math

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


def lens_of(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- rows in and out
def expected_store(codes, params, x, pos, B, Hkv, hd):
    """Plain store of x [B, a, Hkv * hd] at pos [B][a] into clones of codes / params."""
    codes, params = codes.clone(), params.clone()
    code, step, lo = ref.encode4(x.reshape(B, -1, Hkv, hd))
    packed, pair = ref.pack4(code), torch.stack([step, lo], -1).bfloat16()
    for b in range(B):
        for j, p in enumerate(pos[b]):
            if 0 <= p < codes.shape[2]:
                codes[b, :, p], params[b, :, p] = packed[b, j], pair[b, j]
    return codes, params


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,a,cap,Hkv,hd,kind", [(1, 1, 64, 1, 64, "start"), (2, 5, 128, 3, 128, "start"), (1, 64, 768, 32, 128, "pos"),
                                                 (3, 100, 192, 4, 64, "pos"), (2, 130, 192, 7, 128, "odd"), (1, 700, 768, 2, 64, "odd")])
def test_store_and_load(dllm, B, a, cap, Hkv, hd, kind, dtype):
    g = gen(a + cap)
    W = Hkv * hd
    lead = W if kind != "odd" else 3                  # odd: rows off every 16-byte boundary
    rows = torch.randn((B, a, lead + 2 * W + (lead == 3)), generator=g, device="cuda").to(dtype)
    k, v = rows[:, :, lead:lead + W], rows[:, :, lead + W:lead + 2 * W]
    cache = ref.random_cache(dllm, g, B, Hkv, cap, hd)
    before = [t.clone() for t in cache.tensors()]
    start, pos = 0, None
    if kind == "start":
        start = cap - a - 1
        places = [list(range(start, start + a))] * B
    else:
        pos = torch.stack([torch.randperm(cap, generator=g, device="cuda")[:a] for _ in range(B)]).int()
        if kind == "odd":                             # left out, and named twice
            pos[0, 0], pos[0, 1], pos[0, 2] = -1, cap, 2 ** 31 - 1
            pos[B - 1, 3] = pos[B - 1, a - 1]
            pos[B - 1, 5] = pos[B - 1, 6] = pos[B - 1, a // 2]
        places = pos.tolist()
    dllm.kv4_store(cache, k, v, pos=pos, start=start)
    for which, x in ((0, k), (2, v)):
        codes, params = expected_store(before[which], before[which + 1], x, places, B, Hkv, hd)
        assert torch.equal(cache.tensors()[which], codes)
        assert torch.equal(cache.tensors()[which + 1], params)
    lens = lens_of([cap // 2 + 7 * b for b in range(B)])
    for n, ln, out in ((cap, None, torch.float32), (cap - 3, lens, torch.float32), (1, None, torch.bfloat16), (cap - 1, lens, torch.bfloat16)):
        got = dllm.kv4_load(cache, n, lens=ln, dtype=out)
        for which in (0, 1):
            codes, par = cache.tensors()[2 * which], cache.tensors()[2 * which + 1].double()
            want = (ref.unpack4(codes) * par[..., :1] + par[..., 1:]).float().to(out)[:, :, :n].transpose(1, 2).reshape(B, n, W).clone()
            for b in range(B if ln is not None else 0):
                want[b, int(ln[b]):] = 0
            assert torch.equal(got[which], want)


def test_a_stored_row_is_near_what_it_was(dllm):
    """Half a step, and the roundings of step and lo to bf16 (2^-8 of 15 steps and of lo)."""
    x = torch.randn((1, 50, 256), generator=gen(3), device="cuda").bfloat16()
    cache = dllm.KV4Cache(1, 2, 50, 128)
    dllm.kv4_store(cache, x, x)
    k, v = dllm.kv4_load(cache, 50)
    assert torch.equal(k, v)
    spread = x.float().reshape(50, 2, 128)
    step = (spread.amax(-1) - spread.amin(-1)) / 15
    bound = (0.5 + 15 * 2.0 ** -8) * step + 2.0 ** -8 * spread.amin(-1).abs() + 1e-6
    assert bool(((k - x.float()).reshape(50, 2, 128).abs() <= bound[..., None]).all())


def test_rows_without_a_spread_and_without_numbers(dllm):
    x = torch.randn((1, 6, 128), generator=gen(4), device="cuda")
    x[0, 0], x[0, 1] = 0.0, 1.3
    x[0, 2, 5], x[0, 3, 70], x[0, 4, 1] = math.nan, math.inf, -math.inf
    x[0, 5, :64], x[0, 5, 64:] = 3e38, -3e38
    cache = dllm.KV4Cache(1, 2, 6, 64)
    dllm.kv4_store(cache, x, x)
    k, _ = dllm.kv4_load(cache, 6)
    h = k.reshape(6, 2, 64)
    assert not h[0].any() and torch.equal(h[1], torch.full_like(h[1], 1.3).bfloat16().float())
    assert h[2, 0].isnan().all() and h[2, 1].isfinite().all() and h[3, 1].isnan().all() and h[3, 0].isfinite().all()
    assert h[4, 0].isnan().all() and h[5].isfinite().all()      # each head's half of row 5 has one value
    wide = torch.cat([x[:, 5:, :64], x[:, 5:, 64:]], 1).transpose(1, 2).reshape(1, 1, 128).contiguous()   # alternating +-3e38
    dllm.kv4_store(cache, wide, wide)
    k, _ = dllm.kv4_load(cache, 1)
    assert k.isnan().all()


# ---------------------------------------------------------------- attention
@pytest.fixture(params=[(0, 0), (1, 1), (1, 4), (1, 11), (2, 1), (2, 3)], ids=lambda p: f"kernel{p[0]}-ranges{p[1]}")
def plan(request, dllm):
    """The plan's own choice, and both kernels with one range of keys, merged in a cluster and by a launch."""
    dllm.debug_kv4_plan(*request.param)
    yield request.param
    dllm.debug_kv4_plan()


SHAPES = [  # B, a, n, H, Hkv, hd, lens
    (1, 1, 1, 1, 1, 64, None),
    (1, 1, 1, 7, 1, 128, None),
    (1, 3, 65, 4, 4, 128, None),
    (2, 1, 64, 8, 8, 64, [64, 0]),
    (3, 2, 200, 14, 2, 128, [200, 1, 129]),
    (1, 64, 768, 4, 4, 128, None),
    (4, 5, 1000, 8, 2, 64, [1000, 999, 63, -5]),
    (1, 17, 4128, 2, 2, 128, None),
    (2, 9, 3000, 28, 4, 128, [2999, 5000]),
    (1, 130, 513, 6, 3, 64, None),
    (1, 200, 300, 7, 1, 128, [257]),
    (2, 300, 450, 4, 2, 128, [450, 33]),
    (1, 2, 20000, 8, 1, 128, None),
    (2, 5, 700, 71, 1, 64, [700, 300]),
    (1, 2, 300, 260, 1, 128, None),
    (40, 80, 520, 2, 2, 64, [13 * b for b in range(40)]),
]


def queries(g, B, a, H, hd, scale=1.0):
    return (scale * torch.randn((B * a, H * hd), generator=g, device="cuda")).bfloat16()


def check_attention(q, cache, a, n, H, lens, o, lse):
    want, wl, oe, se = ref.attention(q, cache, a, n, H, lens)
    B, hd = cache.B, cache.hd
    o, lse = o.double().reshape(B, a, H, hd), lse.double().reshape(B, a, H)
    empty = torch.isneginf(wl)
    assert torch.equal(torch.isneginf(lse), empty)
    assert not o[empty].any()
    assert bool(((lse - wl).abs()[~empty] <= se[~empty] + 2.0 ** -23 * wl[~empty].abs()).all())
    bound = oe + 2.0 ** -8 * want.abs() * 1.01 + 1e-30
    assert bool(((o - want).abs() <= bound).all()), float(((o - want).abs() / bound).max())


@pytest.mark.parametrize("B,a,n,H,Hkv,hd,lens", SHAPES)
def test_attention(dllm, plan, B, a, n, H, Hkv, hd, lens):
    g = gen(n + a)
    cache = ref.random_cache(dllm, g, B, Hkv, -(-n // 64) * 64, hd)
    q, lens = queries(g, B, a, H, hd), lens_of(lens)
    o, lse = dllm.attention_kv4(q, cache, a, n, H, lens=lens)
    check_attention(q, cache, a, n, H, lens, o, lse)
    again, lse2 = dllm.attention_kv4(q, cache, a, n, H, lens=lens)
    assert torch.equal(o, again) and torch.equal(lse, lse2)
    dllm.kernel_status()


@pytest.mark.parametrize("a,H,Hkv,n", [(2, 8, 2, 150), (90, 8, 2, 700)])
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_ignores_what_lies_behind_a_length(dllm, plan, hd, a, H, Hkv, n):
    """NaN, infinities and the largest numbers behind every length, inside of a tile and behind n; rows of Q inside of wider rows."""
    g = gen(5)
    cap = -(-n // 64) * 64
    cache = ref.random_cache(dllm, g, 2, Hkv, cap, hd)
    rows = queries(g, 2, a, 3 * H, hd)
    q = rows[:, H * hd:2 * H * hd]
    lens = lens_of([n - 50, n - 9])
    o, lse = dllm.attention_kv4(q, cache, a, n, H, lens=lens)
    check_attention(q, cache, a, n, H, lens, o, lse)
    w = torch.zeros((2, Hkv, cap), device="cuda")
    dllm.attention_weights_kv4(q, cache, lse, w, a, n, H, lens=lens)
    for bad in (math.nan, math.inf, -math.inf, 3.3e38):
        for b in range(2):
            for t in (cache.k_params, cache.v_params):
                t[b, :, int(lens[b]):] = bad
            for t in (cache.k_codes, cache.v_codes):
                t[b, :, int(lens[b]):] = 255
        o2, lse2 = dllm.attention_kv4(q, cache, a, n, H, lens=lens)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        w2 = torch.zeros((2, Hkv, cap), device="cuda")
        dllm.attention_weights_kv4(q, cache, lse, w2, a, n, H, lens=lens)
        assert torch.equal(w, w2)


@pytest.mark.parametrize("a", [3, 80])
def test_attention_of_a_row_with_a_nan(dllm, plan, a):
    """A NaN among the keys or values of one head shows in that head's rows and in no other's; so does one in a query."""
    g = gen(6)
    cache = ref.random_cache(dllm, g, 1, 2, 192, 128)
    q = queries(g, 1, a, 4, 128)
    clean, clean_lse = dllm.attention_kv4(q, cache, a, 190, 4)
    for t in (cache.k_params, cache.v_params):
        keep = t.clone()
        t[0, 1, 77] = math.nan
        o, _ = dllm.attention_kv4(q, cache, a, 190, 4)
        assert o.reshape(a, 4, 128)[:, 2:].isnan().all()
        assert torch.equal(o.reshape(a, 4, 128)[:, :2], clean.reshape(a, 4, 128)[:, :2])
        t.copy_(keep)
    q2 = q.clone()
    q2[1, 5] = math.nan
    o, lse = dllm.attention_kv4(q2, cache, a, 190, 4)
    assert o[1, :128].isnan().all() and lse[1, 0].isnan()
    o[1, :128], lse[1, 0] = clean[1, :128], clean_lse[1, 0]
    assert torch.equal(o, clean) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("a,qs,cs", [(4, 40.0, 1.0), (100, 40.0, 1.0), (4, 1e-30, 1.0), (4, 1e30, 1e-30), (100, 1e30, 1e-30), (4, 1.0, 1e-20),
                                     (100, 1.0, 1e-20), (4, 1e-4, 1e4), (100, 1e-4, 1e4)])
def test_attention_of_very_large_and_very_small_numbers(dllm, plan, a, qs, cs):
    """One key ahead of all others, scores of zero, numbers near the ends of bf16's range."""
    g = gen(7)
    cache = ref.random_cache(dllm, g, 1, 2, 320, 128, scale=cs)
    q = queries(g, 1, a, 2, 128, scale=qs)
    o, lse = dllm.attention_kv4(q, cache, a, 311, 2)
    check_attention(q, cache, a, 311, 2, None, o, lse)


@pytest.mark.parametrize("a", [4, 100])
@pytest.mark.parametrize("hd", [64, 128])
def test_huge_keys_under_tiny_queries(dllm, plan, a, hd):
    """Steps of 4 * 10^33 times a product of codes and scaled queries, some 2^18, leave fp32's range; the scores (some tens) do not."""
    g = gen(19)
    cache, ordinary = ref.random_cache(dllm, g, 1, 2, 320, hd, scale=2e34), ref.random_cache(dllm, g, 1, 2, 320, hd)
    cache.v_params.copy_(ordinary.v_params)
    q = queries(g, 1, a, 2, hd, scale=2e-33)
    o, lse = dllm.attention_kv4(q, cache, a, 311, 2)
    check_attention(q, cache, a, 311, 2, None, o, lse)
    w = torch.zeros((1, 2, 320), device="cuda")
    dllm.attention_weights_kv4(q, cache, lse, w, a, 311, 2)
    want, err = ref.weights(q, cache, lse, a, 311, 2)
    # an exponential below fp32's smallest normal number is 0: at most that much per row
    assert bool(((w.double() - want).abs() <= err + 2.0 ** -23 * want + a * 2.0 ** -126).all())


@pytest.mark.parametrize("a", [4, 100])
@pytest.mark.parametrize("hd", [64, 128])
def test_values_near_the_largest_number(dllm, plan, a, hd):
    """Values of some 10^37 under hundreds of keys of like weight: their sums leave fp32's range, their mean does not."""
    g = gen(20)
    cache, huge = ref.random_cache(dllm, g, 1, 2, 1280, hd), ref.random_cache(dllm, g, 1, 2, 1280, hd, scale=2e37)
    huge.v_params[..., 1] = -2.5 * huge.v_params[..., 0]          # 0 .. 15 steps of up to 7e36 from -2.5 of them on
    cache.v_params.copy_(huge.v_params)
    assert bool(torch.isfinite(cache.v_params[..., 1].float() + 15 * cache.v_params[..., 0].float()).all())
    q = queries(g, 1, a, 2, hd, scale=0.1)
    o, lse = dllm.attention_kv4(q, cache, a, 1271, 2)
    assert float(ref.attention(q, cache, a, 1271, 2)[0].abs().max()) > 1e37
    check_attention(q, cache, a, 1271, 2, None, o, lse)


@pytest.mark.parametrize("a", [4, 100])
@pytest.mark.parametrize("big", [2.0 ** 10, 2.0 ** 16])
def test_keys_of_very_different_size(dllm, plan, a, big):
    """A few keys `big` times the others, whose scores under queries with a mean are so low that they count for nothing.  The
    others' numbers are off by up to 2^-31 of the largest number M in the tcgen05 kernel, so a score by 2^-31 M sum|q| / sqrt(hd)."""
    g = gen(22)
    hd, n = 128, 640
    cache = ref.random_cache(dllm, g, 1, 2, n, hd)
    cache.k_params[:, :, 100:600:100, 1] = -big       # their offsets; their steps stay as they are
    q = (1 + torch.randn((a, 4 * hd), generator=g, device="cuda")).bfloat16()
    assert bool((q.double().reshape(a, 4, hd).sum(-1) > 30).all())
    o, lse = dllm.attention_kv4(q, cache, a, n, 4)
    want, wl, oe, se = ref.attention(q, cache, a, n, 4)
    small = cache.k_params.clone()
    small[:, :, 100:600:100] = 0
    _, _, oe, se = ref.attention(q, dllm.KV4Cache.from_tensors(cache.k_codes, small, cache.v_codes, cache.v_params), a, n, 4)   # bounds of the others
    ds = 2.0 ** -31 * big * q.double().reshape(1, a, 4, hd).abs().sum(-1) / math.sqrt(hd)
    size = float((16 * cache.v_params[..., 0].abs() + cache.v_params[..., 1].abs()).double().max())
    assert bool(((lse.double().reshape(wl.shape) - wl).abs() <= se + ds + 2.0 ** -22 * (1 + wl.abs())).all())
    assert bool(((o.double().reshape(want.shape) - want).abs() <= oe + 2 * ds[..., None] * size + 2.0 ** -8 * 1.01 * want.abs()).all())


def offset_cache(dllm, g, B, Hkv, cap, hd):
    """Keys and values whose offsets are some sixty steps: what a score then is made of is the offset times the query's sum."""
    cache = ref.random_cache(dllm, g, B, Hkv, cap, hd)
    for t in (cache.k_params, cache.v_params):
        t[..., 1] += 12 * torch.randn((B, Hkv, cap), generator=g, device="cuda").bfloat16()
    return cache


def offset_queries(g, B, a, H, hd):
    """Rows whose mean is as large as their spread, so small that the scores (some 1.06 * 12 * 0.015 * sqrt(hd) = 2) leave the softmax
    spread."""
    return (0.015 * (1 + torch.randn((B * a, H * hd), generator=g, device="cuda"))).bfloat16()


@pytest.mark.parametrize("B,a,n,H,Hkv,hd,lens", [(1, 1, 65, 1, 1, 128, None), (2, 9, 700, 14, 2, 128, [700, 333]), (1, 64, 768, 4, 4, 64, None),
                                                 (2, 150, 450, 4, 2, 128, [450, 33]), (1, 300, 1300, 2, 1, 64, None)])
def test_scores_made_of_offsets(dllm, plan, B, a, n, H, Hkv, hd, lens):
    """Sums and offsets reach both tensor-core kernels in parts: two parts of three would be off by 2^-17 of a score, and the
    bounds allow some 2^-19 of it."""
    g = gen(17 + n)
    cache = offset_cache(dllm, g, B, Hkv, -(-n // 64) * 64, hd)
    q, lens = offset_queries(g, B, a, H, hd), lens_of(lens)
    o, lse = dllm.attention_kv4(q, cache, a, n, H, lens=lens)
    check_attention(q, cache, a, n, H, lens, o, lse)
    w = torch.zeros((B, Hkv, cache.capacity), device="cuda")
    dllm.attention_weights_kv4(q, cache, lse, w, a, n, H, lens=lens)
    want, err = ref.weights(q, cache, lse, a, n, H, lens)
    bound = err + 2.0 ** -23 * want
    assert bool(((w.double() - want).abs() <= bound).all()), float(((w.double() - want).abs() / bound.clamp_min(1e-300)).max())
    dllm.kernel_status()


@pytest.mark.parametrize("a", [4, 100])
def test_attention_over_values_of_very_different_steps(dllm, plan, a):
    g = gen(8)
    cache = ref.random_cache(dllm, g, 1, 1, 640, 128)
    cache.v_params.mul_(2.0 ** torch.randint(-12, 13, (1, 1, 640, 1), generator=g, device="cuda").float())
    cache.v_params[0, 0, 10:20, 0] = 0          # no spread at all
    cache.k_params[0, 0, 30:40] = 0
    q = queries(g, 1, a, 1, 128)
    o, lse = dllm.attention_kv4(q, cache, a, 640, 1)
    # a weight p * step enters as fp16 at a scale where the largest step is 2^10 or more: below fp16's normal numbers it is off
    # by up to half of 2^-24, i.e. 2^-35 of twice the largest step, times the code's distance from 8, at most 8, for each key
    want, wl, oe, se = ref.attention(q, cache, a, 640, 1)
    floor = 640 * 2.0 ** -34 * 8 * float(cache.v_params[..., 0].abs().max())
    assert bool(((o.double().reshape(want.shape) - want).abs() <= oe + 2.0 ** -8 * 1.01 * want.abs() + floor).all())
    assert bool(((lse.double().reshape(wl.shape) - wl).abs() <= se + 2.0 ** -23 * wl.abs()).all())


@pytest.mark.parametrize("a", [3, 90])
@pytest.mark.parametrize("kscale", [0.0, 1e-12, 1.0])
@pytest.mark.parametrize("qscale", [0.0, 1e-38])
def test_attention_of_queries_of_zeros(dllm, plan, a, kscale, qscale):
    """Rows of zeros (a padded batch) over keys that were never stored, tiny ones and ordinary ones: every key counts alike, and
    those behind the length for nothing."""
    g = gen(12)
    cache = ref.random_cache(dllm, g, 1, 2, 192, 128, scale=kscale if kscale else 1.0)
    if kscale == 0.0:
        cache.k_params.zero_()
    v = torch.randn((1, 192, 256), generator=g, device="cuda").bfloat16()
    keep = [t.clone() for t in (cache.k_codes, cache.k_params)]
    dllm.kv4_store(cache, v, v)
    cache.k_codes.copy_(keep[0])
    cache.k_params.copy_(keep[1])
    q = queries(g, 1, a, 4, 128, scale=qscale)
    o, lse = dllm.attention_kv4(q, cache, a, 133, 4)
    check_attention(q, cache, a, 133, 4, None, o, lse)
    w = torch.zeros((1, 2, 192), device="cuda")
    dllm.attention_weights_kv4(q, cache, lse, w, a, 133, 4)
    want, err = ref.weights(q, cache, lse, a, 133, 4)
    assert bool(((w.double() - want).abs() <= err + 2.0 ** -23 * want).all())


@pytest.mark.parametrize("B,a,n,H,Hkv", [(700, 1, 640, 2, 1), (100, 70, 300, 1, 1)])
def test_many_sequences(dllm, plan, B, a, n, H, Hkv):
    """More sequences than a warp has lanes, the first ones without keys; ranges of keys times sequences within a grid's limit."""
    g = gen(14)
    cache = ref.random_cache(dllm, g, B, Hkv, -(-n // 64) * 64, 64)
    q, lens = queries(g, B, a, H, 64), lens_of([0] * 64 + [(37 * b) % (n + 1) for b in range(64, B)])
    o, lse = dllm.attention_kv4(q, cache, a, n, H, lens=lens)
    check_attention(q, cache, a, n, H, lens, o, lse)
    w = torch.zeros((B, Hkv, cache.capacity), device="cuda")
    dllm.attention_weights_kv4(q, cache, lse, w, a, n, H, lens=lens)
    want, err = ref.weights(q, cache, lse, a, n, H, lens)
    assert bool(((w.double() - want).abs() <= err + 2.0 ** -23 * want).all())


def test_calls_on_two_streams_at_once(dllm):
    """The same products, attention and weights on two streams, each with buffers of its own, twenty times over."""
    g = gen(13)
    cache = ref.random_cache(dllm, g, 1, 2, 20480, 128)
    q = [queries(g, 1, a, 4, 128) for a in (4, 100)]
    x, (W, sw) = queries(g, 1, 3, 8, 128), dllm.quantize_rows_s8(queries(g, 1, 512, 8, 128))

    def work(i):
        o, lse = dllm.attention_kv4(q[i], cache, q[i].shape[0], 20001, 4)
        w = torch.zeros((1, 2, 20480), device="cuda")
        dllm.attention_weights_kv4(q[i], cache, lse, w, q[i].shape[0], 20001, 4)
        return o, lse, w, dllm.linear_s8(x, W, sw), *dllm.kv4_evict(cache, w, 20001, 9000)[1:]

    want = [work(i) for i in (0, 1)]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in (0, 1)]
    got = []
    for _ in range(20):
        for i in (0, 1):
            with torch.cuda.stream(sides[i]):
                got.append((i, work(i)))
    torch.cuda.synchronize()
    for i, ts in got:
        for t, u in zip(ts, want[i]):
            assert torch.equal(t, u)
    dllm.kernel_status()


def test_attention_past_four_gigabytes(dllm, plan):
    """The last plane of a cache whose codes take 4.3 GB a tensor."""
    if plan[1] == 1 or plan == (1, 4):
        pytest.skip("eight million keys in few ranges: enough in the others")
    B, Hkv, cap, hd = 1, 8, 64 * 131200, 128
    cache = dllm.KV4Cache(B, Hkv, cap, hd)
    assert cache.k_codes.numel() > 2 ** 32
    g = gen(9)
    small = ref.random_cache(dllm, g, 1, 1, 128, hd)
    n0 = cap - 128
    k, v = dllm.kv4_load(small, 128, dtype=torch.bfloat16)
    dllm.kv4_store(cache, k.repeat(1, 1, Hkv), v.repeat(1, 1, Hkv), start=n0)
    got_k, _ = dllm.kv4_load(dllm.KV4Cache.from_tensors(*(t[:, :, n0:].contiguous() for t in cache.tensors())), 128)
    again = dllm.KV4Cache(1, 1, 128, hd)
    dllm.kv4_store(again, k, v)
    want_k, _ = dllm.kv4_load(again, 128)
    assert torch.equal(got_k.reshape(128, Hkv, hd)[:, -1], want_k.reshape(128, hd))
    # the other keys get scores of -10^4 or less, so the last ones alone count
    cache.k_params[:, :, :n0, 1] = -1e4
    q = torch.ones((1, Hkv * hd), device="cuda").bfloat16()
    o, lse = dllm.attention_kv4(q, cache, 1, cap, Hkv)
    want, wl, oe, se = ref.attention(torch.ones((1, hd), device="cuda").bfloat16(), again, 1, 128, 1)
    assert bool(((o.double().reshape(Hkv, hd) - want.reshape(1, hd)).abs() <= oe.reshape(1, hd) + 2.0 ** -8 * 1.01 * want.abs().reshape(1, hd)).all())
    assert bool(((lse.double().reshape(-1) - wl.reshape(1)).abs() <= se.reshape(1) + 2.0 ** -22 * wl.abs().reshape(1)).all())
    w = torch.zeros((B, Hkv, cap), device="cuda")
    dllm.attention_weights_kv4(q, cache, lse, w, 1, cap, Hkv)
    assert bool((w.double().sum(-1) - 1).abs().max() < 1e-4) and not w[:, :, :n0].any()


@pytest.mark.parametrize("n", [2048, 20480])
def test_attention_on_another_stream_and_in_a_graph(dllm, n):
    g = gen(10)
    cache = ref.random_cache(dllm, g, 1, 2, n, 128)
    q = queries(g, 1, 4, 4, 128)
    lens = lens_of([n - 48])
    scratch = torch.empty(dllm.lib.dllm_attention_kv4_scratch_bytes(1, 4, n, 4, 2, 128), dtype=torch.uint8, device="cuda")
    assert (scratch.numel() > 0) == (n > 2048)      # a few ranges of keys need none, many do
    want = dllm.attention_kv4(q, cache, 4, n, 4, lens=lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = dllm.attention_kv4(q, cache, 4, n, 4, lens=lens, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = dllm.attention_kv4(q, cache, 4, n, 4, lens=lens, scratch=scratch)
    q.copy_(queries(g, 1, 4, 4, 128))
    lens.fill_(777)
    graph.replay()
    torch.cuda.synchronize()
    check_attention(q, cache, 4, n, 4, lens, o, lse)


def test_all_calls_in_one_graph(dllm):
    """Rows stored, attended to, scored, evicted and read back, few and many of them, and products, captured once and replayed on
    other rows and lengths: what the calls give one by one."""
    g = gen(15)
    B, n, H, Hkv, hd = 2, 8192, 8, 4, 128
    cache, again = dllm.KV4Cache(B, Hkv, n, hd), dllm.KV4Cache(B, Hkv, n, hd)
    k = torch.randn((B, n, Hkv * hd), generator=g, device="cuda").bfloat16()
    qs = [queries(g, B, a, H, hd) for a in (4, 200)]
    xs = [queries(g, 1, rows, 16, hd) for rows in (3, 700)]
    W, sw = dllm.quantize_rows_s8(queries(g, 1, 1024, 16, hd))
    w, lens = torch.zeros((B, Hkv, n), device="cuda"), lens_of([8000, 5000])

    def work(cache):
        out = []
        dllm.kv4_store(cache, k, k)
        w.zero_()
        for q in qs:
            a = q.shape[0] // B
            o, lse = dllm.attention_kv4(q, cache, a, n, H, lens=lens)
            dllm.attention_weights_kv4(q, cache, lse, w, a, n, H, lens=lens)
            out += [o, lse]
        small, *rest = dllm.kv4_evict(cache, w, n, 1000, 4, 32, lens=lens)
        return [*out, *rest, *dllm.kv4_load(small, 1000, lens=rest[2]), *(dllm.linear_s8(x, W, sw) for x in xs)]

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work(cache)
    for t in (k, *qs, *xs):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    lens.copy_(lens_of([900, 8192]))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    kept = [t.clone() for t in got]
    for x, y in zip(kept, work(again)):
        assert torch.equal(x, y)
    dllm.kernel_status()


# ---------------------------------------------------------------- weights
@pytest.mark.parametrize("B,a,n,H,Hkv,hd,lens", SHAPES)
def test_weights(dllm, plan, B, a, n, H, Hkv, hd, lens):
    g = gen(n + 2 * a)
    cap = -(-n // 64) * 64
    cache = ref.random_cache(dllm, g, B, Hkv, cap, hd)
    q, lens = queries(g, B, a, H, hd), lens_of(lens)
    _, lse = dllm.attention_kv4(q, cache, a, n, H, lens=lens)
    if a > 2:
        lse[1, 0] = -math.inf                     # a row that saw nothing
    had = torch.rand((B, Hkv, cap), generator=g, device="cuda")
    w = had.clone()
    dllm.attention_weights_kv4(q, cache, lse, w, a, n, H, lens=lens)
    got, err = ref.weights(q, cache, lse, a, n, H, lens)
    want = had.double() + got
    bound = err + 2.0 ** -23 * want
    assert bool(((w.double() - want).abs() <= bound).all()), float(((w.double() - want).abs() / bound).max())
    for b in range(B):
        L = n if lens is None else min(max(int(lens[b]), 0), n)
        assert torch.equal(w[b, :, L:], had[b, :, L:])
    again = had.clone()
    dllm.attention_weights_kv4(q, cache, lse, again, a, n, H, lens=lens)
    assert torch.equal(w, again)


@pytest.mark.parametrize("B,a,n,H,Hkv,hd,lens", [(1, 3, 65, 4, 4, 128, None), (2, 9, 700, 14, 2, 128, [700, 333]), (1, 60, 513, 2, 2, 64, None),
                                                 (2, 150, 450, 4, 2, 128, [450, 33]), (1, 300, 40000, 1, 1, 64, None)])
def test_rows_that_saw_no_key_give_nothing_whatever_they_hold(dllm, plan, B, a, n, H, Hkv, hd, lens):
    """Rows of a padded batch, left out by an lse of -infinity, hold NaN, infinities or the largest numbers."""
    g = gen(21 + n)
    cap = -(-n // 64) * 64
    cache = ref.random_cache(dllm, g, B, Hkv, cap, hd)
    q, lens = queries(g, B, a, H, hd), lens_of(lens)
    _, lse = dllm.attention_kv4(q, cache, a, n, H, lens=lens)
    out = torch.rand((B * a, H), generator=g, device="cuda") < 0.3
    out[0], out[-1] = True, False
    if Hkv > 1:
        out[:, :H // Hkv] = True                      # all rows of the first KV head
    lse[out] = -math.inf
    zeros = q.reshape(B * a, H, hd).clone()
    zeros[out] = 0
    had = torch.rand((B, Hkv, cap), generator=g, device="cuda")
    got, err = ref.weights(zeros.reshape(B * a, H * hd), cache, lse, a, n, H, lens)
    want = had.double() + got
    for bad in (math.nan, math.inf, -math.inf, 3.3e38, -3.3e38):
        rows = zeros.clone()
        rows[out] = bad
        w = had.clone()
        dllm.attention_weights_kv4(rows.reshape(B * a, H * hd), cache, lse, w, a, n, H, lens=lens)
        assert bool(((w.double() - want).abs() <= err + 2.0 ** -23 * want).all())
        assert Hkv == 1 or torch.equal(w[:, 0], had[:, 0])
    dllm.kernel_status()


def test_exponentials_of_the_weights_alone(dllm):
    """One row per sequence that counts, a query of zeros, over one key: the key gets exp(-lse), by the special-function unit or,
    in rows 6 and 7 of eight, by a polynomial.  x = -lse log2(e), |x| <= 0.73, is off by at most 2^-21.3 of itself (the constant,
    the product, 1 / c and c 2^-25 + 3 * 2^-24, parts left out 2^-26, the matrix instruction's sum 2^-22), so 2e-7 of the result;
    the exponentials by 2^-22.5 each (1.7e-7).  What is rounded either way leaves the mean of 2048 results of a class of rows, with lse
    as often positive as negative, where the polynomial's own mean puts it: 1.7e-8 off."""
    g = gen(16)
    B, a, hd = 8192, 128, 64
    cache = dllm.KV4Cache(B, 1, 64, hd)
    cache.k_params[..., 0] = (1 + torch.rand((B, 1, 64), generator=g, device="cuda")).bfloat16()
    half = (torch.rand(B // 2, generator=g, device="cuda") - 0.5)[:, None]
    live = torch.cat([half, -half], 1).flatten()               # each value beside its negative
    row = (torch.arange(B, device="cuda") // 2) % a
    lse = torch.full((B, a), -math.inf, device="cuda")
    lse[torch.arange(B, device="cuda"), row] = live
    w = torch.zeros((B, 1, 64), device="cuda")
    dllm.attention_weights_kv4(torch.zeros((B * a, hd), device="cuda").bfloat16(), cache, lse.reshape(B * a, 1), w, a, 1, 1)
    assert not w[:, 0, 1:].any()
    off = w[:, 0, 0].double() / torch.exp(-live.double()) - 1
    assert float(off.abs().max()) < 4e-7
    poly = off[row % 8 >= 6]
    assert poly.numel() == B // 4 and abs(float(poly.mean())) < 4e-8, float(poly.mean())
    dllm.kernel_status()


# ---------------------------------------------------------------- eviction
@pytest.mark.parametrize("B,n,keep,first,last,Hkv,hd,lens,ties", [
    (1, 1, 1, 0, 0, 1, 64, None, False), (1, 100, 1, 0, 0, 2, 128, None, False), (1, 100, 40, 0, 0, 2, 128, None, True),
    (2, 700, 300, 4, 32, 3, 64, [700, 299], True), (3, 5000, 777, 0, 777, 2, 128, [5000, 0, 778], False),
    (1, 5000, 2500, 2500, 0, 1, 64, None, False), (2, 20000, 9999, 5, 5, 1, 64, [20000, 19999], True), (1, 130, 192, 3, 3, 2, 128, None, False),
    (1, 9000, 8999, 1, 1, 1, 64, [9001], False)])
def test_evict(dllm, B, n, keep, first, last, Hkv, hd, lens, ties):
    g = gen(n + keep)
    cap = -(-n // 64) * 64
    cache = ref.random_cache(dllm, g, B, Hkv, cap, hd)
    w = torch.rand((B, Hkv, cap), generator=g, device="cuda").pow(6)
    if ties:
        w = (w * 20).floor() / 4 - 0.5
        w[0, 0, n // 3] = math.nan
        w[0, 0, n // 2] = math.inf
        w[0, 0, n // 2 + 1] = -math.inf
        w[0, 0, 5:30:2] = -0.0
        w[0, 0, 6:30:2] = 0.0
    lens = lens_of(lens)
    was = [t.clone() for t in (*cache.tensors(), w)]
    to = dllm.KV4Cache(B, Hkv, keep + 64, hd)
    for t in to.tensors():
        t.fill_(3)
    to, nw, index, new = dllm.kv4_evict(cache, w, n, keep, first, last, lens=lens, to=to)
    want, want_lens = ref.evict(w, n, keep, first, last, lens)
    assert torch.equal(index.cpu(), want) and torch.equal(new.cpu(), want_lens)
    for x, y in zip((*cache.tensors(), w), was):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))       # the source stays as it is
    for b in range(B):
        L = int(want_lens[b])
        for h in range(Hkv):
            rows = index[b, h, :L].long()
            for src, dst in zip(cache.tensors(), to.tensors()):
                assert torch.equal(dst[b, h, :L], src[b, h, rows])
                assert bool((dst[b, h, L:] == 3).all())                    # rows behind the last one as they were
            assert torch.equal(nw[b, h, :L].nan_to_num(-9), w[b, h, rows].nan_to_num(-9)) and not nw[b, h, L:].any()


@pytest.mark.parametrize("Hkv,n,lens", [(300, 41000, None), (300, 300, [41]), (2, 20000, [0]), (2, 20000, [2501]), (2, 330000, None)])
def test_evict_of_many_heads_and_many_keys(dllm, Hkv, n, lens):
    """Distinct weights: the kept keys are the largest ones, sorted.  Heads enough for a CTA each, keys beyond what shared memory
    holds, and lengths that leave most CTAs of a cluster without a key."""
    g = gen(n + Hkv)
    cap, keep = -(-n // 64) * 64, min(n // 8, 5000)
    cache = ref.random_cache(dllm, g, 1, Hkv, cap, 64)
    w = torch.rand((1, Hkv, cap), generator=g, device="cuda").argsort(-1).float()
    L = n if lens is None else lens[0]
    _, nw, index, new = dllm.kv4_evict(cache, w, n, keep, lens=lens_of(lens))
    kept = min(L, keep)
    rows = w[..., :L].topk(kept).indices.sort(-1).values
    assert new.tolist() == [kept] and torch.equal(index[..., :kept].long(), rows) and bool((index[..., kept:] == -1).all())
    assert torch.equal(nw[..., :kept], w.gather(-1, rows)) and not nw[..., kept:].any()


@pytest.mark.parametrize("n,keep,first,last", [(300, 300, 0, 0), (300, 120, 40, 40), (9000, 9000, 3, 3), (9000, 5000, 1500, 1500), (41000, 600, 200, 200)])
def test_evicted_weights_of_minus_zero_are_zero(dllm, n, keep, first, last):
    """To the bit, whichever way a key stays: by its place, by its weight, or because all do."""
    g = gen(n + keep)
    cap = -(-n // 64) * 64
    cache = ref.random_cache(dllm, g, 1, 2, cap, 64)
    w = torch.randint(0, 3, (1, 2, cap), generator=g, device="cuda").float()
    w[(torch.rand(w.shape, generator=g, device="cuda") < 0.5) & (w == 0)] = -0.0
    _, nw, index, _ = dllm.kv4_evict(cache, w, n, keep, first, last)
    want = w.gather(-1, index.long())
    assert bool((want.view(torch.int32) == -2 ** 31).any())          # some of those that stayed were -0
    assert torch.equal(nw[..., :keep].view(torch.int32), (want + 0.0).view(torch.int32))


@pytest.mark.parametrize("Hkv,n", [(75, 8256), (74, 8256), (160, 40960), (160, 41024), (700, 8300)])
def test_evict_on_both_sides_of_the_choice_of_clusters(dllm, Hkv, n):
    """One CTA per head and a cluster of eight give the same: weights of few values, so that places go by index."""
    g = gen(n + Hkv)
    cap, keep = -(-n // 64) * 64, 1000
    cache = dllm.KV4Cache(1, Hkv, cap, 64)
    w = torch.randint(0, 40, (1, Hkv, cap), generator=g, device="cuda").float()
    _, nw, index, new = dllm.kv4_evict(cache, w, n, keep, 3, 5)
    order = w[..., :n].clone()
    order[..., :3] = order[..., n - 5:] = 1e9
    rows = order.sort(dim=-1, descending=True, stable=True).indices[..., :keep].sort(-1).values
    assert new.tolist() == [keep] and torch.equal(index.long(), rows)
    assert torch.equal(nw[..., :keep], w.gather(-1, rows))


# ---------------------------------------------------------------- as they are used together
def test_a_prompt_is_cached_scored_and_thinned_out(dllm):
    """Prompt and response rows go into the cache, the response's queries attend and score, half of the prompt leaves, and
    attention over what stayed equals attention over those rows of the old cache."""
    g = gen(11)
    B, P, R, H, Hkv, hd = 2, 500, 24, 8, 2, 128
    n = P + R
    cache = dllm.KV4Cache(B, Hkv, n, hd)
    qkv = torch.randn((B, n, (H + 2 * Hkv) * hd), generator=g, device="cuda").bfloat16()
    k, v = qkv[..., H * hd:(H + Hkv) * hd], qkv[..., (H + Hkv) * hd:]
    dllm.kv4_store(cache, k[:, :P].contiguous(), v[:, :P].contiguous())
    dllm.kv4_store(cache, k[:, P:].contiguous(), v[:, P:].contiguous(), start=P)
    q = qkv[:, P:, :H * hd].contiguous().reshape(B * R, H * hd)
    o, lse = dllm.attention_kv4(q, cache, R, n, H)
    check_attention(q, cache, R, n, H, None, o, lse)
    weight = torch.zeros((B, Hkv, cache.capacity), device="cuda")
    dllm.attention_weights_kv4(q, cache, lse, weight, R, n, H)
    assert float((weight.sum(-1) - R * (H // Hkv)).abs().max()) < 1e-2      # every row gives one in all
    keep = P // 2 + R
    small, w2, index, lens = dllm.kv4_evict(cache, weight, n, keep, first=4, last=R)
    assert bool((index[:, :, -R:] == torch.arange(P, n, device="cuda")).all()) and lens.tolist() == [keep] * B
    o2, lse2 = dllm.attention_kv4(q, small, R, keep, H, lens=lens)
    rows = index.long()[..., None]
    pick = dllm.KV4Cache(B, Hkv, keep, hd)
    for src, dst in zip(cache.tensors(), pick.tensors()):
        dst[:, :, :keep] = src.gather(2, rows.expand(-1, -1, -1, src.shape[-1]))
    check_attention(q, pick, R, keep, H, None, o2, lse2)
    # the response goes on: its new rows replace the old ones at their new places
    pos = torch.arange(keep - R, keep, device="cuda", dtype=torch.int32).expand(B, R).contiguous()
    dllm.kv4_store(small, k[:, :R].contiguous(), v[:, :R].contiguous(), pos=pos)
    dllm.kv4_store(pick, k[:, :R].contiguous(), v[:, :R].contiguous(), start=keep - R)
    o3, lse3 = dllm.attention_kv4(q, small, R, keep, H, lens=lens)
    check_attention(q, pick, R, keep, H, None, o3, lse3)
    dllm.kernel_status()
