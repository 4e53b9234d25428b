"""Plain 64-bit forms of the 8-bit products and of the 4-bit K / V cache's operators, for their tests."""
import math

import torch


def quantize_rows_s8(x):
    """(codes float64, scale float64): scale = max |x| / 127 and x / scale are float32 quotients by definition."""
    x = x.double()
    scale = (x.abs().amax(1) / 127).float().double()
    codes = torch.where(scale[:, None] > 0, (x / scale[:, None]).float().double().round(), 0.0).clamp(-127, 127)
    return codes, scale


def encode4(x):
    """x [..., hd] -> (codes float64 [..., hd], step, lo float64 [...])."""
    x = x.double()
    low, high = x.amin(-1), x.amax(-1)
    lo = low.float().bfloat16().double()
    step = ((high - low).float().double() / 15).float().bfloat16().double()
    step = torch.where(step == 0, torch.ones_like(step), step)
    code = ((x - lo[..., None]).float().double() / step[..., None]).float().double().round().clamp(0, 15)
    return code, step, lo


def pack4(code):
    c = code.to(torch.uint8)
    return (c[..., 0::2] | (c[..., 1::2] << 4)).contiguous()


def unpack4(codes):
    return torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double()


def random_cache(dllm, gen, B, Hkv, cap, hd, scale=1.0):
    """A cache of random codes, steps and offsets (every row of the capacity)."""
    dev = "cuda"
    codes = [torch.randint(0, 256, (B, Hkv, cap, hd // 2), generator=gen, device=dev, dtype=torch.uint8) for _ in range(2)]
    params = []
    for _ in range(2):
        step = (0.05 + 0.3 * torch.rand((B, Hkv, cap), generator=gen, device=dev)) * scale
        lo = -7.5 * step + 0.3 * scale * torch.randn((B, Hkv, cap), generator=gen, device=dev)
        params.append(torch.stack([step, lo], -1).bfloat16().contiguous())
    return dllm.KV4Cache.from_tensors(codes[0], params[0], codes[1], params[1])


def parts(cache, which):
    """(code - 8, step, lo + 8 step) in float64, [B, Hkv, cap, hd] and [B, Hkv, cap]."""
    codes, par = (cache.k_codes, cache.k_params) if which == 0 else (cache.v_codes, cache.v_params)
    step, lo = par[..., 0].double(), par[..., 1].double()
    return unpack4(codes) - 8, step, lo + 8 * step


def attention(q, cache, a, n, H, lens=None):
    """o, lse, and how far fp32 / fp16 arithmetic may put them: every tensor [B, a, H, ...] in float64.

    A score is step * (q . v) + off * sum(q).  Its fp32 sums are off by at most (hd / 16 + 4) roundings of 2^-22 of the sum of
    absolute values (a matrix instruction adds 16 products with the precision of one fp32 truncation).  A term p step v of the
    output is rounded to fp16 once: 2^-11 of it (the kernel scales it into fp16's range)."""
    B, Hkv, hd = cache.B, cache.Hkv, cache.hd
    G = H // Hkv
    kv, kstep, koff = parts(cache, 0)
    vv, vstep, voff = parts(cache, 1)
    x = q.double().reshape(B, a, Hkv, G, hd)
    o = torch.zeros((B, a, Hkv, G, hd), dtype=torch.float64, device=q.device)
    lse = torch.full((B, a, Hkv, G), -math.inf, dtype=torch.float64, device=q.device)
    o_err, s_err = torch.zeros_like(o), torch.zeros_like(lse)
    for b in range(B):
        L = n if lens is None else min(max(int(lens[b]), 0), n)
        if L == 0:
            continue
        for h in range(Hkv):
            k, v = kv[b, h, :L], vv[b, h, :L]
            dot = lambda u, w: torch.einsum("agd,nd->agn", u, w)  # noqa: E731
            total = x[b, :, h].sum(-1)[..., None]
            s = (kstep[b, h, :L] * dot(x[b, :, h], k) + koff[b, h, :L] * total) / math.sqrt(hd)
            mag = (kstep[b, h, :L].abs() * dot(x[b, :, h].abs(), k.abs()) +
                   koff[b, h, :L].abs() * x[b, :, h].abs().sum(-1)[..., None]) / math.sqrt(hd)
            lse[b, :, h] = torch.logsumexp(s, -1)
            p = torch.softmax(s, -1)
            num = v * vstep[b, h, :L, None] + voff[b, h, :L, None]
            o[b, :, h] = p @ num
            ds = (hd / 16 + 4) * 2.0 ** -22 * mag.amax(-1) + 2.0 ** -21 * (1 + s.abs().amax(-1))
            s_err[b, :, h] = ds
            size = p @ ((v * vstep[b, h, :L, None]).abs() + voff[b, h, :L, None].abs())
            o_err[b, :, h] = size * (3 * 2.0 ** -11 + 2 * ds[..., None] + L ** 0.5 * 2.0 ** -22)
    return [t.reshape(B, a, H, *t.shape[4:]) for t in (o, lse, o_err, s_err)]


def weights(q, cache, lse, a, n, H, lens=None):
    """What every key gets, [B, Hkv, cap], and how far fp32 may put it."""
    B, Hkv, hd = cache.B, cache.Hkv, cache.hd
    G = H // Hkv
    kv, kstep, koff = parts(cache, 0)
    x, e = q.double().reshape(B, a, Hkv, G, hd), lse.double().reshape(B, a, Hkv, G)
    w = torch.zeros((B, Hkv, cache.capacity), dtype=torch.float64, device=q.device)
    err = torch.zeros_like(w)
    for b in range(B):
        L = n if lens is None else min(max(int(lens[b]), 0), n)
        for h in range(Hkv if L else 0):
            total = x[b, :, h].sum(-1)[..., None]
            s = (kstep[b, h, :L] * torch.einsum("agd,nd->agn", x[b, :, h], kv[b, h, :L]) + koff[b, h, :L] * total) / math.sqrt(hd)
            mag = (kstep[b, h, :L].abs() * torch.einsum("agd,nd->agn", x[b, :, h].abs(), kv[b, h, :L].abs()) +
                   koff[b, h, :L].abs() * x[b, :, h].abs().sum(-1)[..., None]) / math.sqrt(hd)
            diff = torch.where(torch.isneginf(e[b, :, h])[..., None], torch.full_like(s, -math.inf), s - e[b, :, h][..., None])
            p = torch.exp(diff)
            w[b, h, :L] = p.sum((0, 1))
            ds = (hd / 16 + 4) * 2.0 ** -22 * mag + 2.0 ** -21 * (1 + s.abs() + e[b, :, h].abs().nan_to_num(posinf=0.0)[..., None])
            err[b, h, :L] = (p * ds).sum((0, 1)) + (a * G) ** 0.5 * 2.0 ** -22 * w[b, h, :L]
    return w, err


def evict(weight, n, keep, first, last, lens=None):
    """index [B, Hkv, keep] (-1 behind), new lengths."""
    B, Hkv, _ = weight.shape
    index = torch.full((B, Hkv, keep), -1, dtype=torch.int32)
    new = torch.zeros(B, dtype=torch.int32)
    w = weight.cpu()
    for b in range(B):
        L = n if lens is None else min(max(int(lens[b]), 0), n)
        new[b] = min(L, keep)
        for h in range(Hkv):
            if L <= keep:
                rows = list(range(L))
            else:
                forced = list(range(first)) + list(range(L - last, L))
                key = lambda j: (-math.inf if math.isnan(v := float(w[b, h, j])) else v)  # noqa: E731
                nan = lambda j: math.isnan(float(w[b, h, j]))                             # noqa: E731
                free = sorted(range(first, L - last), key=lambda j: (nan(j), -key(j), j))
                rows = sorted(forced + free[:keep - first - last])
            index[b, h, :len(rows)] = torch.tensor(rows, dtype=torch.int32)
    return index, new
