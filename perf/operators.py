"""The operators that keep a cached step's two streams, weights and K / V cache, in fewer bits and fewer rows.

A partial step of a few rows is bound by streaming the projections' weights, and against a long prompt by streaming
the K / V cache.  Five operators, each in its plain form and as the framework's call:

    linear    y = x W^T with W in 8-bit integers and a scale per output channel; the rows of x (tokens) are brought to
              8-bit integers with a scale each within the call
    store     rows of K and V into a cache of 4-bit codes (one step and one offset per token and KV head), and the
              cache's rows read back as numbers
    attention queries over such a cache, sequences of their own lengths, with the log of each row's softmax sum
    weights   what every cached key has got of the queries' attention, added to what it had before
    evict     the keys with the least of it leave the cache, the others move up

Codes.  A head's K (or V) of one token, hd numbers x: lo = bf16(min x), step = bf16((max x - min x) / 15), or 1 where
that is 0; code = rint((x - lo) / step) between 0 and 15, in float32 arithmetic; it stands for lo + step * code.  Byte
i of the row holds the code of element 2i in its low half and that of 2i + 1 in its high half.  A cache is four
tensors: K codes [B, Hkv, capacity, hd / 2] uint8, K (step, lo) [B, Hkv, capacity, 2] bf16, and the same for V.

Rows of 8-bit integers.  scale = max |x| / 127, q = rint(x / scale) within +-127, both in float32; a row of zeros has
scale 0 and codes 0.
"""
import math

import torch

own = False

LINEAR_MOST = 8192 * 24576 * 4096     # products of the largest listed linear


def _linear(name, M, K, N, x, y):
    return {"name": name, "op": "linear", "M": M, "K": K, "N": N, "x": x, "y": y}


def _store(name, B, a, n, Hkv, hd, dtype, scattered):
    return {"name": name, "op": "store", "B": B, "a": a, "n": n, "Hkv": Hkv, "hd": hd, "dtype": dtype,
            "scattered": scattered}


def _attention(name, B, a, n, H, Hkv, hd, ragged):
    return {"name": name, "op": "attention", "B": B, "a": a, "n": n, "H": H, "Hkv": Hkv, "hd": hd, "ragged": ragged}


def _weights(name, B, a, n, H, Hkv, hd, ragged):
    return {"name": name, "op": "weights", "B": B, "a": a, "n": n, "H": H, "Hkv": Hkv, "hd": hd, "ragged": ragged}


def _evict(name, B, n, keep, first, last, Hkv, hd, ragged):
    return {"name": name, "op": "evict", "B": B, "n": n, "keep": keep, "first": first, "last": last, "Hkv": Hkv,
            "hd": hd, "ragged": ragged}


def listed():
    return [
        # the three rows that a partial step of 32 response rows recomputes, through W_o of the LLaDA-8B shape: the
        # smallest call, launch latency and 17 MB of weights
        _linear("linear_3_rows", 3, 4096, 4096, "bf16", "bf16"),
        # a partial step of the Dream-7B shape through its down projection
        _linear("linear_dream_down", 128, 18944, 3584, "bf16", "fp32"),
        # a response refresh of 16 sequences through gate and up of the LLaDA-8B shape: bound by the tensor cores
        _linear("linear_batch_gate_up", 8192, 4096, 24576, "bf16", "bf16"),
        # the selected rows of a partial step go to their places in one layer's cache
        _store("store_selected", 1, 64, 768, 32, 128, "bf16", True),
        # a full step of 16 sequences fills one layer's cache
        _store("store_batch", 16, 1536, 1536, 32, 128, "bf16", False),
        # a partial step of one sequence (LLaDA-8B): 64 rows against 768 keys, latency
        _attention("attention_partial", 1, 64, 768, 32, 32, 128, False),
        # a few rows of eight sequences over long documents of their own lengths, grouped heads: the cache's bytes
        _attention("attention_long_ragged", 8, 2, 32768, 28, 4, 128, True),
        # a response refresh of 16 sequences: bound by the tensor cores
        _attention("attention_batch_refresh", 16, 512, 1536, 32, 32, 128, False),
        # the 32 response rows of a question score the document's 4096 tokens (and themselves) before some leave
        _weights("weights_long_prompt", 1, 32, 4128, 32, 32, 128, False),
        # the same for four long documents with grouped heads, 192 rows each
        _weights("weights_documents", 4, 192, 16384, 28, 4, 128, True),
        # half of that document leaves one layer's cache; its first tokens and the response stay
        _evict("evict_long_prompt", 1, 4128, 2080, 4, 32, 32, 128, False),
        # eight long documents of their own lengths come down to 4096 tokens
        _evict("evict_documents", 8, 65536, 4096, 16, 64, 4, 128, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    Hkv = rng.choice([1, 2, 4, 8, 32])
    return (Hkv if Hkv == 32 else Hkv * rng.choice([1, 4, 7, 8])), Hkv, rng.choice([64, 128, 128])


def draw(rng):
    op = rng.choice(["linear", "linear", "store", "attention", "attention", "weights", "evict"])
    ragged = rng.random() < 0.5
    H, Hkv, hd = _heads(rng)
    if op == "linear":
        M, K = _log_int(rng, 1, 8192), _log_int(rng, 200, 18944)
        K = K if rng.random() < 0.3 else K // 64 * 64
        N = min(_log_int(rng, 64, 24576), 24576 * 4096 // K, max(64, LINEAR_MOST // (M * K)))
        case = _linear("", M, K, N, rng.choice(["bf16", "bf16", "fp32"]), rng.choice(["bf16", "fp32"]))
    elif op == "store":
        n = min(_log_int(rng, 16, 32768), 16 * 1536 * 32 * 128 // (Hkv * hd))
        a = _log_int(rng, 1, n)
        B = max(1, min(_log_int(rng, 1, 16), 16 * 1536 * 32 * 128 // (n * Hkv * hd)))
        case = _store("", B, a, n, Hkv, hd, rng.choice(["bf16", "bf16", "fp32"]), rng.random() < 0.5)
    elif op == "attention":
        n = min(_log_int(rng, 20, 32768), 8 * 32768 * 4 * 128 // (Hkv * hd))
        B = max(1, min(_log_int(rng, 1, 16), 8 * 32768 * 4 * 128 // (n * Hkv * hd)))
        a = max(1, min(_log_int(rng, 1, 1024), 16 * 512 * 1536 * 32 // (B * n * H)))
        case = _attention("", B, a, n, H, Hkv, hd, ragged)
    elif op == "weights":
        n = min(_log_int(rng, 20, 32768), 4 * 16384 * 4 * 128 // (Hkv * hd))
        B = max(1, min(_log_int(rng, 1, 16), 4 * 16384 * 4 * 128 // (n * Hkv * hd)))
        a = max(1, min(_log_int(rng, 1, 512), 4 * 192 * 16384 * 28 // (B * n * H)))
        case = _weights("", B, a, n, H, Hkv, hd, ragged)
    else:
        n = _log_int(rng, 40, 65536)
        B = max(1, min(_log_int(rng, 1, 16), 8 * 65536 * 4 * 128 // (n * Hkv * hd)))
        keep = max(8, min(int(n * rng.uniform(0.05, 0.9)), 8 * 4096 * 4 * 128 // (B * Hkv * hd)))
        first = rng.randint(0, keep // 4)
        case = _evict("", B, n, keep, first, rng.randint(0, keep // 2), Hkv, hd, ragged)
    del case["name"]
    return case


# ---------------------------------------------------------------- what a user's program holds before the call
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _capacity(n):
    return -(-n // 64) * 64


def _lengths(case, gen):
    """Lengths between half of n and n, the same ones in any order."""
    B, n = case["B"], case["n"]
    if not case["ragged"]:
        return None
    lens = torch.tensor([max(1, n - n * b // (2 * B)) for b in range(B)], dtype=torch.int32, device="cuda")
    return lens[torch.randperm(B, generator=gen, device="cuda")].contiguous()


def _kv(gen, B, n, Hkv, hd, dtype):
    """Keys (or values) [B, n, Hkv * hd]: unit noise about a mean per channel, a few channels four times as large."""
    scale = 1.0 + 3.0 * (torch.rand(Hkv * hd, generator=gen, device="cuda") < 0.03)
    mean = 0.5 * torch.randn(Hkv * hd, generator=gen, device="cuda")
    x = torch.randn((B, n, Hkv * hd), generator=gen, device="cuda")
    return x.add_(mean).mul_(scale).to(dtype)


def _new_cache(B, Hkv, capacity, hd):
    codes, pair = (B, Hkv, capacity, hd // 2), (B, Hkv, capacity, 2)
    return [torch.zeros(shape, dtype=dt, device="cuda")
            for shape, dt in ((codes, torch.uint8), (pair, torch.bfloat16)) * 2]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = {"case": case}
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        # normalised activations with a few large channels; weights as everywhere in this repository
        gain = 1.0 + 9.0 * (torch.rand(K, generator=gen, device="cuda") < 0.01)
        state["x"] = (torch.randn((M, K), generator=gen, device="cuda") * gain).to(DTYPES[case["x"]])
        w = 0.02 * torch.randn((N, K), generator=gen, device="cuda")
        codes, state["w_scale"] = _rows_s8(w)
        pitch = -(-K // 16) * 16
        store = torch.zeros((N, pitch), dtype=torch.int8, device="cuda")
        store[:, :K] = codes
        state["w"] = store[:, :K]
        return state
    B, n, Hkv, hd = case["B"], case["n"], case["Hkv"], case["hd"]
    cap = _capacity(n)
    state["cache"] = cache = _new_cache(B, Hkv, cap, hd)
    if case["op"] == "store":
        a, dtype = case["a"], DTYPES[case["dtype"]]
        # K and V are the last columns of the rows that one product for Q, K and V leaves
        rows = torch.cat([torch.zeros((B, a, Hkv * hd), dtype=dtype, device="cuda"),
                          _kv(gen, B, a, Hkv, hd, dtype), _kv(gen, B, a, Hkv, hd, dtype)], dim=2)
        state["k"], state["v"] = rows[:, :, Hkv * hd:2 * Hkv * hd], rows[:, :, 2 * Hkv * hd:]
        state["pos"] = None
        if case["scattered"]:
            places = torch.rand((B, n), generator=gen, device="cuda").topk(a, dim=1).indices
            state["pos"] = places.sort(dim=1).values.to(torch.int32).contiguous()
        return state
    _fill(cache, _kv(gen, B, n, Hkv, hd, torch.bfloat16), _kv(gen, B, n, Hkv, hd, torch.bfloat16))
    state["lens"] = _lengths(case, gen)
    if case["op"] == "evict":
        # accumulated weights: a long tail, some tokens never looked at (equal weights of zero)
        w = torch.rand((B, Hkv, cap), generator=gen, device="cuda").pow_(6).mul_(8.0)
        state["weight"] = w * (torch.rand((B, Hkv, cap), generator=gen, device="cuda") > 0.1)
        return state
    q = torch.randn((B * case["a"], case["H"] * hd), generator=gen, device="cuda")
    state["q"] = q.to(torch.bfloat16)
    if case["op"] == "weights":
        state["lse"] = torch.logsumexp(_scores(state), dim=3).view(B, Hkv, case["a"], -1).transpose(1, 2).reshape(
            B * case["a"], case["H"]).contiguous()
        state["weight"] = torch.rand((B, Hkv, cap), generator=gen, device="cuda")
    return state


# ---------------------------------------------------------------- plain forms
def _over(x, divisor):
    """x / divisor as IEEE division: torch multiplies by the reciprocal of a divisor that is a Python number."""
    return x / torch.full((), divisor, device="cuda")


def _rows_s8(x):
    x = x.float()
    scale = _over(x.abs().amax(dim=1), 127.0)
    safe = torch.where(scale > 0, scale, 1.0)
    return (x / safe[:, None]).round().clamp(-127, 127).to(torch.int8), scale


def _plain_linear(state):
    case = state["case"]
    q, scale = _rows_s8(state["x"])
    # sums of up to 18944 products of 8-bit integers do not fit 24 bits
    total = torch.matmul(q.double(), state["w"].double().t())
    return (total.float() * scale[:, None] * state["w_scale"][None, :]).to(DTYPES[case["y"]])


def _codes(x):
    """x [..., hd] -> codes in bytes, (step, lo)."""
    x = x.float()
    low, high = x.amin(dim=-1), x.amax(dim=-1)
    lo = low.to(torch.bfloat16)
    step = _over(high - low, 15.0).to(torch.bfloat16)
    step = torch.where(step > 0, step, torch.ones_like(step))
    code = ((x - lo.float()[..., None]) / step.float()[..., None]).round().clamp(0, 15).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.stack([step, lo], dim=-1)


def _numbers(codes, pair):
    """[B, Hkv, rows, hd / 2] -> what the codes stand for, [B, Hkv, rows, hd] in float32."""
    code = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).float()
    return code * pair[..., 0:1].float() + pair[..., 1:2].float()


def _fill(cache, k, v, pos=None):
    """k, v [B, a, Hkv * hd] into the cache's rows pos [B, a] (or the first a)."""
    B, Hkv, cap, half = cache[0].shape
    kc, kp = _codes(k.reshape(B, -1, Hkv, 2 * half).transpose(1, 2))
    vc, vp = _codes(v.reshape(B, -1, Hkv, 2 * half).transpose(1, 2))
    a = kc.shape[2]
    at = torch.arange(a, device="cuda").expand(B, a) if pos is None else pos.long()
    at = at[:, None, :, None].expand(B, Hkv, a, 1)
    cache[0].scatter_(2, at.expand(-1, -1, -1, half), kc)
    cache[1].scatter_(2, at.expand(-1, -1, -1, 2), kp)
    cache[2].scatter_(2, at.expand(-1, -1, -1, half), vc)
    cache[3].scatter_(2, at.expand(-1, -1, -1, 2), vp)


def _token_major(x):
    return x.transpose(1, 2).flatten(2).contiguous()


def _plain_store(state):
    cache, n = state["cache"], state["case"]["n"]
    _fill(cache, state["k"], state["v"], state["pos"])
    return {"k": _token_major(_numbers(cache[0][:, :, :n], cache[1][:, :, :n])),
            "v": _token_major(_numbers(cache[2][:, :, :n], cache[3][:, :, :n]))}


def _scores(state):
    """[B, Hkv, a * G, n]: softmax's arguments, -inf behind a sequence's length; row i * G + g is head g of query i."""
    case, cache = state["case"], state["cache"]
    B, a, n, H, Hkv, hd = (case[k] for k in ("B", "a", "n", "H", "Hkv", "hd"))
    q = state["q"].float().view(B, a, Hkv, H // Hkv, hd).transpose(1, 2).reshape(B, Hkv, -1, hd)
    s = torch.matmul(q, _numbers(cache[0][:, :, :n], cache[1][:, :, :n]).transpose(2, 3)).mul_(1.0 / math.sqrt(hd))
    if state["lens"] is not None:
        s.masked_fill_(torch.arange(n, device="cuda") >= state["lens"][:, None, None, None], -math.inf)
    return s


def _query_major(x, B, a):
    """[B, Hkv, a * G, ...] -> [B * a, Hkv * G, ...]"""
    return x.reshape(B, x.shape[1], a, -1, *x.shape[3:]).transpose(1, 2).flatten(2, 3).flatten(0, 1)


def _plain_attention(state):
    case, cache = state["case"], state["cache"]
    n = case["n"]
    s = _scores(state)
    top = s.amax(dim=3, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(dim=3, keepdim=True)
    o = torch.matmul(p, _numbers(cache[2][:, :, :n], cache[3][:, :, :n])).div_(total)
    lse = (top + total.log()).squeeze(3)
    return {"o": _query_major(o, case["B"], case["a"]).flatten(1).to(torch.bfloat16),
            "lse": _query_major(lse, case["B"], case["a"]).contiguous()}


def _plain_weights(state):
    case = state["case"]
    B, a, n, Hkv = case["B"], case["a"], case["n"], case["Hkv"]
    lse = state["lse"].view(B, a, Hkv, -1).transpose(1, 2).reshape(B, Hkv, -1, 1)
    weight = state["weight"].clone()
    weight[:, :, :n] += _scores(state).sub_(lse).exp_().sum(dim=2)
    return weight


def _plain_evict(state):
    case, cache, weight = state["case"], state["cache"], state["weight"]
    B, n, keep, Hkv, hd = (case[k] for k in ("B", "n", "keep", "Hkv", "hd"))
    at = torch.arange(n, device="cuda")
    lens = torch.full((B,), n, device="cuda") if state["lens"] is None else state["lens"].long()
    lens = lens[:, None, None]
    # the protected ones before all others, what lies behind a sequence's length after all others; equal ones in order
    rank = weight[:, :, :n].masked_fill((at < case["first"]) | (at >= lens - case["last"]), math.inf)
    rank = rank.masked_fill(at >= lens, -math.inf)
    chosen = rank.sort(dim=2, descending=True, stable=True).indices[:, :, :keep]
    kept = lens.clamp(max=keep)
    live = torch.arange(keep, device="cuda") < kept
    chosen = torch.where(live, chosen, n).sort(dim=2).values
    rows = chosen.clamp(max=n - 1)
    take = lambda x: x.gather(2, rows[..., None].expand(-1, -1, -1, x.shape[3]))  # noqa: E731
    zero = lambda x: torch.where(live.expand(B, Hkv, keep)[..., None], x, 0.0)    # noqa: E731
    return {"index": torch.where(live, chosen, -1).to(torch.int32), "lens": kept.view(B).to(torch.int32),
            "weight": torch.where(live, weight.gather(2, rows), 0.0),
            "k": _token_major(zero(_numbers(take(cache[0]), take(cache[1])))),
            "v": _token_major(zero(_numbers(take(cache[2]), take(cache[3]))))}


# ---------------------------------------------------------------- the framework's calls
def _framework(state):
    from paper_2506_06295_b200 import dllm
    case = state["case"]
    if case["op"] == "linear":
        return dllm.linear_s8(state["x"], state["w"], state["w_scale"], out_dtype=DTYPES[case["y"]])
    if "handle" not in state:
        state["handle"] = dllm.KV4Cache.from_tensors(*state["cache"])
    cache, n = state["handle"], case["n"]
    if case["op"] == "store":
        dllm.kv4_store(cache, state["k"], state["v"], pos=state["pos"])
        k, v = dllm.kv4_load(cache, n)
        return {"k": k, "v": v}
    if case["op"] == "attention":
        o, lse = dllm.attention_kv4(state["q"], cache, case["a"], n, case["H"], lens=state["lens"])
        return {"o": o, "lse": lse}
    if case["op"] == "weights":
        weight = state["weight"].clone()
        dllm.attention_weights_kv4(state["q"], cache, state["lse"], weight, case["a"], n, case["H"],
                                   lens=state["lens"])
        return weight
    kept, weight, index, lens = dllm.kv4_evict(cache, state["weight"], n, case["keep"], first=case["first"],
                                               last=case["last"], lens=state["lens"])
    k, v = dllm.kv4_load(kept, case["keep"], lens=lens)
    return {"index": index, "lens": lens, "weight": weight[:, :, :case["keep"]], "k": k, "v": v}


PLAIN = {"linear": _plain_linear, "store": _plain_store, "attention": _plain_attention, "weights": _plain_weights,
         "evict": _plain_evict}


def run(state):
    return _framework(state) if own else PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    size = {"bf16": 2.0, "fp32": 4.0}
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": M * K * size[case["x"]] + N * (K + 4.0) + M * N * size[case["y"]], "flops": 2.0 * M * N * K}
    B, n, Hkv, hd = case["B"], case["n"], case["Hkv"], case["hd"]
    row = hd / 2 + 4.0                                               # one head of one token, K or V
    heads = B * Hkv
    if case["op"] == "store":
        a = case["a"]
        moved = 2.0 * heads * (a * (hd * size[case["dtype"]] + row) + n * (row + 4.0 * hd))
        return {"bytes": moved, "flops": 2.0 * heads * hd * (4.0 * a + 2.0 * n)}
    lens = [max(1, n - n * b // (2 * B)) for b in range(B)] if case["ragged"] else [n] * B
    if case["op"] == "evict":
        kept = sum(min(m, case["keep"]) for m in lens) * Hkv
        moved = 4.0 * Hkv * sum(lens) + kept * (4.0 * row + 8.0 * hd + 8.0) + 4.0 * heads * case["keep"]
        return {"bytes": moved, "flops": 4.0 * kept * hd}
    rows = B * case["a"] * case["H"]
    pairs = case["a"] * case["H"] * float(sum(lens))
    if case["op"] == "attention":
        return {"bytes": 2.0 * Hkv * sum(lens) * row + rows * (4.0 * hd + 4.0), "flops": 4.0 * pairs * hd}
    return {"bytes": Hkv * sum(lens) * (row + 8.0) + rows * (2.0 * hd + 4.0), "flops": 2.0 * pairs * hd}


# ---------------------------------------------------------------- the definitions in 64 bits
def _bf16(x):
    return x.float().to(torch.bfloat16).double()


def _exact_values(cache, which, b, n):
    """Head by head what sequence b's codes stand for: [Hkv, n, hd]."""
    codes, pair = cache[2 * which][b, :, :n].int(), cache[2 * which + 1][b, :, :n].double()
    out = torch.empty((*codes.shape[:2], 2 * codes.shape[2]), dtype=torch.float64, device="cuda")
    out[:, :, 0::2] = (codes % 16) * pair[:, :, :1] + pair[:, :, 1:]
    out[:, :, 1::2] = (codes // 16) * pair[:, :, :1] + pair[:, :, 1:]
    return out


def exact(case, seed):
    state = prepare(case, seed)
    return {"linear": _exact_linear, "store": _exact_store, "attention": _exact_attention, "weights": _exact_weights,
            "evict": _exact_evict}[case["op"]](case, state)


def _exact_linear(case, state):
    out = torch.empty((case["M"], case["N"]), dtype=torch.float64, device="cuda")
    w = state["w"].double() * state["w_scale"].double()[:, None]
    for lo in range(0, case["M"], 1024):
        x = state["x"][lo:lo + 1024].double()
        scale = (x.abs().max(dim=1).values / 127).float().double()[:, None]      # the scale is a float32 number
        codes = torch.where(scale > 0, (x / scale).float().double().round(), 0.0).clamp(-127, 127)
        out[lo:lo + 1024] = (codes * scale) @ w.t()
    return out


def _exact_store(case, state):
    B, a, n, Hkv, hd = (case[k] for k in ("B", "a", "n", "Hkv", "hd"))
    found = {}
    for name in ("k", "v"):
        out = torch.zeros((B, n, Hkv, hd), dtype=torch.float64, device="cuda")
        for b in range(B):
            x = state[name][b].double().view(a, Hkv, hd)
            low, high = x.min(dim=2, keepdim=True).values, x.max(dim=2, keepdim=True).values
            lo, step = _bf16(low), _bf16((high - low).float().double() / 15)     # steps and offsets are bf16 numbers
            step = torch.where(step == 0, 1.0, step)
            code = ((x - lo).float().double() / step).float().double().round().clamp(0, 15)
            at = torch.arange(a, device="cuda") if state["pos"] is None else state["pos"][b].long()
            out[b, at] = lo + step * code
        found[name] = out.view(B, n, Hkv * hd)
    return found


def _exact_softmax(case, state, b, h):
    """Scores of sequence b's queries with KV head h's query heads: [a, G, len]."""
    B, a, H, Hkv, hd = (case[k] for k in ("B", "a", "H", "Hkv", "hd"))
    G = H // Hkv
    length = case["n"] if state["lens"] is None else int(state["lens"][b])
    q = state["q"].view(B, a, H, hd)[b, :, h * G:(h + 1) * G].double()
    return torch.einsum("agd,nd->agn", q, _exact_values(state["cache"], 0, b, length)[h]) / math.sqrt(hd), length


def _exact_attention(case, state):
    B, a, H, Hkv, hd = (case[k] for k in ("B", "a", "H", "Hkv", "hd"))
    o = torch.empty((B, a, Hkv, H // Hkv, hd), dtype=torch.float64, device="cuda")
    lse = torch.empty((B, a, Hkv, H // Hkv), dtype=torch.float64, device="cuda")
    for b in range(B):
        for h in range(Hkv):
            s, length = _exact_softmax(case, state, b, h)
            lse[b, :, h] = torch.logsumexp(s, dim=2)
            o[b, :, h] = torch.softmax(s, dim=2) @ _exact_values(state["cache"], 1, b, length)[h]
    return {"o": o.view(B * a, H * hd), "lse": lse.view(B * a, H)}


def _exact_weights(case, state):
    B, a, H, Hkv = (case[k] for k in ("B", "a", "H", "Hkv"))
    weight = state["weight"].double()
    lse = state["lse"].double().view(B, a, Hkv, H // Hkv, 1)
    for b in range(B):
        for h in range(Hkv):
            s, length = _exact_softmax(case, state, b, h)
            weight[b, h, :length] += torch.exp(s - lse[b, :, h]).sum(dim=(0, 1))
    return weight


def _exact_evict(case, state):
    B, n, keep, Hkv, hd = (case[k] for k in ("B", "n", "keep", "Hkv", "hd"))
    index = torch.full((B, Hkv, keep), -1, dtype=torch.int32, device="cuda")
    lens = torch.empty(B, dtype=torch.int32, device="cuda")
    weight = torch.zeros((B, Hkv, keep), dtype=torch.float64, device="cuda")
    k, v = (torch.zeros((B, keep, Hkv, hd), dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(B):
        length = n if state["lens"] is None else int(state["lens"][b])
        count = min(length, keep)
        lens[b] = count
        values = [_exact_values(state["cache"], which, b, length) for which in (0, 1)]
        first, last = min(case["first"], length), min(case["last"], length)
        for h in range(Hkv):
            w = state["weight"][b, h, :length].double()
            must = torch.zeros(length, dtype=torch.bool, device="cuda")
            must[:first] = True
            must[length - last:] = True
            free = (~must).nonzero()[:, 0]
            order = torch.argsort(-w[free], stable=True)[:count - int(must.sum())]
            rows = torch.cat([must.nonzero()[:, 0], free[order]]).sort().values[:count]
            index[b, h, :count] = rows.int()
            weight[b, h, :count] = w[rows]
            k[b, :count, h], v[b, :count, h] = values[0][h, rows], values[1][h, rows]
    return {"index": index, "lens": lens, "weight": weight, "k": k.view(B, keep, -1), "v": v.view(B, keep, -1)}
