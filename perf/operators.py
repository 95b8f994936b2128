"""The operators around a decode step that are timed and compared: normalising and rotating queries and keys, attention
with a sliding window and visible first tokens, and the paged cache held in 4 bits.

A case is a dict of plain values.  `prepare` makes what a serving program holds before the call, `run` is one pass: in
elementary torch operations where `own` is false, through the library's entry points where it is true.  `exact` gives
the same results from the definitions in 64 bits, `work` the bytes and operations that a pass cannot do without.

The 4-bit cache: a record of 2176 bytes holds the 16 tokens of one page for one KV head.  An element is a sign, two bits
of exponent and one of mantissa (0, 0.5, 1, 1.5, 2, 3, 4, 6), 32 channels of a token share a power of two, stored as its
exponent plus 127 (255: the block holds an infinity or a NaN and reads as NaN).
  bytes    0..1023   keys: [token][channel / 2], the even channel in the low half of a byte
  bytes 1024..2047   values: [token / 4][channel / 8][token % 4][channel % 8 / 2]
  bytes 2048..2111   the keys' exponents: [token][channel / 32]
  bytes 2112..2175   the values' exponents: [channel / 32][token]
"""
import math

import torch

own = False

PAGE, DIM, RECORD = 16, 128, 2176
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
EVERYTHING = 2 ** 31 - 1               # a window that holds every token


# ---- the cases ------------------------------------------------------------------------------------------------------
def _rotate(tokens, kv_heads, group, dtype, rot=128, interleaved=False, far=4096, normalize=True):
    return {"op": "norm_rotate", "tokens": tokens, "kv_heads": kv_heads, "group": group, "dtype": dtype, "rot": rot,
            "interleaved": interleaved, "far": far, "normalize": normalize}


def _attend(op, batch, ctx, kv_heads, group, dtype, window, sinks, ragged):
    return {"op": op, "batch": batch, "ctx": ctx, "kv_heads": kv_heads, "group": group, "dtype": dtype, "window": window,
            "sinks": sinks, "ragged": ragged}


def _pages(pages, chosen, kv_heads, dtype):
    return {"op": "pack", "pages": pages, "chosen": chosen, "kv_heads": kv_heads, "dtype": dtype}


def listed():
    named = {
        # one request's next token, far into a long context: nothing but latency
        "rotate_1": _rotate(1, 8, 4, "bf16", far=1 << 20),
        # a serving batch's next tokens, half of each head rotated, neighbouring channels as pairs
        "rotate_61_half": _rotate(61, 4, 8, "f16", rot=64, interleaved=True, far=131072),
        # a prompt of 16K tokens
        "rotate_16k": _rotate(16384, 8, 4, "bf16", far=16384),
        # one request with a short window: latency
        "window_1k_b1": _attend("window", 1, 8192, 8, 4, "bf16", 1024, 4, False),
        # a ragged serving batch, 4K tokens visible of up to 32K, one request without tokens
        "window_4k_ragged_b64": _attend("window", 64, 32768, 8, 8, "f16", 4096, 16, True),
        # many requests with a window of a few pages that begins inside one
        "window_130_b240": _attend("window", 240, 2050, 4, 2, "bf16", 130, 1, True),
        # pages that filled up in a decode step go to the 4-bit cache, and are read back
        "pack_listed_64": _pages(1024, 64, 8, "bf16"),
        # a whole cache goes to 4 bits and is read back
        "pack_8192": _pages(8192, 0, 8, "f16"),
        # a decode step of one long request over the 4-bit cache
        "packed_32k_b1": _attend("packed", 1, 32768, 8, 4, "bf16", EVERYTHING, 0, False),
        # a decode step of four requests of 128K tokens over the 4-bit cache
        "packed_128k_b4": _attend("packed", 4, 131072, 8, 4, "bf16", EVERYTHING, 0, False),
        # a ragged batch over the 4-bit cache through a window
        "packed_window_ragged_b33": _attend("packed", 33, 30001, 8, 1, "f16", 8000, 64, True),
        # a decode step's append and attention over the 4-bit cache
        "append_attend_16k_b16": _attend("step", 16, 16000, 8, 8, "bf16", EVERYTHING, 0, True),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["norm_rotate", "window", "pack", "packed", "step"])
    heads, group, dtype = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8]), rng.choice(["f16", "bf16"])
    if op == "norm_rotate":
        return _rotate(_log(rng, 1, min(65536, 655360 // (heads * (group + 1)))), heads, group, dtype, rng.choice([128, 96, 64, 32]),
                       rng.random() < 0.5, _log(rng, 128, 1 << 20), rng.random() < 0.8)
    if op == "pack":
        pages = _log(rng, 8, 65536 // heads)
        return _pages(pages, rng.choice([0, rng.randint(1, pages)]), heads, dtype)
    batch = _log(rng, 1, 128)
    ctx = _log(rng, 1, min(131072, (4 << 20) // (heads * batch)))       # four requests of 128K tokens and 8 heads at most
    if op == "window":
        ctx = min(ctx, 65536)
        return _attend(op, batch, ctx, heads, group, dtype, _log(rng, 1, 4096), rng.choice([0, 1, 4, 16, 64]), rng.random() < 0.7)
    if op == "step":
        ctx = max(1, ctx - 1)
    window = EVERYTHING if rng.random() < 0.6 else _log(rng, 1, 8192)
    return _attend(op, batch, ctx, heads, group, dtype, window, rng.choice([0, 1, 4, 16, 64]), rng.random() < 0.7)


def _lengths(case):
    """The requests' lengths: all ctx, or spread evenly from nearly nothing to ctx (the first of four or more is empty)."""
    n, ctx = case["batch"], case["ctx"]
    if not case["ragged"] or n == 1:
        return [ctx] * n
    got = [max(1, round(ctx * (i + 1) / n)) for i in range(n)]
    if n >= 4:
        got[0] = 0
    return got


def _visible_tokens(case, length):
    return length if case["window"] + case["sinks"] >= length else case["window"] + case["sinks"]


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _generator(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + sum(ord(ch) * (i + 1) for i, ch in enumerate(str(sorted(case.items())))) % 1000003)
    return g


def _table(case, gen, extra=0):
    """Every request's pages, anywhere in the pool."""
    width = max(1, (case["ctx"] + extra + PAGE - 1) // PAGE)
    pages = case["batch"] * width + 3
    order = torch.randperm(pages, generator=gen, device="cuda")[: case["batch"] * width]
    return order.view(case["batch"], width).to(torch.int32), pages


def _keys_and_values(pages, heads, gen, dtype):
    """Keys with a few strong channels, as after a model's projections; values N(0, 1)."""
    loud = 1 + 3 * (torch.rand((heads, 1, DIM), generator=gen, device="cuda") < 0.05)
    k = torch.randn((pages, heads, PAGE, DIM), generator=gen, device="cuda", dtype=dtype).mul_(loud.to(dtype))
    return k, torch.randn((pages, heads, PAGE, DIM), generator=gen, device="cuda", dtype=dtype)


def prepare(case, seed):
    gen, dtype, heads = _generator(case, seed), TYPES[case["dtype"]], case["kv_heads"]
    if case["op"] == "pack":
        k, v = _keys_and_values(case["pages"], heads, gen, dtype)
        state = {"case": case, "k": k, "v": v, "packed": torch.zeros((case["pages"], heads, RECORD), dtype=torch.uint8, device="cuda"),
                 "k_back": torch.zeros_like(k), "v_back": torch.zeros_like(v), "list": None}
        if case["chosen"]:
            state["list"] = torch.randperm(case["pages"], generator=gen, device="cuda")[: case["chosen"]].to(torch.int32)
        return state
    q_heads = heads * case["group"]
    if case["op"] == "norm_rotate":
        rows = (q_heads + 2 * heads) * DIM                   # as a projection to queries, keys and values leaves it
        qkv = torch.randn((case["tokens"], rows), generator=gen, device="cuda").to(dtype)
        base = torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64)
        start = int(torch.randint(0, case["far"], (1,), generator=gen, device="cuda"))
        one = case["tokens"] < 256                           # next tokens of many requests, or one request's prompt
        where = torch.randint(0, case["far"], (case["tokens"],), generator=gen, device="cuda") if one else \
            start + torch.arange(case["tokens"], device="cuda")
        weights = 1 + 0.2 * torch.randn((2, DIM), generator=gen, device="cuda")
        return {"case": case, "q": qkv[:, : q_heads * DIM].view(-1, q_heads, DIM),
                "k": qkv[:, q_heads * DIM: (q_heads + heads) * DIM].view(-1, heads, DIM), "positions": where.to(torch.int32),
                "inv_freq": (500000.0 ** (-base / case["rot"])).float(), "q_weight": weights[0].to(dtype), "k_weight": weights[1].to(dtype)}
    extra = 1 if case["op"] == "step" else 0
    table, pages = _table(case, gen, extra)
    lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    lens = lens[torch.randperm(case["batch"], generator=gen, device="cuda")].contiguous()
    q = 1.5 * torch.randn((case["batch"], q_heads, DIM), generator=gen, device="cuda")
    state = {"case": case, "q": q.to(dtype), "table": table, "lens": lens}
    if case["op"] == "window":
        state["k"], state["v"] = _keys_and_values(pages, heads, gen, dtype)
        return state
    # a cache in 4 bits: codes of N(0, 1) under exponents that vary as those of keys and values do
    near = torch.tensor([0, 1, 1, 2, 2, 3, 4, 5], dtype=torch.uint8, device="cuda")
    raw = torch.randint(0, 256, (pages, heads, RECORD), generator=gen, device="cuda", dtype=torch.uint8)
    raw[..., :2048] = (near[(raw[..., :2048] & 7).long()] | near[(raw[..., :2048] >> 4 & 7).long()] << 4) | raw[..., :2048] & 0x88
    raw[..., 2048:] = 125 + raw[..., 2048:] % 3
    state["packed"] = raw
    if extra:
        state["k_new"], state["v_new"] = (torch.randn((case["batch"], heads, DIM), generator=gen, device="cuda").to(dtype) for _ in range(2))
        state["at"] = torch.empty_like(lens)
    return state


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _constants(device):
    codes = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=device)
    powers = torch.exp2(torch.arange(256, device=device, dtype=torch.float64) - 127)
    powers[255] = math.nan
    return torch.cat([codes, -codes]), powers.float()


def _norm_rotate(x, weight, cos, sin, case):
    y = x.float()
    if case["normalize"]:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * weight.float()
    rot = case["rot"]
    turned, rest = y[..., :rot], y[..., rot:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = turned[..., : rot // 2], turned[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, rest], -1).to(x.dtype)


def _attention(q, k, v, seen):
    """q [B][H][G][128], k and v [B][T][H][128], seen [B][T]: in 32 bits, a request that sees nothing gets 0 and -inf."""
    k, v = k.permute(0, 2, 3, 1), v.permute(0, 2, 1, 3)
    s = torch.matmul(q.float(), k) / math.sqrt(DIM)
    s = torch.where(seen[:, None, None], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    return out.flatten(1, 2), (top + torch.log(total)).flatten(1)


def _visible(lens, case, width):
    """Positions that may be visible, [B][sinks + window] at most, and which of them are."""
    span = width * PAGE
    sinks, window = min(case["sinks"], span), min(case["window"], span)
    if window == span:
        sinks = 0
    first = torch.arange(sinks, device=lens.device)
    last = lens.long()[:, None] - window + torch.arange(window, device=lens.device)
    at = torch.cat([first.expand(lens.numel(), -1), last], 1)
    seen = torch.cat([first < lens[:, None], last >= sinks], 1)
    return torch.where(seen, at, 0), seen


def _read_packed(raw, page, slot):
    """Keys and values of the tokens (page, slot), [B][T][H][128] in 32 bits."""
    pages, heads, _ = raw.shape
    codes, powers = _constants(raw.device)
    k = raw[..., :1024].view(pages, heads, PAGE, 64)[page, :, slot]
    v = raw[..., 1024:2048].view(pages, heads, 4, 16, 4, 4)[page, :, slot // 4, :, slot % 4].flatten(-2)
    ks = raw[..., 2048:2112].view(pages, heads, PAGE, 4)[page, :, slot]
    vs = raw[..., 2112:].view(pages, heads, 4, PAGE)[page, :, :, slot]
    return tuple((codes[torch.stack([c & 15, c >> 4], -1).flatten(-2).int()].unflatten(-1, (4, 32)) * powers[e.int()][..., None]).flatten(-2)
                 for c, e in ((k, ks), (v, vs)))


def _to_codes(x):
    """x [..., 128] to codes [..., 128] and exponents [..., 4], both uint8."""
    x = x.float().unflatten(-1, (4, 32))
    top = x.abs().amax(-1)
    fine = torch.isfinite(x).all(-1)
    fraction, power = torch.frexp(torch.where(fine, top, 1.0))           # top = fraction * 2^power, fraction in [1/2, 1)
    exponent = torch.where(top == 0, -126, power - 3 + (fraction > 0.875)).clamp(min=-126)
    y = x.double() / torch.exp2(exponent.double())[..., None]
    a = y.abs()
    code = (a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    code = torch.where(fine[..., None], code | torch.signbit(x).byte() << 3, 0)
    return code.flatten(-2), torch.where(fine, exponent + 127, 255).byte()


def _pack(k, v):
    """[..., H, 16, 128] to records [..., H, 2176]."""
    (kc, ke), (vc, ve) = _to_codes(k), _to_codes(v)
    kc, vc = (c[..., 0::2] | c[..., 1::2] << 4 for c in (kc, vc))
    vc = vc.unflatten(-1, (16, 4)).unflatten(-3, (4, 4)).transpose(-3, -2)
    return torch.cat([kc.flatten(-2), vc.flatten(-4), ke.flatten(-2), ve.transpose(-1, -2).flatten(-2)], -1)


def _plain(state):
    case = state["case"]
    if case["op"] == "norm_rotate":
        angle = state["positions"].double()[:, None] * state["inv_freq"].double()
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        return {"q": _norm_rotate(state["q"], state["q_weight"], cos, sin, case), "k": _norm_rotate(state["k"], state["k_weight"], cos, sin, case)}
    if case["op"] == "pack":
        at = slice(None) if state["list"] is None else state["list"].long()
        state["packed"][at] = _pack(state["k"][at], state["v"][at])
        pages = torch.arange(case["pages"], device="cuda") if state["list"] is None else at
        k, v = _read_packed(state["packed"], pages[:, None], torch.arange(PAGE, device="cuda")[None])
        state["k_back"][at], state["v_back"][at] = (x.permute(0, 2, 1, 3).to(state["k"].dtype) for x in (k, v))
        return {"k": state["k_back"], "v": state["v_back"]}
    table, lens = state["table"].long(), state["lens"]
    more = {}
    if case["op"] == "step":
        page, slot = table.gather(1, lens.long()[:, None] // PAGE)[:, 0], lens.long() % PAGE
        pages, heads, _ = state["packed"].shape
        (kc, ke), (vc, ve) = _to_codes(state["k_new"]), _to_codes(state["v_new"])
        raw = state["packed"]
        raw[..., :1024].view(pages, heads, PAGE, 64)[page, :, slot] = kc[..., 0::2] | kc[..., 1::2] << 4
        raw[..., 1024:2048].view(pages, heads, 4, 16, 4, 4)[page, :, slot // 4, :, slot % 4] = (vc[..., 0::2] | vc[..., 1::2] << 4).unflatten(-1, (16, 4))
        raw[..., 2048:2112].view(pages, heads, PAGE, 4)[page, :, slot] = ke
        raw[..., 2112:].view(pages, heads, 4, PAGE)[page, :, :, slot] = ve
        state["at"].copy_(lens)
        state["at"] += 1
        lens = state["at"]
        more = {"lens": lens}
    at, seen = _visible(lens, case, table.shape[1])
    page, slot = table.gather(1, at // PAGE), at % PAGE
    if case["op"] == "window":
        k, v = state["k"][page, :, slot].float(), state["v"][page, :, slot].float()
    else:
        k, v = _read_packed(state["packed"], page, slot)
    q = state["q"].unflatten(1, (case["kv_heads"], case["group"]))
    out, lse = _attention(q, k, v, seen)
    return {"out": out, "lse": lse, **more}


# ---- through the library --------------------------------------------------------------------------------------------
def _held(state):
    """What a serving program makes once and keeps beside its cache: the handle, the workspace, the output buffers."""
    if "held" not in state:
        import paper_2503_00392_amd as psa

        case = state["case"]
        held = {"psa": psa}
        if case["op"] == "norm_rotate":
            held["q"], held["k"] = torch.empty_like(state["q"].contiguous()), torch.empty_like(state["k"].contiguous())
        elif case["op"] == "pack":
            none = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
            held["from"] = psa.KvCache(state["k"], state["v"], none, none[0], case["kv_heads"])
            held["to"] = psa.KvCache(state["k_back"], state["v_back"], none, none[0], case["kv_heads"])
        else:
            lens = state["at"] if case["op"] == "step" else state["lens"]
            if case["op"] == "window":
                held["kv"] = psa.KvCache(state["k"], state["v"], state["table"], lens, state["q"].shape[1])
                size = psa.window_workspace_bytes(held["kv"], case["window"], case["sinks"])
            else:
                held["kv"] = psa.PackedCache(state["packed"], state["table"], lens, state["q"].shape[1], state["q"].dtype)
                size = psa.packed_workspace_bytes(held["kv"], case["window"], case["sinks"])
            held["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
            held["out"] = torch.empty(state["q"].shape, dtype=torch.float32, device="cuda")
            held["lse"] = torch.empty(state["q"].shape[:2], dtype=torch.float32, device="cuda")
        state["held"] = held
    return state["held"]


def _own(state):
    case, held = state["case"], _held(state)
    psa = held["psa"]
    if case["op"] == "norm_rotate":
        q, k = psa.norm_rotate(state["q"], state["k"], state["positions"], state["inv_freq"], q_weight=state["q_weight"],
                               k_weight=state["k_weight"], eps=1e-6, normalize=case["normalize"], interleaved=case["interleaved"],
                               q_out=held["q"], k_out=held["k"])
        return {"q": q, "k": k}
    if case["op"] == "pack":
        psa.pack_pages(held["from"], state["packed"], page_list=state["list"])
        psa.unpack_pages(held["to"], state["packed"], page_list=state["list"])
        return {"k": state["k_back"], "v": state["v_back"]}
    kept = {"workspace": held["workspace"], "out": held["out"], "lse": held["lse"]}
    more = {}
    if case["op"] == "window":
        out, lse = psa.window_attention(held["kv"], state["q"], case["window"], case["sinks"], **kept)
    else:
        if case["op"] == "step":
            state["at"].copy_(state["lens"])                 # the lengths that the scheduler gives for this step
            psa.append_kv_packed(held["kv"], state["k_new"], state["v_new"])
            more = {"lens": state["at"]}
        out, lse = psa.packed_attention(held["kv"], state["q"], case["window"], case["sinks"], **kept)
    return {"out": out, "lse": lse, **more}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    heads, group = case["kv_heads"], case["group"] if "group" in case else 0
    if case["op"] == "norm_rotate":
        n = case["tokens"] * heads * (group + 1) * DIM
        return {"bytes": 4 * n + 4 * case["tokens"] + 2 * case["rot"] + 4 * DIM, "flops": 10 * n}
    if case["op"] == "pack":
        n = (case["chosen"] or case["pages"]) * heads
        return {"bytes": n * 4 * PAGE * DIM * 2 + 2 * n * RECORD, "flops": n * 4 * PAGE * DIM}
    lens = [n + (case["op"] == "step") for n in _lengths(case)]
    tokens = sum(_visible_tokens(case, n) for n in lens)
    kept = 2 * 2 * DIM if case["op"] == "window" else RECORD / PAGE
    rows = case["batch"] * heads * group
    moved = tokens * heads * kept + rows * DIM * (2 + 4) + 4 * rows
    if case["op"] == "step":
        moved += case["batch"] * heads * (2 * 2 * DIM + RECORD / PAGE)
    return {"bytes": moved, "flops": tokens * heads * group * 4 * DIM}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _element(code):
    """A 4-bit element by its fields: sign, exponent (0: no hidden one), mantissa bit."""
    code = code.long()
    power, half = code >> 1 & 3, code & 1
    size = torch.where(power == 0, half * 0.5, (1 + half * 0.5) * 2.0 ** (power - 1).double())
    return torch.where(code >= 8, -size, size)


def _exact_page(raw):
    """Records [..., 2176] to keys and values [..., 16, 128] in 64 bits."""
    t, c = torch.arange(PAGE, device=raw.device)[:, None], torch.arange(DIM, device=raw.device)[None]
    k_byte = t * 64 + torch.div(c, 2, rounding_mode="floor")
    v_byte = 1024 + ((t // 4 * 16 + c // 8) * 4 + t % 4) * 4 + c % 8 // 2
    k_exp, v_exp = 2048 + t * 4 + c // 32, 2112 + c // 32 * 16 + t
    got = []
    for at, e in ((k_byte, k_exp), (v_byte, v_exp)):
        code = raw[..., at] >> (c % 2 * 4).byte() & 15
        power = raw[..., e].double()
        got.append(_element(code) * torch.where(power == 255, math.nan, 2.0 ** (power - 127)))
    return got


def _exact_nearest(x):
    """Each element of x [..., 128] as the 4-bit cache holds it, by trying every element value."""
    x = x.double().unflatten(-1, (4, 32))
    top = x.abs().amax(-1, keepdim=True)
    power = torch.ceil(torch.log2(torch.where(top == 0, 1.0, top) / 7)).clamp(min=-126)
    power = torch.where(top <= 7 * 2.0 ** (power - 1), power - 1, power)          # (the logarithm's own rounding)
    power = torch.where(top > 7 * 2.0 ** power, power + 1, power).clamp(min=-126)
    y = (x / 2.0 ** power).abs()
    best, least = torch.zeros_like(y), torch.full_like(y, math.inf)
    for value, even in ((0, True), (0.5, False), (1, True), (1.5, False), (2, True), (3, False), (4, True), (6, False)):
        off = (y - value).abs()
        better = (off < least) | ((off == least) & even)
        best, least = torch.where(better, value, best), torch.minimum(off, least)
    return (torch.sign(x) * best * 2.0 ** power).flatten(-2)


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "norm_rotate":
        turns = state["positions"].double()[:, None, None] * state["inv_freq"].double()
        result = {}
        for name in ("q", "k"):
            y = state[name].double()
            if case["normalize"]:
                y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / DIM + 1e-6) * state[name + "_weight"].double()
            half = case["rot"] // 2
            index = torch.arange(half, device=y.device)
            a, b = (2 * index, 2 * index + 1) if case["interleaved"] else (index, index + half)
            z = torch.complex(y[..., a], y[..., b]) * torch.polar(torch.ones_like(turns), turns)
            y[..., a], y[..., b] = z.real, z.imag
            result[name] = y
        return result
    if case["op"] == "pack":
        chosen = torch.ones(case["pages"], dtype=torch.bool, device="cuda")
        if state["list"] is not None:
            chosen[:] = False
            chosen[state["list"].long()] = True
        result = {}
        for name in ("k", "v"):
            result[name] = torch.zeros(state[name].shape, dtype=torch.float64, device="cuda")
            for at in torch.nonzero(chosen)[:, 0].split(512):
                result[name][at] = _exact_nearest(state[name][at])
        return result
    outs, sums = [], []
    heads, group = case["kv_heads"], case["group"]
    for r, length in enumerate(state["lens"].tolist()):
        total = length + (case["op"] == "step")
        seen = torch.arange(total, device="cuda")
        seen = (seen < case["sinks"]) | (seen >= total - case["window"])
        pages = state["table"][r].long()[: (total + PAGE - 1) // PAGE]
        used = torch.nonzero(torch.nn.functional.pad(seen, (0, pages.numel() * PAGE - total)).view(-1, PAGE).any(1))[:, 0]
        if case["op"] == "window":
            k, v = state["k"][pages[used]].double(), state["v"][pages[used]].double()
        else:
            k, v = _exact_page(state["packed"][pages[used]])
        if case["op"] == "step":
            k[-1, :, length % PAGE], v[-1, :, length % PAGE] = _exact_nearest(state["k_new"][r]), _exact_nearest(state["v_new"][r])
        at = (used[:, None] * PAGE + torch.arange(PAGE, device="cuda")).flatten()
        keep = at[at < total]
        keep = torch.nonzero(seen[keep])[:, 0]
        k, v = (x.transpose(0, 1).reshape(heads, -1, DIM)[:, keep] for x in (k, v))
        s = torch.matmul(state["q"][r].double().view(heads, group, DIM), k.transpose(1, 2).contiguous()) / DIM ** 0.5
        sums.append(torch.logsumexp(s, -1).flatten())
        outs.append(torch.matmul(torch.softmax(s, -1), v).reshape(heads * group, DIM))
    return {"out": torch.stack(outs), "lse": torch.stack(sums), **({"lens": state["lens"] + 1} if case["op"] == "step" else {})}
