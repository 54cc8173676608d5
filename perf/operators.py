"""Long-context serving operators as they are timed: one layer's calls of a
decoding or serving program, over the sizes it makes them at.

A case is a dict of plain values.  Every kind shares a layer of h query heads
of D channels over g KV heads (the layer's heads are the second group's of a
map with two groups of layers), B sequences and contexts ctx_lo .. ctx_hi:

  attend   attention of one new token per sequence over a cache held in 4 bits
           (window 0: every position, else the last `window` and `sinks` first)
  window   the same over a bf16 cache, always with a window
  prefill  causal attention of T new tokens over a bf16 cache with a window
  store    T new rows per sequence into the 4-bit cache, and read back
  norm     queries and keys of T tokens normed per head and rotated, keys and
           values stored in a bf16 cache

4 bits: blocks of 32 channels of a row share a power of two 2^e, and a value is
one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^e with a sign (nearest, ties to the
even code); e is the least for which the block's largest magnitude is below
7 * 2^e, so that it rounds to 4 or 6.

Inputs are N(0, 1) in bf16 (keys times k_scale); norm weights 1 + 0.1 N(0, 1).
"""
import math

import torch

own = False

ROPE_BASE = 10000.0
EPS = 1e-6
LAYERS, OWNERS, OWNER, READER = 4, 2, 2, 3  # layer 2 stores the heads that layers 2 and 3 read
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    pythia = dict(h=12, g=1, D=64, T=1, k_scale=1.0, window=0, sinks=0, rope=0)
    wide = dict(pythia, h=32, g=8, D=128)
    return [
        # One user's short chat: a single sequence of 129 tokens, where launches are all there is.
        dict(pythia, name="attend_one", kind="attend", B=1, ctx_lo=128, ctx_hi=128),
        # A serving batch of sequences of very different lengths, one shared head a layer.
        dict(pythia, name="attend_ragged", kind="attend", B=128, ctx_lo=512, ctx_hi=2048),
        # Few long documents, grouped heads, a peaked softmax.
        dict(pythia, name="attend_long", kind="attend", g=4, B=8, ctx_lo=32768, ctx_hi=32768,
             k_scale=3.0),
        # A layer of a 7B-like model at a full serving batch: the largest read.
        dict(wide, name="attend_7b", kind="attend", B=64, ctx_lo=8192, ctx_hi=8192),
        # Streaming conversations that outgrew their window, odd batch.
        dict(pythia, name="attend_window", kind="attend", g=4, B=31, ctx_lo=9001, ctx_hi=32767,
             window=2047, sinks=5),
        # A local layer of a 7B-like model over a bf16 cache.
        dict(wide, name="window_7b", kind="window", B=48, ctx_lo=4001, ctx_hi=16000, window=1023,
             sinks=4),
        # A batch of 2000-token prompts through a local layer.
        dict(pythia, name="prefill_prompt", kind="prefill", B=8, ctx_lo=0, ctx_hi=0, T=2000,
             window=256, sinks=4),
        # A local layer of a 7B-like model on two long prompts.
        dict(wide, name="prefill_7b", kind="prefill", B=2, ctx_lo=0, ctx_hi=0, T=4096, window=1024,
             sinks=4),
        # A batch of prompts handed to the 4-bit cache.
        dict(pythia, name="store_prompt", kind="store", g=4, B=8, ctx_lo=0, ctx_hi=0, T=2000),
        # The newest token of a serving batch stored.
        dict(pythia, name="store_token", kind="store", B=128, ctx_lo=512, ctx_hi=2047),
        # Between the projections and the attention of one decode step.
        dict(wide, name="norm_token", kind="norm", B=64, ctx_lo=100, ctx_hi=500, rope=128),
        # The same of the second part of a batch of long prompts.
        dict(pythia, name="norm_prompt", kind="norm", g=4, B=8, ctx_lo=4001, ctx_hi=4100, T=2000,
             rope=16),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["attend", "attend", "attend", "window", "window", "prefill", "prefill",
                           "store", "norm"])
        c = dict(kind=kind, h=12, g=rng.choice([1, 1, 3, 4, 12]), D=64, T=1, window=0, sinks=0,
                 rope=0, k_scale=rng.choice([1.0, 1.0, 3.0]))
        if rng.random() < 0.4:
            c.update(h=32, g=rng.choice([2, 4, 8]), D=128)
        c["B"] = _log_int(rng, 1, 160)
        c["ctx_hi"] = _log_int(rng, 16, 32768)
        if kind in ("prefill", "store", "norm") and (kind == "prefill" or rng.random() < 0.5):
            c["T"] = _log_int(rng, 2, 4096)
            c["B"] = _log_int(rng, 1, 16)
            c["ctx_hi"] = rng.choice([0, _log_int(rng, 16, 8192)])
        if kind in ("window", "prefill") or (kind == "attend" and rng.random() < 0.4):
            c["window"] = _log_int(rng, 16, 4096)
            c["sinks"] = rng.choice([0, 1, 4, 4, rng.randint(5, 128)])
        if kind == "norm":
            c["rope"] = rng.choice([16, c["D"] // 4, c["D"]])
        c["ctx_lo"] = c["ctx_hi"] if rng.random() < 0.4 else rng.randint(c["ctx_hi"] // 4, c["ctx_hi"])
        w = work(c)
        held = 4 * c["B"] * c["g"] * _capacity(c) * c["D"]
        pairs = c["B"] * c["h"] * c["T"] * _capacity(c) if kind == "prefill" else 0
        if kind == "norm":
            held *= 8  # its whole planes are outputs
        if w["bytes"] <= 1.1e9 and held <= 2.2e9 and pairs <= 1.07e9:
            return c


def _capacity(c):
    return (c["ctx_hi"] + c["T"] + 63) // 64 * 64


def _normal(shape, seed, stream, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed((int(seed) & 0x7FFFFFFF) * 64 + stream)
    t = torch.randn(shape, dtype=torch.bfloat16, device="cuda", generator=g)
    return t if scale == 1.0 else t * scale


Q, K_ROWS, V_ROWS, K_NEW, V_NEW, Q_WEIGHT, K_WEIGHT = range(7)


def _ctx(c, seed):
    g = torch.Generator().manual_seed(int(seed) + 99)
    ctx = torch.randint(c["ctx_lo"], c["ctx_hi"] + 1, (c["B"],), generator=g, dtype=torch.int32)
    return ctx.cuda()


def _rows(c, seed):
    """The layer's cached keys and values, [g][B][S][D]."""
    shape = (c["g"], c["B"], _capacity(c), c["D"])
    return (_normal(shape, seed, K_ROWS, c["k_scale"]), _normal(shape, seed, V_ROWS))


def _projected(c, seed):
    """Queries, keys and values of the T new tokens, as one projection leaves
    them: columns of one [B][T][(h + 2 g) D] tensor."""
    B, T, h, g, D = c["B"], c["T"], c["h"], c["g"], c["D"]
    x = _normal((B, T, (h + 2 * g) * D), seed, Q)
    return (x[..., :h * D].view(B, T, h, D), x[..., h * D:(h + g) * D].view(B, T, g, D),
            x[..., (h + g) * D:].view(B, T, g, D))


def _weights(c, seed):
    return tuple(1 + 0.1 * _normal((c["D"],), seed, w) for w in (Q_WEIGHT, K_WEIGHT))


def _query_shape(c):
    return (c["B"], c["T"], c["h"], c["D"]) if c["kind"] == "prefill" else \
        (c["B"], c["h"], c["D"])


def prepare(case, seed):
    c = case
    B, T, h, g, D, S = c["B"], c["T"], c["h"], c["g"], c["D"], _capacity(c)
    s = dict(case=c, ctx=_ctx(c, seed))
    if own:
        import paper_2406_09297_amd as mlkv

        s["mlkv"] = mlkv
        s["map"] = mlkv.Map.uniform(LAYERS, h, OWNERS, g)
    n_kv, first = OWNERS * g, g  # the layer's heads are the second group's
    if c["kind"] in ("attend", "window", "prefill"):
        s["q"] = _normal(_query_shape(c), seed, Q)
        s["out"] = torch.empty_like(s["q"])
        s["lens"] = s["ctx"] + 1
        k, v = _rows(c, seed)
        if own:
            kind = s["mlkv"].QCache if c["kind"] == "attend" else s["mlkv"].Cache
            s["cache"] = kind.empty(n_kv, B, S, D)
            s["cache"].write_rows(k, v, first)
            s["ws"] = s["mlkv"].window_workspace(s["map"], B, S, D)
        elif c["kind"] == "attend":
            s["k"], s["v"] = _pack(k), _pack(v)
        else:
            s["k"], s["v"] = k, v
    elif c["kind"] == "store":
        shape = (B, T, g, D)
        s["k_new"], s["v_new"] = _normal(shape, seed, K_NEW, c["k_scale"]), _normal(shape, seed, V_NEW)
        if own:
            s["cache"] = s["mlkv"].QCache.empty(n_kv, B, S, D)
        else:
            s["k"], s["v"] = (tuple(torch.zeros((g, B, S, n), dtype=torch.uint8, device="cuda")
                                    for n in (D // 2, D // 32)) for _ in range(2))
    else:
        s["q"], s["k_new"], s["v_new"] = _projected(c, seed)
        s["q_weight"], s["k_weight"] = _weights(c, seed)
        s["q_out"] = torch.empty((B, T, h, D), dtype=torch.bfloat16, device="cuda")
        s["k"] = torch.zeros((n_kv, B, S, D), dtype=torch.bfloat16, device="cuda")
        s["v"] = torch.zeros((n_kv, B, S // 32, D, 32), dtype=torch.bfloat16, device="cuda")
        if own:
            s["cache"] = s["mlkv"].Cache(s["k"], s["v"])
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    c, mlkv, cache = s["case"], s["mlkv"], s["cache"]
    if c["kind"] == "attend":
        mlkv.qcache_decode_attention(READER, s["q"], cache, s["map"], s["lens"], s["out"],
                                     window=c["window"], sinks=c["sinks"],
                                     max_len_hint=c["ctx_hi"] + 1, ws=s["ws"])
        return {"out": s["out"]}
    if c["kind"] == "window":
        mlkv.decode_attention_window(READER, s["q"], cache, s["map"], s["lens"], s["out"],
                                     window=c["window"], sinks=c["sinks"],
                                     max_len_hint=c["ctx_hi"] + 1, ws=s["ws"])
        return {"out": s["out"]}
    if c["kind"] == "prefill":
        mlkv.prefill_attention_window(READER, s["q"], cache, s["map"], s["ctx"], s["out"],
                                      window=c["window"], sinks=c["sinks"])
        return {"out": s["out"]}
    if c["kind"] == "store":
        mlkv.qcache_append_rows(OWNER, s["map"], cache, s["k_new"], s["v_new"], s["ctx"])
        k, v = cache.read_rows(c["g"], c["g"], starts=s["ctx"], T=c["T"])
        return {"k": k, "v": v}
    mlkv.norm_rope_append(OWNER, s["map"], cache, s["q"], s["k_new"], s["v_new"], s["ctx"],
                          s["q_out"], q_norm=s["q_weight"], k_norm=s["k_weight"], eps=EPS,
                          rotary_dims=c["rope"], rotary_base=ROPE_BASE)
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


# ---------------------------------------------------------------------------
# The plain form.
# ---------------------------------------------------------------------------
def _pack(x):
    """bf16 rows [..., D] -> (codes [..., D/2], two a byte, exponents + 127 [..., D/32])."""
    b = x.float().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    mantissa, exponent = torch.frexp(top)  # top = mantissa 2^exponent, mantissa in [0.5, 1)
    e = (exponent - 3 + (mantissa >= 0.875)).clamp(-125, 125)
    m = torch.ldexp(b.abs(), -e)
    code = ((m > 0.25).byte() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5)
            + (m > 5.0)) | (torch.signbit(b).byte() << 3)
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).squeeze(-1).byte()


def _unpack(codes, exponents):
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)
    x = torch.stack((grid[(codes & 15).int()], grid[(codes >> 4).int()]), -1).flatten(-2)
    scale = torch.exp2(exponents.float() - 127)
    return (x.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


def _softmax(x):
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _run_plain(s):
    c = s["case"]
    B, T, h, g, D = c["B"], c["T"], c["h"], c["g"], c["D"]
    if c["kind"] in ("attend", "window"):
        k, v, lens = s["k"], s["v"], s["lens"].long()
        S = _capacity(c)
        if c["window"]:  # only the rows that are attended: the first ones and the last ones
            width, first = min(c["window"], S), min(c["sinks"], S)
            recent = lens[:, None] - width + torch.arange(width, device="cuda")
            early = torch.arange(first, device="cuda").expand(B, first)
            at = torch.cat((early, recent), 1)
            kept = torch.cat((early < lens[:, None] - width, recent >= 0), 1)
            seqs, at = torch.arange(B, device="cuda")[:, None], at.clamp(min=0)
            pick = lambda x: x[:, seqs, at]  # noqa: E731
        else:
            kept = torch.arange(S, device="cuda") < lens[:, None]
            pick = lambda x: x  # noqa: E731
        if c["kind"] == "attend":
            k, v = _unpack(*map(pick, k)), _unpack(*map(pick, v))
        else:
            k, v = pick(k).float(), pick(v).float()
        q = s["q"].float().view(B, g, h // g, D).transpose(0, 1)
        x = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(D)
        w = _softmax(x.masked_fill(~kept[None, :, None], -math.inf))
        return {"out": torch.matmul(w, v).transpose(0, 1).reshape(B, h, D).bfloat16()}
    ctx = s["ctx"].long()
    at = ctx[:, None] + torch.arange(T, device="cuda")  # [B][T]
    seqs = torch.arange(B, device="cuda")[:, None]
    if c["kind"] == "prefill":
        k, v = s["k"].float(), s["v"].float()
        q = s["q"].float().view(B, T, g, h // g, D).permute(2, 0, 3, 1, 4).flatten(2, 3)
        x = torch.matmul(q, k.transpose(2, 3)).unflatten(2, (h // g, T)) / math.sqrt(D)
        p, n = torch.arange(k.shape[2], device="cuda"), at[..., None]
        kept = (p <= n) & ((p < c["sinks"]) | (p > n - c["window"]))
        w = _softmax(x.masked_fill_(~kept[None, :, None], -math.inf)).flatten(2, 3)
        out = torch.matmul(w, v).unflatten(2, (h // g, T))
        return {"out": out.permute(1, 3, 0, 2, 4).reshape(B, T, h, D).bfloat16()}
    if c["kind"] == "store":
        result = {}
        for name in ("k", "v"):
            codes, exponents = _pack(s[name + "_new"].permute(2, 0, 1, 3))  # [g][B][T][D]
            s[name][0][:, seqs, at] = codes
            s[name][1][:, seqs, at] = exponents
            result[name] = _unpack(s[name][0][:, seqs, at], s[name][1][:, seqs, at]).bfloat16()
        return result
    # norm
    half = c["rope"] // 2
    turn = at.double()[..., None] * ROPE_BASE ** (-torch.arange(half, device="cuda").double() / half)
    cos, sin = turn.cos().float()[:, :, None], turn.sin().float()[:, :, None]

    def normed(x, weight):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
        lo, hi = x[..., :half], x[..., half:2 * half]
        return torch.cat((lo * cos - hi * sin, hi * cos + lo * sin, x[..., 2 * half:]), -1).bfloat16()

    s["q_out"].copy_(normed(s["q"], s["q_weight"]))
    k_new, v_new = normed(s["k_new"], s["k_weight"]), s["v_new"]
    # The cache's planes: keys in blocks of 32 tokens of matrix-core operands, values in
    # blocks of 32 tokens, channel by channel.
    u, chunk = (at & 31)[..., None], torch.arange(D // 8, device="cuda")
    place = ((((u >> 2) & 1) * (D // 32) + (chunk >> 2)) * 64 + (chunk & 3) * 16
             + ((u >> 3) << 2) + (u & 3))
    keys = s["k"].view(-1, B, s["k"].shape[2] // 32, 4 * D, 8)
    keys[g:, seqs[..., None], (at >> 5)[..., None], place] = \
        k_new.permute(2, 0, 1, 3).unflatten(-1, (-1, 8))
    s["v"].transpose(3, 4)[g:, seqs, at >> 5, at & 31] = v_new.permute(2, 0, 1, 3)
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


# ---------------------------------------------------------------------------
# What a pass cannot do without.
# ---------------------------------------------------------------------------
def _attended(n, c):
    """Positions that a query at position n (n + 1 tokens in all) attends."""
    if not c["window"]:
        return n + 1
    return min(n + 1, c["window"]) + min(max(n + 1 - c["window"], 0), c["sinks"])


def work(case):
    c = case
    B, T, h, g, D = c["B"], c["T"], c["h"], c["g"], c["D"]
    n = (c["ctx_lo"] + c["ctx_hi"]) // 2
    packed, plain = D + D // 16, 4 * D  # bytes of a token's key and value
    if c["kind"] in ("attend", "window"):
        rows = _attended(n, c)
        return {"bytes": B * (g * rows * (packed if c["kind"] == "attend" else plain) + 4 * h * D),
                "flops": 4 * B * h * D * rows}
    if c["kind"] == "prefill":
        pairs = sum(_attended(n + t, c) for t in range(T))
        rows = min(n + T, T + c["window"] + c["sinks"]) if c["window"] else n + T
        return {"bytes": B * (g * rows * plain + 4 * T * h * D), "flops": 4 * B * h * D * pairs}
    if c["kind"] == "store":
        return {"bytes": 2 * B * T * g * (plain + packed), "flops": 0}
    return {"bytes": B * T * (4 * h * D + 2 * g * plain), "flops": 8 * B * T * (h + g) * D}


# ---------------------------------------------------------------------------
# The same results in 64 bits, from the definition.
# ---------------------------------------------------------------------------
def _held(x):
    """The values that rows [..., D] stand for in 4 bits: each rounded to the
    grid's step in its own binade."""
    x = x.double()
    blocks = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    top = blocks.abs().max(-1, keepdim=True).values
    e = torch.where(top > 0, torch.floor(torch.log2(top.clamp(min=2.0 ** -140) / 7)) + 1, -125.0)
    e = torch.where(top < 7 * torch.exp2(e - 1), e - 1, e)
    e = torch.where(top >= 7 * torch.exp2(e), e + 1, e).clamp(-125, 125)
    y = blocks / torch.exp2(e)
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return (torch.round(y / step) * step * torch.exp2(e)).reshape(x.shape)


def _attend(q, k, v, kept):
    """q [..., R][D] over k, v [..., N][D]; kept [..., R][N]."""
    x = (q @ k.transpose(-1, -2)) * (q.shape[-1] ** -0.5)
    return torch.softmax(torch.where(kept, x, -math.inf), -1) @ v


def exact(case, seed):
    c = case
    B, T, h, g, D = c["B"], c["T"], c["h"], c["g"], c["D"]
    ctx, G = _ctx(c, seed).long(), c["h"] // c["g"]
    limit = c["window"] or 1 << 40
    if c["kind"] in ("attend", "window", "prefill"):
        q = _normal(_query_shape(c), seed, Q).double().reshape(B, T, h, D)
        k, v = _rows(c, seed)
        p = torch.arange(k.shape[2], device="cuda")
        out = torch.empty_like(q)
        for b in range(B):
            n = (ctx[b] + torch.arange(T, device="cuda"))[:, None]
            kept = (p <= n) & ((p < c["sinks"]) | (n - p < limit))
            for r in range(g):
                kr, vr = k[r, b], v[r, b]
                kr, vr = (_held(kr), _held(vr)) if c["kind"] == "attend" else (kr.double(), vr.double())
                for i in range(r * G, (r + 1) * G) if T > 1 else (slice(r * G, (r + 1) * G),):
                    if T > 1:
                        out[b, :, i] = _attend(q[b, :, i], kr, vr, kept)
                    else:
                        out[b, 0, i] = _attend(q[b, 0, i], kr, vr, kept.expand(G, -1))
        return {"out": out.reshape(_query_shape(c))}
    if c["kind"] == "store":
        shape = (B, T, g, D)
        return {"k": _held(_normal(shape, seed, K_NEW, c["k_scale"])).permute(2, 0, 1, 3),
                "v": _held(_normal(shape, seed, V_NEW)).permute(2, 0, 1, 3)}
    q, k, v = (x.double() for x in _projected(c, seed))
    wq, wk = (w.double() for w in _weights(c, seed))
    j = torch.arange(c["rope"] // 2, dtype=torch.float64, device="cuda")
    angle = (ctx[:, None] + torch.arange(T, device="cuda")).double()[:, :, None, None] \
        / ROPE_BASE ** (2 * j / c["rope"])
    turned = torch.polar(torch.ones_like(angle), angle)

    def of(x, w):
        y = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / D + EPS) * w
        z = torch.complex(y[..., :c["rope"] // 2], y[..., c["rope"] // 2:c["rope"]]) * turned
        return torch.cat((z.real, z.imag, y[..., c["rope"]:]), -1)

    kn = of(k, wk)
    S = _capacity(c)
    keys = torch.zeros((OWNERS * g, B, S // 32, 2, D // 32, 4, 4, 4, 8), dtype=torch.float64,
                       device="cuda")
    values = torch.zeros((OWNERS * g, B, S // 32, D, 32), dtype=torch.float64, device="cuda")
    rows = torch.zeros((2, g, B, S, D), dtype=torch.float64, device="cuda")
    for b in range(B):
        rows[0, :, b, ctx[b]:ctx[b] + T] = kn[b].transpose(0, 1)
        rows[1, :, b, ctx[b]:ctx[b] + T] = v[b].transpose(0, 1)
    # token of a block = 8 a + 4 half + i, channel = 32 step + 8 part + e; held as
    # [half][step][part][a][i][e].
    keys[g:] = rows[0].reshape(g, B, S // 32, 4, 2, 4, D // 32, 4, 8).permute(0, 1, 2, 4, 6, 7, 3, 5, 8)
    values[g:] = rows[1].reshape(g, B, S // 32, 32, D).transpose(3, 4)
    return {"q": of(q, wq), "k": keys.reshape(OWNERS * g, B, S, D), "v": values}
