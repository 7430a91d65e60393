"""Cases of the 4-bit cache path: what a serving program calls its operators for, and their plain form.

Queries and keys of a transformer layer are normed for each head and rotated by their positions (one
axis for text, several for images and video), keys and values are kept in 4 bits, and attention reads
them there.  4-bit form: e2m1 codes (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives; channel 2 i in
the low half of byte i) with one power-of-two scale per 32 channels of a token and head (value = code
* 2^(e - 127) for the scale byte e, the smallest that fits the block's largest value under 6).  A
page holds 64 tokens.

What the ranges stand for
  rope     queries and keys between their product and the cache: a decode step's tokens at far
           positions, the latent tokens of images with their text, of a video
  append   keys and values of new tokens into the pages of their sequences, and their values as the
           cache now holds them (the pages themselves are returned too: bytes of two codes, scale bytes)
  read     what the cache holds, in 16 bits: a kept prefix on its way to another operator, the last
           tokens of many sequences
  attention  queries over a cache: one token of many sequences, one very long sequence, a chunk of
           prompt under its causal limit, latent tokens over a text context
"""
import math

import torch

own = False

if torch.cuda.is_available():
    torch.backends.cuda.matmul.allow_tf32 = False

PAGE = 64    # tokens of a cache page
BLOCK = 32   # channels of a scale
EPS = 1e-6
THETA = 10000.0
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # the next token of 32 sequences, as far as 200000 tokens in: launches are all there is
        dict(name="rope_tokens", kind="rope", form="text", R=32, S=1, Hq=32, H=8, dh=128,
             axes="128", halves=True, norm=True, dtype="bf16"),
        # 64 x 64 latent tokens behind 77 text tokens, with guidance, 20 heads of 64
        dict(name="rope_image", kind="rope", form="image", R=2, S=4173, Hq=20, H=20, dh=64,
             axes="16,24,24", halves=False, norm=True, dtype="f16"),
        # 16 latent frames of 32 x 32, 20 heads of 128, uneven axes
        dict(name="rope_video", kind="rope", form="video", R=1, S=16384, Hq=20, H=20, dh=128,
             axes="44,42,42", halves=False, norm=True, dtype="bf16"),
        # one token of each of 64 sequences
        dict(name="append_tokens", kind="append", R=64, T=1, H=8, dh=128, past=1000, dtype="bf16"),
        # ragged prompts, some behind a kept prefix
        dict(name="append_prompts", kind="append", R=8, T=2000, H=8, dh=128, past=300, dtype="f16"),
        # the last tokens of 64 sequences, heads of 80
        dict(name="read_window", kind="read", R=64, T=16, H=8, dh=80, past=1000, dtype="f16"),
        # kept prefixes of eight sequences, whole
        dict(name="read_prefix", kind="read", R=8, T=4096, H=8, dh=128, past=0, dtype="bf16"),
        # the next token of one short sequence: launches again
        dict(name="attn_first", kind="attention", R=1, S=1, L=100, Hq=8, H=2, dh=64, causal=False,
             dtype="f16"),
        # the next token of 32 sequences of up to 8192, four query heads to a key head
        dict(name="attn_tokens", kind="attention", R=32, S=1, L=8192, Hq=32, H=8, dh=128,
             causal=False, dtype="bf16"),
        # the next token of one long sequence
        dict(name="attn_long", kind="attention", R=1, S=1, L=200_000, Hq=32, H=8, dh=128,
             causal=False, dtype="f16"),
        # a chunk of two prompts behind what is cached already
        dict(name="attn_chunk", kind="attention", R=2, S=2048, L=4096, Hq=16, H=4, dh=128,
             causal=True, dtype="bf16"),
        # 64 x 64 latent tokens of two images, with guidance, over their text
        dict(name="attn_context", kind="attention", R=4, S=4096, L=77, Hq=10, H=10, dh=64,
             causal=False, dtype="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rope", "rope", "rope", "append", "append", "read", "read", "attention",
                       "attention", "attention", "attention"))
    dtype = rng.choice(("f16", "bf16"))
    dh = rng.choice((64, 128, 128, 40, 80, 160, 32, 16))
    H = rng.choice((1, 2, 4, 8, 8, 10))
    if kind == "rope":
        form = rng.choice(("text", "image", "video"))
        group = rng.choice((1, 1, 2, 4, 8)) if form == "text" else 1
        halves = rng.random() < 0.5
        if form == "text":  # some turn only the first channels of a head
            axes = (rng.choice((dh, dh, dh // 2)),)
        else:               # uneven thirds, or the last two axes alone
            a = 2 * rng.randint(1, dh // 6)
            b = (dh - a) // 4 * 2
            axes = (a, b, dh - a - b) if form == "video" or rng.random() < 0.5 else (0, b, b)
        most = 40_000_000 // (dh * H * (group + 1))
        R, S = rng.choice(((_log(rng, 1, 200), 1), (rng.randint(1, 4), _log(rng, 16, 16384))))
        return dict(kind=kind, form=form, R=R, S=max(1, min(S, most // R)), Hq=H * group, H=H, dh=dh,
                    axes=",".join(map(str, axes)), halves=halves, norm=rng.random() < 0.8,
                    dtype=dtype)
    if kind in ("append", "read"):
        R, T = rng.choice(((_log(rng, 1, 200), rng.randint(1, 4)), (rng.randint(1, 8),
                                                                    _log(rng, 16, 2000))))
        return dict(kind=kind, R=R, T=T, H=H, dh=dh, past=_log(rng, 1, 1500), dtype=dtype)
    form = rng.choice(("tokens", "tokens", "long", "chunk", "context"))
    group = rng.choice((1, 2, 4, 4, 8))
    if form == "tokens":
        R, S, L = _log(rng, 1, 64), rng.choice((1, 1, 1, 2, 5)), _log(rng, 64, 4096)
    elif form == "long":
        R, S, L = rng.randint(1, 2), 1, _log(rng, 20_000, 90_000)
    elif form == "chunk":
        R, S = rng.randint(1, 3), _log(rng, 16, 1500)
        L, group = S + _log(rng, 1, 1500), min(group, 4)
        H = min(H, 4)
    else:
        R, S, L, group = rng.randint(2, 8), rng.choice((256, 1024, 900)), 77, 1
    return dict(kind=kind, R=R, S=S, L=L, Hq=H * group, H=H, dh=dh, causal=form == "chunk",
                dtype=dtype)


# ------------------------------------------------------------------------------ 4-bit values

def _scale(e):
    """2^(e - 127) of scale bytes in [1, 254], as float32."""
    return (e.int() << 23).view(torch.float32)


def _exponent(amax):
    """The scale byte of blocks whose largest magnitudes are amax (float32): 6 = 1.5 * 2^2."""
    return (((amax.view(torch.int32) + 0x3FFFFF) >> 23) - 2).clamp(1, 254)


def _codes(x):
    """Nearest e2m1 codes of float32 |x| <= 6, ties to the even code; the sign is bit 3."""
    a = x.abs()
    c = torch.zeros_like(x, dtype=torch.uint8)
    for step, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False),
                     (3.5, True), (5.0, False)):
        c += (a >= step) if up else (a > step)
    return c | (torch.signbit(x).to(torch.uint8) << 3)


def _quantise(x):
    """float32 x [..., dh] -> (bytes [..., dh / 2], scale bytes [..., ceil(dh / 32)])."""
    dh = x.shape[-1]
    b = torch.nn.functional.pad(x, (0, -dh % BLOCK)).unflatten(-1, (-1, BLOCK))
    e = _exponent(b.abs().amax(-1))
    c = _codes(b * _scale(254 - e)[..., None]).flatten(-2)[..., :dh]
    return c[..., ::2] | (c[..., 1::2] << 4), e.to(torch.uint8)


def _values(codes, e):
    """The float32 values of bytes [..., dh / 2] with their scale bytes."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    table = torch.cat((table, -table))
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    return table[c] * _scale(e).repeat_interleave(BLOCK, -1)[..., :c.shape[-1]]


# ------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) & 0x7FFFFFFF)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _pool(g, c, W):
    """A cache of R sequences of W pages each, in shuffled pages, and some free pages."""
    R, H, dh = c["R"], c["H"], c["dh"]
    P = R * W + 3
    ch = 0.5 + torch.rand(H, 1, dh, generator=g, device="cuda")
    out = []
    for gain in (ch, 1.0):
        codes = torch.empty(P, H, PAGE, dh // 2, dtype=torch.uint8, device="cuda")
        e = torch.empty(P, H, PAGE, -(-dh // BLOCK), dtype=torch.uint8, device="cuda")
        for a in range(0, P, 512):
            b = min(P, a + 512)
            codes[a:b], e[a:b] = _quantise(_randn(g, b - a, H, PAGE, dh) * gain)
        out.append((codes, e.view(torch.float8_e8m0fnu)))
    table = torch.randperm(P, generator=g, device="cuda")[:R * W].view(R, W).int()
    return dict(kp=out[0][0], vp=out[1][0], ks=out[0][1], vs=out[1][1], table=table)


def _lengths(g, R, most, least):
    """Ragged lengths, the first row's the longest."""
    n = torch.randint(least, most + 1, (R,), generator=g, device="cuda")
    n[0] = most
    return n.int()


def _positions(g, c, n):
    """Positions [R][S][n]: far ones of single tokens, or the places of a grid."""
    R, S = c["R"], c["S"]
    if c["form"] == "text":
        first = torch.randint(0, 200_000, (R, 1, 1), generator=g, device="cuda")
        return (first + torch.arange(S, device="cuda")[:, None]).int()
    text = 77 if c["form"] == "image" and S > 400 else 0   # text tokens stand at 0
    side = max(1, math.isqrt((S - text) // (16 if c["form"] == "video" else 1)))
    i = (torch.arange(S, device="cuda") - text).clamp(min=0)
    first = torch.randint(0, 16, (R, 1), generator=g, device="cuda")
    t, y, x = (i // (side * side)) + first, (i // side % side).expand(R, S), (i % side).expand(R, S)
    return torch.stack((t, y, x), -1)[..., 3 - n:].int().contiguous()


def prepare(case, seed):
    g, c, t = _gen(seed), case, TYPES[case["dtype"]]
    R, H, dh = c["R"], c["H"], c["dh"]
    if c["kind"] == "rope":
        axes = tuple(map(int, c["axes"].split(",")))
        f = [THETA ** (-2.0 * i / a) for a in axes for i in range(a // 2)]
        # queries, keys and values come out of one product
        qkv = _randn(g, R, c["S"], (c["Hq"] + 2 * H) * dh) * \
            (0.5 + 2 * torch.rand((c["Hq"] + 2 * H) * dh, generator=g, device="cuda"))
        w = lambda: 1 + 0.2 * _randn(g, dh) if c["norm"] else None
        return dict(case=c, axes=axes, qkv=qkv.to(t), pos=_positions(g, c, len(axes)), wq=w(), wk=w(),
                    freqs=torch.tensor(f, dtype=torch.float64, device="cuda"))
    if c["kind"] in ("append", "read"):
        s = _pool(g, c, -(-(c["past"] + c["T"]) // PAGE))
        pos = _lengths(g, R, c["past"], 0)
        count = _lengths(g, R, c["T"], 1 if c["T"] < 16 else c["T"] // 4)
        if c["kind"] == "read":
            return dict(s, case=c, pos=pos, count=count)
        return dict(s, case=c, pos=pos, count=count, k=(1.5 * _randn(g, R, c["T"], H * dh)).to(t),
                    v=_randn(g, R, c["T"], H * dh).to(t))
    lens = _lengths(g, R, c["L"], c["L"] if c["L"] < 100 else max(c["S"], c["L"] // 4))
    s = _pool(g, c, -(-c["L"] // PAGE))
    return dict(s, case=c, lens=lens, qpos=(lens - c["S"]).contiguous() if c["causal"] else None,
                q=_randn(g, R, c["S"], c["Hq"] * dh).to(t))


def _qk(s):
    """Views of the queries and keys in the product's rows."""
    c = s["case"]
    nq, nk = c["Hq"] * c["dh"], c["H"] * c["dh"]
    return s["qkv"][..., :nq], s["qkv"][..., nq:nq + nk]


# ------------------------------------------------------------------------------ the plain form

def _rope_one(x, w, s, cos, sin):
    c = s["case"]
    x = x.float().unflatten(-1, (-1, c["dh"]))                     # [R][S][heads][dh]
    if c["norm"]:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
    parts, at, p = [], 0, 0
    for a in s["axes"]:
        y, co, si = x[..., at:at + a], cos[:, :, None, p:p + a // 2], sin[:, :, None, p:p + a // 2]
        if c["halves"]:
            u, v = y[..., :a // 2], y[..., a // 2:]
            parts += [u * co - v * si, v * co + u * si]
        else:
            u, v = y[..., ::2], y[..., 1::2]
            parts.append(torch.stack((u * co - v * si, v * co + u * si), -1).flatten(-2))
        at, p = at + a, p + a // 2
    return torch.cat(parts + [x[..., at:]], -1).flatten(-2).to(TYPES[c["dtype"]])


def _rope(s):
    axis = torch.repeat_interleave(torch.arange(len(s["axes"]), device="cuda"),
                                   torch.tensor([a // 2 for a in s["axes"]], device="cuda"),
                                   output_size=sum(s["axes"]) // 2)
    angle = s["pos"].double()[..., axis] * s["freqs"]              # far positions: 64 bits
    cos, sin = angle.cos().float(), angle.sin().float()
    q, k = _qk(s)
    return _rope_one(q, s["wq"], s, cos, sin), _rope_one(k, s["wk"], s, cos, sin)


def _places(s):
    """(rows, tokens, page, slot) of the tokens of a call that the cache holds, and their mask."""
    T, table = s["case"]["T"], s["table"]
    t = torch.arange(T, device=table.device)
    at = s["pos"].long()[:, None] + t
    there = (t < s["count"][:, None]) & (at // PAGE < table.shape[1])
    page = table.gather(1, (at // PAGE).clamp(max=table.shape[1] - 1)).long()
    return page, at % PAGE, there


def _read(s):
    c, t = s["case"], TYPES[s["case"]["dtype"]]
    page, slot, there = _places(s)
    out = []
    for codes, e in ((s["kp"], s["ks"]), (s["vp"], s["vs"])):
        x = _values(codes[page, :, slot], e.view(torch.uint8)[page, :, slot])   # [R][T][H][dh]
        out.append(torch.where(there[..., None], x.flatten(-2), 0.0).to(t))
    return tuple(out)


def _append(s):
    c = s["case"]
    page, slot, there = _places(s)
    for x, codes, e in ((s["k"], s["kp"], s["ks"]), (s["v"], s["vp"], s["vs"])):
        q, sc = _quantise(x.float().unflatten(-1, (c["H"], c["dh"])))
        codes[page[there], :, slot[there]] = q[there]
        e.view(torch.uint8)[page[there], :, slot[there]] = sc[there]
    return _read(s) + _state(s)


def _state(s):
    return s["kp"], s["vp"], s["ks"].view(torch.uint8), s["vs"].view(torch.uint8)


def _attention(s):
    c = s["case"]
    R, S, Hq, H, dh = (c[n] for n in ("R", "S", "Hq", "H", "dh"))
    ids = s["table"].long()
    read = lambda codes, e: _values(codes[ids], e.view(torch.uint8)[ids])  # [R][W][H][64][dh]
    k = read(s["kp"], s["ks"]).permute(0, 2, 4, 1, 3).reshape(R, H, dh, -1)
    v = read(s["vp"], s["vs"]).permute(0, 2, 1, 3, 4).reshape(R, H, -1, dh)
    q = s["q"].float().view(R, S, H, Hq // H, dh).permute(0, 2, 1, 3, 4).reshape(R, H, -1, dh)
    a = (q * dh ** -0.5) @ k                                     # [R][H][S * group][tokens]
    last = s["lens"].long()[:, None].expand(R, S)
    if s["qpos"] is not None:
        last = torch.minimum(last, s["qpos"].long()[:, None] + 1 + torch.arange(S, device=q.device))
    last = last[:, :, None].expand(R, S, Hq // H).reshape(R, 1, -1, 1)
    a.masked_fill_(torch.arange(a.shape[-1], device=q.device) >= last, -math.inf)
    a = (a - a.amax(-1, keepdim=True)).exp_()
    o = (a @ v) / a.sum(-1, keepdim=True)
    return o.view(R, H, S, Hq // H, dh).permute(0, 2, 1, 3, 4).reshape(R, S, Hq * dh).to(s["q"].dtype)


# ------------------------------------------------------------------------------ the pass

def _own(s):
    import paper_2312_04429_amd as nv
    c = s["case"]
    if c["kind"] == "rope":
        q, k = _qk(s)
        return nv.nv_op_qk_rope(q, k, c["dh"], s["pos"], s["axes"], s["freqs"], q_weight=s["wq"],
                                k_weight=s["wk"], eps=EPS if c["norm"] else None,
                                halves=c["halves"])
    pages = (s["kp"], s["vp"], s["ks"], s["vs"])
    if c["kind"] == "attention":
        return nv.nv_op_attention_kv4(s["q"], pages, s["table"], s["lens"], c["dh"] ** -0.5,
                                      qpos=s["qpos"])
    if c["kind"] == "append":
        nv.nv_op_kv4_append(s["k"], s["v"], pages, s["table"], s["pos"], s["count"])
    out = nv.nv_op_kv4_read(pages, s["table"], s["pos"], c["T"], s["count"], TYPES[c["dtype"]])
    return out + _state(s) if c["kind"] == "append" else out


def run(s):
    if own:
        return _own(s)
    return {"rope": _rope, "append": _append, "read": _read,
            "attention": _attention}[s["case"]["kind"]](s)


# ------------------------------------------------------------------------------ its work

def work(case):
    c, k = case, case["kind"]
    H, dh = c["H"], c["dh"]
    if k == "rope":
        n = c["R"] * c["S"] * (c["Hq"] + H) * dh
        return dict(bytes=4.0 * n + 4.0 * c["R"] * c["S"] * len(c["axes"].split(",")),
                    flops=(8.0 if c["norm"] else 3.0) * n)
    kept = dh / 2 + -(-dh // BLOCK)  # bytes of a token's head in the cache
    if k in ("append", "read"):  # lengths are spread evenly below the longest; all of T is returned
        tokens = c["R"] * (c["T"] if c["T"] < 4 else 0.625 * c["T"])
        new = 4.0 * tokens * H * dh if k == "append" else 0.0
        return dict(bytes=new + 2.0 * tokens * H * kept + 4.0 * c["R"] * c["T"] * H * dh,
                    flops=2.0 * tokens * H * dh * (2 if k == "append" else 1))
    R, S, L = c["R"], c["S"], c["L"]
    mean = L if L < 100 else L - (R - 1) / R * (L - max(S, L // 4)) / 2
    seen = mean - (S - 1) / 2 if c["causal"] else mean
    return dict(bytes=2.0 * R * mean * H * kept + 4.0 * R * S * c["Hq"] * dh,
                flops=4.0 * R * S * seen * c["Hq"] * dh)


# ------------------------------------------------------------------------------ float64

def _values64(codes, e):
    """Values by the definition of e2m1: sign, two exponent bits (bias 1), one mantissa bit."""
    n = torch.stack((codes % 16, codes // 16), -1).flatten(-2).long()
    ex, m = n // 2 % 4, (n % 2).double()
    v = torch.where(ex == 0, m / 2, (1 + m / 2) * torch.exp2(ex.double() - 1))
    v = torch.where(n >= 8, -v, v)
    s = torch.exp2(e.view(torch.uint8).double() - 127)
    return v * s.repeat_interleave(BLOCK, -1)[..., :v.shape[-1]]


def _quantised64(x):
    """The values that float64 x [..., dh] has in 4 bits: the smallest power of two 2^p with amax
    <= 6 * 2^p, then steps of 2^(exponent - 1), at least 1/2, ties to the even code."""
    out = torch.empty_like(x)
    for j in range(0, x.shape[-1], BLOCK):
        b = x[..., j:j + BLOCK]
        top = b.abs().amax(-1, keepdim=True)
        p = torch.ceil(torch.log2(top.clamp(min=2.0 ** -150) / 6))
        p = torch.where(top > 6 * torch.exp2(p), p + 1, p)
        p = torch.where(top <= 6 * torch.exp2(p - 1), p - 1, p).clamp(min=-126)
        y = b / torch.exp2(p)
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1.0))) - 1)
        out[..., j:j + BLOCK] = torch.round(y / step) * step * torch.exp2(p)
    return out


def _rope64(x, w, s):
    c, dh = s["case"], s["case"]["dh"]
    out = torch.empty(*x.shape, dtype=torch.float64, device="cuda")
    for h in range(x.shape[-1] // dh):
        y = x[..., h * dh:(h + 1) * dh].double()
        if c["norm"]:
            y = y / (y.square().mean(-1, keepdim=True) + EPS).sqrt() * w.double()
        z = y.clone()
        at = 0
        for n, a in enumerate(s["axes"]):
            for i in range(a // 2):
                angle = s["pos"][..., n].double() * THETA ** (-2.0 * i / a)
                u, v = (at + i, at + a // 2 + i) if c["halves"] else (at + 2 * i, at + 2 * i + 1)
                z[..., u] = y[..., u] * angle.cos() - y[..., v] * angle.sin()
                z[..., v] = y[..., u] * angle.sin() + y[..., v] * angle.cos()
            at += a
        out[..., h * dh:(h + 1) * dh] = z
    return out


def exact(case, seed):
    s, c = prepare(case, seed), case
    H, dh = c["H"], c["dh"]
    if c["kind"] == "rope":
        q, k = _qk(s)
        return _rope64(q, s["wq"], s), _rope64(k, s["wk"], s)
    if c["kind"] in ("append", "read"):
        out = []
        table, pos, count = (s[n].cpu() for n in ("table", "pos", "count"))
        for name in "kv":
            y = torch.zeros(c["R"], c["T"], H * dh, dtype=torch.float64, device="cuda")
            for r in range(c["R"]):
                n, first = int(count[r]), int(pos[r])
                if c["kind"] == "append":
                    x = s[name][r, :n].double().view(n, H, dh)
                    y[r, :n] = _quantised64(x).view(n, -1)
                    continue
                ids = table[r].long().cuda()
                held = _values64(s[name + "p"][ids], s[name + "s"].view(torch.uint8)[ids])
                held = held.transpose(1, 2).reshape(-1, H * dh)
                y[r, :n] = held[first:first + n]
            out.append(y)
        return tuple(out) if c["kind"] == "read" else (*out, None, None, None, None)
    R, S, Hq = c["R"], c["S"], c["Hq"]
    out = torch.zeros(R, S, Hq, dh, dtype=torch.float64, device="cuda")
    for r in range(R):
        n, ids = int(s["lens"][r]), s["table"][r].long()
        for h in range(H):
            k = _values64(s["kp"][ids, h], s["ks"].view(torch.uint8)[ids, h]).reshape(-1, dh)[:n]
            v = _values64(s["vp"][ids, h], s["vs"].view(torch.uint8)[ids, h]).reshape(-1, dh)[:n]
            for i in range(h * Hq // H, (h + 1) * Hq // H):
                a = s["q"][r].double().view(S, Hq, dh)[:, i] @ k.T / math.sqrt(dh)
                if c["causal"]:
                    see = n - S + torch.arange(S, device="cuda")
                    a.masked_fill_(torch.arange(n, device="cuda") > see[:, None], -math.inf)
                out[r, :, i] = torch.softmax(a, -1) @ v
    return out.view(R, S, Hq * dh)
