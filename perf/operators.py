"""What the operators around the quantised KV cache are timed on, with their plain forms.

A case is one pass of one of these operators:

  table   cos/sin of a chunk with scaled frequencies, for the rotated part of a head (rotary_table)
  rotate  the rotation of a chunk's queries or keys, or its transpose (rotary_apply)
  append  rotation, and k and v quantised into the cache, with or without the q/k norm (rotary_kv_append_q8)
  read    frames of the cache read back as bf16 (kv_read_q8)
  attn    attention of a chunk's queries over the quantised window (window_attn_q8)

The cache holds e4m3 codes; every 32 neighbouring dims of a head share a power of two, an e8m0 byte.  Activations are
N(0, 1) per coordinate, as behind the q/k norm of a video DiT, keys times `k_scale` where attention is peaked.
"""

from __future__ import annotations

import math

import torch

own = False

BF16, F8, E8 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu
EPS = 1e-6
D = 128
BANDS = {128: (44, 42, 42), 96: (32, 32, 32), 64: (24, 20, 20), 32: (16, 8, 8)}   # dims of the time, row and column axis


def _case(name, op, heads, chunk_frames, grid_h, grid_w, ring, window, starts, **more):
    case = {"name": name, "op": op, "heads": heads, "chunk_frames": chunk_frames, "grid_h": grid_h, "grid_w": grid_w,
            "ring": ring, "window": window, "starts": starts, "sink": 0, "sink_attend": 0, "norm": False,
            "half": False, "rotated": D, "factor": 1.0, "trained": 0, "transposed": False, "k_scale": 1.0}
    case.update(more)
    return case


def listed():
    return [
        # table of a toy chunk: what a call costs when there is next to nothing to do
        _case("table_toy", "table", 1, 2, 8, 8, 2, 2, "4"),
        # table of a new chunk at 720p, far behind the 21 frames a model was trained on, time axis scaled by four
        _case("table_720p", "table", 1, 3, 45, 80, 3, 3, "120", factor=4.0, trained=21, rotated=96),
        # rotation of a toy layer's queries
        _case("rotate_toy", "rotate", 2, 2, 8, 8, 2, 2, "4", half=True),
        # backward pass of the rotation of a 40-head layer at 720p, halves of the first 96 dims
        _case("rotate_14b_back", "rotate", 40, 3, 45, 80, 3, 3, "9", half=True, rotated=96, transposed=True),
        # cache entries of a chunk behind the q/k norm, 1.3B class (12 heads, 30 x 52 tokens), halves
        _case("append_norm", "append", 12, 3, 30, 52, 21, 21, "18", norm=True, half=True),
        # the same without the norm for four streams at different fill levels, interleaved
        _case("append_streams4", "append", 12, 3, 30, 52, 21, 21, "0,6,12,18"),
        # a ragged share of a cache handed on: 391 tokens a frame, 5 heads, wrapped ring behind a sink
        _case("read_ragged", "read", 5, 2, 17, 23, 7, 6, "12,8", sink=2),
        # the whole window of a 40-head layer at 720p
        _case("read_14b", "read", 40, 3, 45, 80, 12, 12, "9"),
        # one new token a stream over up to 4096 cached ones
        _case("attn_token", "attn", 12, 1, 1, 1, 4096, 4096, "5000,1234,4095"),
        # two streams with sizes that divide nothing, sink and wrapped ring
        _case("attn_ragged", "attn", 5, 2, 17, 23, 7, 5, "12,9", sink=2, sink_attend=1, k_scale=4.0),
        # 3 sink + 6 recent frames, the operating point of long clips
        _case("attn_sink9", "attn", 12, 3, 30, 52, 6, 6, "120", sink=3, sink_attend=3),
        # the last chunk of a 21-frame clip, every frame attended: 32760 keys
        _case("attn_window21", "attn", 12, 3, 30, 52, 21, 21, "18"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _scores(case):
    starts = _starts(case)
    widest = max(_keys(case, s) for s in starts)
    return len(starts) * case["heads"] * case["chunk_frames"] * case["grid_h"] * case["grid_w"] * widest


def draw(rng):
    """One more case of the same operators and ranges."""
    most = {}
    for c in listed():
        w = work(c)
        most[c["op"]] = max(most.get(c["op"], 0), w["flops"] if c["op"] == "attn" else w["bytes"])
    scores = max(_scores(c) for c in listed() if c["op"] == "attn")
    while True:
        op = rng.choice(["table", "rotate", "append", "append", "read", "attn", "attn", "attn"])
        chunk_frames = rng.choice([1, 2, 3, 3, 4])
        grid_h, grid_w = _log_int(rng, 1, 45), _log_int(rng, 1, 80)
        if op == "attn" and rng.random() < 0.2:
            chunk_frames, grid_h, grid_w = 1, 1, 1
        tokens = grid_h * grid_w
        heads = _log_int(rng, 1, 40)
        # small frames come with longer windows
        ring = max(chunk_frames, _log_int(rng, 3, max(21, 4096 // tokens)))
        window = rng.choice([ring, rng.randint(chunk_frames, ring)])
        sink = rng.choice([0, 0, 1, 3])
        batch = 1 if op == "table" else rng.choice([1, 1, 2, 3, 4])
        last = 6 * ring + 120
        starts = [chunk_frames * rng.randint(0, last // chunk_frames) for _ in range(batch)]
        factor = rng.choice([1.0, 2.0, 8.0])
        case = _case("", op, heads, chunk_frames, grid_h, grid_w, ring, window, ",".join(str(s) for s in starts),
                     sink=sink, sink_attend=rng.randint(max(0, sink - 1), sink), norm=rng.random() < 0.5,
                     half=rng.random() < 0.5, rotated=rng.choice([128, 128, 96, 64, 32]), factor=factor,
                     trained=rng.choice([0, 21]) if factor > 1 else 0, transposed=op == "rotate" and rng.random() < 0.5,
                     k_scale=rng.choice([1.0, 1.0, 4.0]))
        del case["name"]
        w = work(case)
        if op in ("append", "read", "attn") and 2 * batch * (sink + ring) * tokens * heads * D > 5.0e8:   # bytes of a cache
            continue
        if op == "attn" and _scores(case) > scores:
            continue
        if (w["flops"] if op == "attn" else w["bytes"]) <= most[op]:
            return case


def _starts(case):
    return [int(s) for s in case["starts"].split(",")]


def _frames(case, start):
    """The frames that a chunk at `start` attends, in order."""
    hi = start + case["chunk_frames"]
    lo = max(0, hi - case["window"])
    return list(range(min(case["sink_attend"], lo))) + list(range(lo, hi))


def _keys(case, start):
    return len(_frames(case, start)) * case["grid_h"] * case["grid_w"]


def _slot(case, frame):
    return frame if frame < case["sink"] else case["sink"] + (frame - case["sink"]) % case["ring"]


def _read_frames(case):
    """How many frames a read takes, and the first one of each stream: those that its window still holds."""
    n = min(min(case["window"], s + case["chunk_frames"]) for s in _starts(case))
    return n, [s + case["chunk_frames"] - n for s in _starts(case)]


def _normal(gen, dims, scale=1.0):
    x = torch.empty(dims, dtype=torch.float32, device="cuda").normal_(generator=gen)
    return (x * scale if scale != 1.0 else x).to(BF16)


# ------------------------------------------------------------------ plain forms

def _frequencies(case):
    """Scaled frequencies of the rotated pairs of each axis, float64."""
    t, h, w = (10000.0 ** (-torch.arange(0, dims, 2, dtype=torch.float64, device="cuda") / dims)
               for dims in BANDS[case["rotated"]])
    keep = ((case["trained"] * t / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)   # none if trained is 0
    return t * (keep + (1.0 - keep) / case["factor"]), h, w


def _magnitude(case):
    return 1.0 + 0.1 * math.log(case["factor"])


def _plain_table(case, start):
    omega = _frequencies(case)
    fc, gh, gw = case["chunk_frames"], case["grid_h"], case["grid_w"]
    n = torch.arange(fc * gh * gw, device="cuda")
    pos = torch.stack([start + n // (gh * gw), n // gw % gh, n % gw]).double()
    angle = torch.cat([pos[a][:, None] * omega[a] for a in range(3)], dim=1)
    m = _magnitude(case)
    return (m * angle.cos()).float(), (m * angle.sin()).float()


def _rotate(case, x, cos, sin):
    """The rotation of x [B, L, H, 128] in float32: products and sums rounded one by one."""
    r, c, s = case["rotated"], cos[:, :, None], sin[:, :, None]
    if case["half"]:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * c - b * s, a * s + b * c, x[..., r:]], dim=-1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    y = torch.stack([a * c - b * s, a * s + b * c], dim=-1).flatten(-2)
    return torch.cat([y, x[..., r:]], dim=-1)


def _quantise(x):
    """Codes [.., 128] and scale bytes [.., 4] of float32 values."""
    blocks = x.unflatten(-1, (4, 32))
    top = blocks.abs().amax(-1)
    bits = top.view(torch.int32)
    byte = (((bits + 0x1FFFFF) >> 23) - 8).clamp(min=3)     # least power of two with top <= 448 * 2^(byte - 127)
    byte = torch.where(bits >= 0x7F780000, 255, byte)       # not finite, or too large to be read as bf16
    inverse = ((254 - byte).clamp(min=0) << 23).view(torch.float32)
    codes = torch.where((byte == 255)[..., None], torch.zeros_like(blocks), blocks * inverse[..., None])
    return codes.flatten(-2).to(F8), byte.to(torch.uint8).view(E8)


def _decode(codes, scales):
    return (codes.float().unflatten(-1, (4, 32)) * scales.float()[..., None]).flatten(-2)


def _norm(x, gain):
    wide = x.flatten(-2)
    return (wide * (1.0 / (wide.square().mean(-1, keepdim=True) + EPS).sqrt()) * gain).view_as(x)


def _write(cache, scale, at, x):
    """Quantises x [B, F, T, H, 128] into the frames `at` of a cache."""
    codes, powers = _quantise(x)
    cache.view(torch.uint8)[at] = codes.view(torch.uint8)
    scale.view(torch.uint8)[at] = powers.view(torch.uint8)


def _plain_append(s):
    case = s["case"]
    q, k, v = (t.float() for t in s["qkv"])
    if case["norm"]:
        q, k = _norm(q, s["gain_q"]), _norm(k, s["gain_k"])
    q, k = _rotate(case, q, s["cos"], s["sin"]), _rotate(case, k, s["cos"], s["sin"])
    s["q_rot"].copy_(q)
    frames = (case["chunk_frames"], case["grid_h"] * case["grid_w"])
    at = (s["streams"], s["chunk_slots"])
    _write(s["cache_k"], s["scale_k"], at, k.unflatten(1, frames))
    _write(s["cache_v"], s["scale_v"], at, v.unflatten(1, frames))
    return s["q_rot"], s["cache_k"], s["scale_k"], s["cache_v"], s["scale_v"]


def _gather(cache, scale, streams, slots):
    """Frames [B, F] of a cache as float32 [B, F, T, H, 128]."""
    return _decode(cache.view(torch.uint8)[streams, slots].view(F8), scale.view(torch.uint8)[streams, slots].view(E8))


def _plain_attn(s):
    k = _gather(s["cache_k"], s["scale_k"], s["streams"], s["window_slots"]).flatten(1, 2)
    v = _gather(s["cache_v"], s["scale_v"], s["streams"], s["window_slots"]).flatten(1, 2)
    q = s["qkv"][0].float().transpose(1, 2)
    p = q @ k.permute(0, 2, 3, 1)
    p *= 1.0 / math.sqrt(D)
    if s["hidden"] is not None:
        p.masked_fill_(s["hidden"][:, None, None, :], -math.inf)
    p -= p.amax(-1, keepdim=True)
    p.exp_()
    out = (p @ v.transpose(1, 2)) / p.sum(-1, keepdim=True)
    return out.transpose(1, 2).to(BF16).contiguous()


# ------------------------------------------------------------------ the cases

def prepare(case, seed):
    """Activations of a chunk, the cache behind it, its table, buffers for the results, and the slots of its frames."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, starts = case["op"], _starts(case)
    batch, tokens = len(starts), case["grid_h"] * case["grid_w"]
    length = case["chunk_frames"] * tokens
    s = {"case": case, "starts": starts}
    if op == "table":
        s["starts"] = [starts[0] + 1 + int(seed) % 997]   # the seed moves the chunk along the clip
        s["cos"] = torch.empty((length, case["rotated"] // 2), dtype=torch.float32, device="cuda")
        s["sin"] = torch.empty_like(s["cos"])
    else:
        act = (batch, length, case["heads"], D)
        cache = (batch, case["sink"] + case["ring"], tokens, case["heads"], D)
        s["qkv"] = tuple(_normal(gen, act, scale) for scale in (1.0, case["k_scale"], 1.0))
        s["q_rot"] = torch.empty(act, dtype=BF16, device="cuda")
    if op in ("rotate", "append"):
        tables = [_plain_table(case, x) for x in sorted(set(starts), key=starts.index)]
        if len(tables) > 1:
            tables = [_plain_table(case, x) for x in starts]
        s["cos"], s["sin"] = (torch.stack(x).contiguous() for x in zip(*tables))
        s["stride"] = length * (case["rotated"] // 2) if len(tables) > 1 else 0
    if op in ("append", "read", "attn"):
        s["cache_k"], s["scale_k"] = _quantise(_normal(gen, cache, case["k_scale"]).float())
        s["cache_v"], s["scale_v"] = _quantise(_normal(gen, cache).float())
        s["streams"] = torch.arange(batch, device="cuda")[:, None]
    if op == "append":
        if case["norm"]:
            wide = case["heads"] * D
            s["gain_q"] = 1.0 + 0.2 * torch.empty(wide, device="cuda").normal_(generator=gen)
            s["gain_k"] = 1.0 + 0.2 * torch.empty(wide, device="cuda").normal_(generator=gen)
        s["chunk_slots"] = torch.tensor([[_slot(case, x + f) for f in range(case["chunk_frames"])] for x in starts],
                                        device="cuda")
    if op == "read":
        n, first = _read_frames(case)
        s["first"], s["frames"] = first, n
        s["window_slots"] = torch.tensor([[_slot(case, x + f) for f in range(n)] for x in first], device="cuda")
        s["out"] = [torch.empty((batch, n, tokens, case["heads"], D), dtype=BF16, device="cuda") for _ in range(2)]
    if op == "attn":
        frames = [_frames(case, x) for x in starts]
        n = max(len(f) for f in frames)
        padded = [[_slot(case, p) for p in f] + [0] * (n - len(f)) for f in frames]
        s["window_slots"] = torch.tensor(padded, device="cuda")
        hidden = torch.tensor([[i >= len(f) for i in range(n)] for f in frames], device="cuda")
        s["hidden"] = hidden.repeat_interleave(tokens, 1) if min(len(f) for f in frames) < n else None
        s["out"] = torch.empty(act, dtype=BF16, device="cuda")
    if own:
        import paper_2609_32518_b200 as U
        s["shape"] = U.Shape.make(batch, case["heads"], case["chunk_frames"], case["grid_h"], case["grid_w"],
                                  case["ring"], bands=BANDS[case["rotated"]])
        s["rope"] = U.Rope.make(half=case["half"], factor=(case["factor"], 1.0, 1.0), trained=(case["trained"], 0, 0),
                                beta=(1.0, 4.0), magnitude=_magnitude(case))
    return s


def run(s):
    case, op = s["case"], s["case"]["op"]
    if own:
        import paper_2609_32518_b200 as U
    if op == "table":
        if own:
            U.rotary_table(s["shape"], s["rope"], s["starts"][0], s["cos"], s["sin"])
            return s["cos"], s["sin"]
        return _plain_table(case, s["starts"][0])
    if op == "rotate":
        if own:
            U.rotary_apply(s["shape"], s["rope"], s["qkv"][0], s["cos"], s["sin"], s["q_rot"],
                           transposed=case["transposed"], table_stream_stride=s["stride"])
            return s["q_rot"]
        sin = -s["sin"] if case["transposed"] else s["sin"]
        return _rotate(case, s["qkv"][0].float(), s["cos"], sin).to(BF16)
    if op == "append":
        if own:
            q, k, v = s["qkv"]
            U.rotary_kv_append_q8(s["shape"], s["rope"], case["sink"], s["starts"], q, k, v, s["cos"], s["sin"],
                                  s["q_rot"], s["cache_k"], s["scale_k"], s["cache_v"], s["scale_v"],
                                  gain_q=s.get("gain_q"), gain_k=s.get("gain_k"), eps=EPS,
                                  table_stream_stride=s["stride"])
            return s["q_rot"], s["cache_k"], s["scale_k"], s["cache_v"], s["scale_v"]
        return _plain_append(s)
    if op == "read":
        if own:
            U.kv_read_q8(s["shape"], case["sink"], s["first"], s["frames"], s["cache_k"], s["scale_k"], s["cache_v"],
                         s["scale_v"], s["out"][0], s["out"][1])
            return s["out"]
        return [_gather(s[c], s[e], s["streams"], s["window_slots"]).to(BF16)
                for c, e in (("cache_k", "scale_k"), ("cache_v", "scale_v"))]
    if own:
        U.window_attn_q8(s["shape"], case["sink"], s["starts"], case["window"], case["sink_attend"], s["qkv"][0],
                         s["cache_k"], s["scale_k"], s["cache_v"], s["scale_v"], s["out"])
        return s["out"]
    return _plain_attn(s)


def work(case):
    """Bytes and operations of one pass: inputs read once, results and the chunk's cache entries written once."""
    starts, tokens = _starts(case), case["grid_h"] * case["grid_w"]
    length, wide = case["chunk_frames"] * tokens, case["heads"] * D
    pairs = case["rotated"] // 2
    table = 2 * length * pairs * 4
    if case["op"] == "table":
        # an angle, a sine and a cosine of each distinct (position, pair), about 50 operations in double
        t, h, w = (d // 2 for d in BANDS[case["rotated"]])
        return {"bytes": table, "flops": 50 * (t * case["chunk_frames"] + h * case["grid_h"] + w * case["grid_w"])}
    values = len(starts) * length * wide
    tables = len(set(starts)) * table
    if case["op"] == "rotate":
        return {"bytes": 4 * values + tables, "flops": 3.0 * values * case["rotated"] / D}
    if case["op"] == "append":
        # codes, a scale byte for 32 of them; a maximum, a product and a conversion for each
        return {"bytes": 10 * values + values // 16 + tables + (8 * wide if case["norm"] else 0),
                "flops": (2 * 3.0 + 2 * 3.0 + (2 * 4.0 if case["norm"] else 0.0)) * values}
    if case["op"] == "read":
        held = 2 * len(starts) * _read_frames(case)[0] * tokens * wide
        return {"bytes": 3 * held + held // 32, "flops": 1.0 * held}
    keys = sum(_keys(case, x) for x in starts)
    return {"bytes": 4 * values + 2 * keys * wide + keys * wide // 16, "flops": 4.0 * length * keys * wide}


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op, starts = case["op"], s["starts"]
    tokens = case["grid_h"] * case["grid_w"]

    def rotation(x, cos, sin):
        y = x.clone()
        half = case["rotated"] // 2
        for j in range(half):
            a, b = (j, j + half) if case["half"] else (2 * j, 2 * j + 1)
            c, d = cos[:, :, None, j], sin[:, :, None, j]
            y[..., a] = x[..., a] * c - x[..., b] * d
            y[..., b] = x[..., a] * d + x[..., b] * c
        return y

    def quantised(x):
        """The e4m3 value of each x / 2^e, and 2^e, of each block of 32."""
        b = x.reshape(*x.shape[:-1], 4, 32)
        top = b.abs().amax(-1)
        e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0)).clamp(min=-124)
        e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e)                       # log2 is not exact
        e = torch.where((e > -124) & (top <= 448.0 * torch.exp2(e - 1)), e - 1, e)
        y = b / torch.exp2(e)[..., None]
        _, exponent = torch.frexp(y)                                                 # |y| in [2^(exponent - 1), 2^exponent)
        step = torch.exp2((exponent - 1).clamp(min=-6).double() - 3)                 # three bits behind the leading one
        return (torch.round(y / step) * step).reshape(x.shape), torch.exp2(e)

    def held(cache, scale, b, frames, head=slice(None)):
        """Frames of stream b's cache [F, T, heads, 128], decoded."""
        slots = torch.tensor([_slot(case, p) for p in frames], device="cuda")
        c = cache[b].view(torch.uint8)[slots][:, :, head].contiguous().view(F8).double()
        e = scale[b].view(torch.uint8)[slots][:, :, head].contiguous().view(E8).double()
        return c * e.repeat_interleave(32, -1)

    if op == "table":
        cos, sin = [], []
        place = torch.arange(case["chunk_frames"] * tokens, device="cuda").double()
        position = (starts[0] + torch.floor(place / tokens),
                    torch.floor(torch.remainder(place, tokens) / case["grid_w"]), torch.remainder(place, case["grid_w"]))
        for axis, dims in enumerate(BANDS[case["rotated"]]):
            for i in range(dims // 2):
                w = math.pow(10000.0, -2.0 * i / dims)
                if axis == 0 and case["factor"] > 1.0:
                    turns = case["trained"] * w / math.tau
                    keep = min(1.0, max(0.0, (turns - 1.0) / 3.0)) if case["trained"] else 0.0
                    w = keep * w + (1.0 - keep) * w / case["factor"]
                cos.append(_magnitude(case) * torch.cos(position[axis] * w))
                sin.append(_magnitude(case) * torch.sin(position[axis] * w))
        return torch.stack(cos, 1), torch.stack(sin, 1)
    if op == "rotate":
        sign = -1.0 if case["transposed"] else 1.0
        return rotation(s["qkv"][0].double(), s["cos"].double(), sign * s["sin"].double())
    if op == "append":
        q, k, v = (t.double() for t in s["qkv"])
        if case["norm"]:
            q, k = (x / torch.sqrt((x * x).mean((2, 3), keepdim=True) + EPS) * g.double().view(1, 1, -1, D)
                    for x, g in ((q, s["gain_q"]), (k, s["gain_k"])))
        q, k = (rotation(x, s["cos"].double(), s["sin"].double()) for x in (q, k))
        out = [q]
        for x, cache, scale in ((k, "cache_k", "scale_k"), (v, "cache_v", "scale_v")):
            codes, powers = quantised(x)
            c, e = s[cache].double(), s[scale].double()
            for b, start in enumerate(starts):
                for f in range(case["chunk_frames"]):
                    c[b, _slot(case, start + f)] = codes[b, f * tokens:(f + 1) * tokens]
                    e[b, _slot(case, start + f)] = powers[b, f * tokens:(f + 1) * tokens]
            out += [c, e]
        return tuple(out)
    if op == "read":
        return [torch.stack([held(s[c], s[e], b, range(x, x + s["frames"])) for b, x in enumerate(s["first"])])
                for c, e in (("cache_k", "scale_k"), ("cache_v", "scale_v"))]
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    for b, start in enumerate(starts):
        for h in range(case["heads"]):
            k, v = (held(s[c], s[e], b, _frames(case, start), slice(h, h + 1)).reshape(-1, D)
                    for c, e in (("cache_k", "scale_k"), ("cache_v", "scale_v")))
            score = s["qkv"][0][b, :, h].double() @ k.t() / math.sqrt(D)
            out[b, :, h] = torch.softmax(score, -1) @ v
    return out
