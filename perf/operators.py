"""The operators of self-attention with positions and with a cache, as cases that can be timed: the plain form of each in
elementary torch operations, and the calls of `paper_2203_15952_amd.binding` that a program makes instead.

A case is a dict of plain values; its `kind` says what it stands for:

  rotate         queries and keys normalised per head and rotated by their frame's position, as a serving step does it
  rotate_train   the same and its backward, as a training step does it
  store          keys and values of new frames quantized into the cache of their streams, and read back
  attend         attention of the new frames of every stream over what the cache holds of it

A projected row holds `heads` queries, `kv_heads` keys and `kv_heads` values of `dh` columns each.  Streams stand at
different lengths, and in a ragged batch some bring fewer new frames than others, or none: both follow from the case alone.
Values: queries, keys and values N(0, 1), the queries times `sharp`, one column in sixteen of the keys four times larger (such
columns are what makes a cache's scales matter), gains about 1, upstream gradients N(0, 0.01).  Everything is drawn on the
GPU from the seed.
"""
import math

import torch

own = False

HALVES, PAIRS = 0, 1
FILL = 4096          # history frames that are drawn and quantized at a time


def listed():
    return [
        # one new frame of eight streams, far into their recordings: a few kilobytes, latency is all there is
        dict(name="rotate_frame", kind="rotate", B=8, T=1, heads=8, kv_heads=8, dh=64, rot=64, pairing=HALVES, norm=True,
             base=10000.0, first=200000),
        # the batch of the encoder-layer configuration, training
        dict(name="rotate_train_batch", kind="rotate_train", B=32, T=400, heads=8, kv_heads=8, dh=64, rot=64, pairing=HALVES,
             norm=True, base=10000.0, first=0),
        # the narrow model, heads of 36 columns, neighbouring columns paired, ragged length
        dict(name="rotate_train_narrow", kind="rotate_train", B=24, T=417, heads=4, kv_heads=4, dh=36, rot=36, pairing=PAIRS,
             norm=True, base=10000.0, first=0),
        # the large training batch, keys and values shared by two heads each, half of every head rotated
        dict(name="rotate_train_large", kind="rotate_train", B=128, T=512, heads=8, kv_heads=4, dh=64, rot=32, pairing=HALVES,
             norm=True, base=10000.0, first=0),
        # one new frame of sixty-four streams into an int8 cache and back
        dict(name="store_frame", kind="store", streams=64, T=1, capacity=512, heads=8, kv_heads=8, dh=64, bits=8, shortest=100,
             longest=2000, ragged=False),
        # a narrow model's utterances, ragged, int4, into a cache that they go round in
        dict(name="store_narrow_int4", kind="store", streams=24, T=417, capacity=448, heads=4, kv_heads=4, dh=36, bits=4, shortest=0,
             longest=900, ragged=True),
        # long recordings taken in at once, int8
        dict(name="store_long", kind="store", streams=16, T=4096, capacity=8192, heads=8, kv_heads=8, dh=64, bits=8, shortest=0,
             longest=4096, ragged=False),
        # one frame of one stream with the paper's limited left context: latency
        dict(name="attend_window", kind="attend", streams=1, T=1, capacity=128, heads=8, kv_heads=8, dh=64, bits=8, shortest=777,
             longest=777, left=65, right=0, ragged=False, sharp=1.0),
        # chunks of a streaming encoder: a little right context inside the chunk, ragged
        dict(name="attend_chunks", kind="attend", streams=32, T=16, capacity=512, heads=4, kv_heads=4, dh=36, bits=4, shortest=0,
             longest=1500, left=256, right=3, ragged=True, sharp=2.0),
        # one frame each over long histories, int8
        dict(name="attend_frame_long", kind="attend", streams=16, T=1, capacity=16384, heads=8, kv_heads=8, dh=64, bits=8, shortest=4000,
             longest=16000, left=-1, right=0, ragged=False, sharp=2.0),
        # one frame each, keys and values shared by four heads, wide heads, int4, full caches
        dict(name="attend_grouped_int4", kind="attend", streams=32, T=1, capacity=16384, heads=32, kv_heads=8, dh=128, bits=4,
             shortest=12000, longest=30000, left=-1, right=0, ragged=False, sharp=2.0),
        # a chunk of every stream over a long history: many queries for each key
        dict(name="attend_chunk_long", kind="attend", streams=8, T=128, capacity=8192, heads=8, kv_heads=8, dh=64, bits=8, shortest=5000,
             longest=8000, left=-1, right=0, ragged=False, sharp=2.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate_train", "rotate_train", "store", "store", "attend", "attend", "attend"])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 4])
    dh = rng.choice([64, 64, 128, 32, 36, 4 * rng.randint(2, 32), rng.randint(5, 128)])
    if kind.startswith("rotate"):
        rot = dh // 2 * 2 if rng.random() < 0.6 else 2 * rng.randint(1, dh // 2)
        tokens = _log(rng, 1, max(1, min(65536, 65536 * 1024 // ((heads + 2 * kv) * dh))))
        T = _log(rng, 1, min(tokens, 4096))
        return dict(kind=kind, B=max(1, tokens // T), T=T, heads=heads, kv_heads=kv, dh=dh, rot=rot, pairing=rng.choice([HALVES, PAIRS]),
                    norm=rng.random() < 0.8, base=rng.choice([10000.0, 500000.0]), first=rng.choice([0, _log(rng, 1, 1000000)]))
    capacity = 64 * _log(rng, 1, 256)
    c = dict(kind=kind, capacity=capacity, heads=heads, kv_heads=kv, dh=dh, bits=rng.choice([8, 8, 4, 4, rng.randint(2, 8)]),
             ragged=rng.random() < 0.4)
    c["shortest"] = rng.choice([0, _log(rng, 1, capacity)])
    c["longest"] = c["shortest"] + _log(rng, 1, 2 * capacity)
    if kind == "store":
        c["T"] = _log(rng, 1, min(4096, capacity))
        c["streams"] = _log(rng, 1, max(1, min(64, 65536 * 1536 // (c["T"] * (heads + 2 * kv) * dh), (1 << 26) // (capacity * kv))))
        return c
    c["T"] = _log(rng, 1, min(128, capacity))
    most = min(64, (1 << 30) // (capacity * kv * dh), 8 * 128 * 8192 * 512 // (c["T"] * capacity * heads * dh))
    c["streams"] = _log(rng, 1, max(1, most))
    c.update(left=rng.choice([-1, -1, _log(rng, 1, capacity)]), right=rng.choice([0, 0, 3, -1]), sharp=rng.choice([1.0, 2.0]))
    return c


# ---- what follows from a case alone ------------------------------------------------------------------------


def _lengths(c):
    """Frames that every stream has behind it."""
    return [c["shortest"] + int((c["longest"] - c["shortest"]) * ((b * 0.6180339887498949) % 1.0)) for b in range(c["streams"])]


def _counts(c):
    """New frames that every stream brings."""
    return [(7 * b + 3) % (c["T"] + 1) if c["ragged"] else c["T"] for b in range(c["streams"])]


def _held(c, L, n):
    """The first frame that a stream's cache holds after n more."""
    return max(0, L + n - c["capacity"])


def _columns(c):
    return (c["heads"] + 2 * c["kv_heads"]) * c["dh"]


def _container_bits(c):
    return 4 if c["bits"] <= 4 else 8


# ---- the plain forms ---------------------------------------------------------------------------------------


def _split(c, rows):
    """[R, columns] -> queries [R, heads, dh], keys and values [R, kv_heads, dh]."""
    q, k = c["heads"] * c["dh"], c["kv_heads"] * c["dh"]
    return (rows[:, :q].unflatten(1, (c["heads"], c["dh"])), rows[:, q:q + k].unflatten(1, (c["kv_heads"], c["dh"])),
            rows[:, q + k:].unflatten(1, (c["kv_heads"], c["dh"])))


def _angles(c, first):
    frames = (first[:, None] + torch.arange(c["T"], device="cuda")).reshape(-1).double()
    rate = c["base"] ** (-2.0 * torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64) / c["rot"])
    angle = frames[:, None, None] * rate
    return torch.cos(angle).float(), torch.sin(angle).float()


def _turn(c, x, cos, sin):
    """x [R, h, dh] with its first rot columns rotated."""
    r = c["rot"]
    if c["pairing"] == HALVES:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., r:]], -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., r:]], -1)


def _plain_rotate(s):
    c = s["case"]
    cos, sin = _angles(c, s["first"])
    q, k, v = _split(c, s["qkv"])
    parts, scaled = [], []
    for x, gain in ((q, s["gain_q"]), (k, s["gain_k"])):
        if c["norm"]:
            r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + s["eps"])
            x = x * r
            scaled.append((x, r))
            x = x * gain
        parts.append(_turn(c, x, cos, sin).flatten(1))
    out = torch.cat(parts + [v.flatten(1)], 1)
    if c["kind"] == "rotate":
        return dict(out=out)
    dq, dk, dv = _split(c, s["dout"])
    back, gains = [], []
    for i, (g, gain) in enumerate(((dq, s["gain_q"]), (dk, s["gain_k"]))):
        g = _turn(c, g, cos, -sin)
        if c["norm"]:
            x, r = scaled[i]
            gains.append((g * x).double().sum((0, 1)).float())
            g = g * gain
            g = r * (g - x * (g * x).mean(-1, keepdim=True))
        back.append(g.flatten(1))
    grads = dict(out=out, dqkv=torch.cat(back + [dv.flatten(1)], 1))
    return grads | dict(dgain_q=gains[0], dgain_k=gains[1]) if c["norm"] else grads


def _quantize(x, bits):
    """Fig. 2 of the paper over the last axis, every operation one float32 rounding: codes as float32, scales."""
    qmax = float(2 ** (bits - 1) - 1)
    top = x.abs().amax(-1, keepdim=True)
    scale = top / torch.full_like(top, qmax)                     # a divide: a number on the host would be a reciprocal's product
    t = torch.where(scale == 0, torch.zeros_like(x), x / scale)
    return torch.clamp(torch.floor(t + 0.5), -qmax, qmax), scale.squeeze(-1)


def _plain_write(s, rows, T, length, count):
    """New frames' keys and values into the plain cache: codes [streams, capacity + 1, kv_heads, dh], scales without dh."""
    c = s["case"]
    t = torch.arange(T, device="cuda")
    new = t < count[:, None]
    keep = new & (t >= count[:, None] - c["capacity"])          # a later frame of this call takes the place of the others
    b = torch.arange(c["streams"], device="cuda")[:, None]
    slot = torch.where(keep, (length[:, None] + t) % c["capacity"], c["capacity"])   # what is not kept: a slot that nothing reads
    for name, x in zip(("k", "v"), _split(c, rows)[1:]):
        code, scale = _quantize(x.unflatten(0, (c["streams"], T)), c["bits"])
        s[name + "_codes"][b, slot] = code.to(torch.int8)
        s[name + "_scale"][b, slot] = scale


def _plain_store(s):
    c = s["case"]
    _plain_write(s, s["qkv"], c["T"], s["length"], s["count"])
    t = torch.arange(c["T"], device="cuda")
    end = s["length"] + s["count"]
    frame = end[:, None] - c["T"] + t                            # the last T frames of every stream
    held = (frame >= 0) & (frame >= end[:, None] - c["capacity"])
    b, slot = torch.arange(c["streams"], device="cuda")[:, None], frame % c["capacity"]
    out = {}
    for name, key in (("k", "keys"), ("v", "values")):
        x = s[name + "_codes"][b, slot].float() * s[name + "_scale"][b, slot][..., None]
        out[key] = torch.where(held[..., None, None], x, torch.zeros_like(x)).flatten(0, 1).flatten(1)
    return out


def _plain_attend(s):
    c = s["case"]
    S, T, kv, dh = c["streams"], c["T"], c["kv_heads"], c["dh"]
    end = (s["length"] + s["count"])[:, None]
    slot = torch.arange(c["capacity"], device="cuda")
    frame = end - 1 - (end - 1 - slot) % c["capacity"]           # [S, capacity]: the frame that a slot holds, negative: none yet
    at = s["length"][:, None] + torch.arange(T, device="cuda")   # [S, T]: the frames of the queries
    seen = (frame >= 0)[:, None, :].expand(S, T, c["capacity"])
    if c["left"] >= 0:
        seen = seen & (frame[:, None, :] >= at[:, :, None] - c["left"])
    if c["right"] >= 0:
        seen = seen & (frame[:, None, :] <= at[:, :, None] + c["right"])
    k, v = (s[n + "_codes"][:, :-1].float() * s[n + "_scale"][:, :-1, :, None] for n in ("k", "v"))
    k, v = k.permute(0, 2, 3, 1).contiguous(), v.permute(0, 2, 1, 3).contiguous()   # [S, kv, dh, capacity], [S, kv, capacity, dh]
    group = c["heads"] // kv
    q = _split(c, s["qkv"])[0].view(S, T, kv, group, dh).permute(0, 2, 1, 3, 4).reshape(S, kv, T * group, dh)
    score = torch.matmul(q, k) / math.sqrt(dh)                   # [S, kv, T * group, capacity]
    seen = seen[:, None, :, None, :].expand(S, 1, T, group, c["capacity"]).reshape(S, 1, T * group, c["capacity"])
    score = torch.where(seen, score, torch.full_like(score, -math.inf))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    ctx = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    ctx = ctx.view(S, kv, T, group, dh).permute(0, 2, 1, 3, 4).reshape(S * T, c["heads"] * dh)
    new = (torch.arange(T, device="cuda") < s["count"][:, None]).reshape(-1, 1)
    return dict(ctx=torch.where(new, ctx, s["ctx"]))             # the rows of frames that a stream did not bring stay as they are


# ---- inputs ------------------------------------------------------------------------------------------------


def _rows(c, gen, n):
    rows = torch.randn((n, _columns(c)), device="cuda", generator=gen)
    k = c["heads"] * c["dh"]
    rows[:, k:k + c["kv_heads"] * c["dh"]:16] *= 4.0
    rows[:, :k] *= c.get("sharp", 1.0)
    return rows


def _rotate_inputs(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    M = c["B"] * c["T"]
    gain = 1.0 + 0.2 * torch.randn((2, c["dh"]), device="cuda", generator=gen)
    s = dict(case=c, eps=1e-6, qkv=_rows(c, gen, M), gain_q=gain[0].clone(), gain_k=gain[1].clone(),
             first=c["first"] + 131 * torch.arange(c["B"], device="cuda") % 1009 if c["first"] else torch.zeros(c["B"], dtype=torch.int64, device="cuda"))
    if c["kind"] == "rotate_train":
        s["dout"] = torch.randn((M, _columns(c)), device="cuda", generator=gen) * 0.1
    return s


def _history(c, gen):
    """The rows of what the streams have behind them, as far as a cache can hold it: (rows, frames each, length, count) at a time."""
    L = torch.tensor(_lengths(c), dtype=torch.int64, device="cuda")
    start = (L - c["capacity"]).clamp(min=0)
    longest = max(min(n, c["capacity"]) for n in _lengths(c))
    step = max(1, min(FILL, (1 << 28) // (c["streams"] * _columns(c))))
    for at in range(0, longest, step):
        T = min(step, longest - at)
        yield _rows(c, gen, c["streams"] * T), T, start + at, (L - start - at).clamp(0, T).to(torch.int32)


def _cache_inputs(c, gen):
    s = dict(case=c, length=torch.tensor(_lengths(c), dtype=torch.int64, device="cuda"),
             count=torch.tensor(_counts(c), dtype=torch.int32, device="cuda"))
    shape = (c["streams"], c["capacity"] + 1, c["kv_heads"])
    for name in ("k", "v"):
        s[name + "_codes"] = torch.zeros((*shape, c["dh"]), dtype=torch.int8, device="cuda")
        s[name + "_scale"] = torch.zeros(shape, device="cuda")
    return s


def prepare(case, seed):
    c = case
    if c["kind"].startswith("rotate"):
        s = _rotate_inputs(c, seed)
        if own:
            from paper_2203_15952_amd import binding as B
            s["spec"] = B.QkNormRotate(c["heads"], c["kv_heads"], c["dh"], rot=c["rot"], base=c["base"], norm=c["norm"], eps=s["eps"],
                                       pairing=B.AQT_ROTATE_HALVES if c["pairing"] == HALVES else B.AQT_ROTATE_PAIRS,
                                       gamma_q=s["gain_q"] if c["norm"] else None, gamma_k=s["gain_k"] if c["norm"] else None)
            s["out"] = torch.empty_like(s["qkv"])
            if c["kind"] == "rotate_train":
                s["dqkv"] = torch.empty_like(s["qkv"])
                s["ws"] = B.workspace(B.aqt_workspace_bytes(B.AQT_OP_QK_NORM_ROTATE_BWD, c["B"] * c["T"], c["dh"], 1))
        return s
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    if own:
        from paper_2203_15952_amd import binding as B
        s = dict(case=c, cache=B.KvCache(c["streams"], c["capacity"], c["kv_heads"], c["dh"], c["bits"]),
                 count=torch.tensor(_counts(c), dtype=torch.int32, device="cuda"), status=B.new_status())
        for rows, T, length, count in _history(c, gen):
            s["cache"].length.copy_(length)
            B.aqt_cache_append(rows, s["cache"], T, c["heads"], count=count, dev_status=s["status"])
        s["cache"].length.copy_(torch.tensor(_lengths(c), dtype=torch.int64))
    else:
        s = _cache_inputs(c, gen)
        for rows, T, length, count in _history(c, gen):
            _plain_write(s, rows, T, length, count)
    s["qkv"] = _rows(c, gen, c["streams"] * c["T"])
    if c["kind"] == "attend":
        s["ctx"] = torch.zeros((c["streams"] * c["T"], c["heads"] * c["dh"]), device="cuda")
        if own:                                                  # the new frames are in the cache before they are attended to
            B.aqt_cache_append(s["qkv"], s["cache"], c["T"], c["heads"], count=s["count"], dev_status=s["status"])
            s["ws"] = B.workspace(B.aqt_attention_cached_workspace_bytes(s["cache"], c["T"], c["heads"]))
        else:
            _plain_write(s, s["qkv"], c["T"], s["length"], s["count"])
    elif own:
        n = (c["streams"] * c["T"], c["kv_heads"] * c["dh"])
        s.update(keys=torch.empty(n, device="cuda"), values=torch.empty(n, device="cuda"))
    return s


def run(s):
    c = s["case"]
    if own:
        from paper_2203_15952_amd import binding as B
        if c["kind"].startswith("rotate"):
            out = B.aqt_qk_norm_rotate_fwd(s["qkv"], c["B"], c["T"], s["spec"], first=s["first"], out=s["out"])
            if c["kind"] == "rotate":
                return dict(out=out)
            dqkv, dq, dk = B.aqt_qk_norm_rotate_bwd(s["qkv"], s["dout"], c["B"], c["T"], s["spec"], first=s["first"], dqkv=s["dqkv"],
                                                    ws=s["ws"])
            grads = dict(out=out, dqkv=dqkv)
            return grads | dict(dgain_q=dq, dgain_k=dk) if c["norm"] else grads
        if c["kind"] == "store":
            B.aqt_cache_append(s["qkv"], s["cache"], c["T"], c["heads"], count=s["count"], dev_status=s["status"])
            keys, values = B.aqt_cache_read(s["cache"], c["T"], pending=c["T"], count=s["count"], keys=s["keys"], values=s["values"])
            return dict(keys=keys, values=values)
        ctx, _ = B.aqt_attention_cached_fwd(s["qkv"], s["cache"], c["T"], c["heads"], left=c["left"], right=c["right"], count=s["count"],
                                            ctx=s["ctx"], ws=s["ws"])
        return dict(ctx=ctx)
    if c["kind"].startswith("rotate"):
        return _plain_rotate(s)
    return _plain_store(s) if c["kind"] == "store" else _plain_attend(s)


def work(case):
    c = case
    if c["kind"].startswith("rotate"):
        M = c["B"] * c["T"]
        turned = M * (c["heads"] + c["kv_heads"]) * c["dh"]
        if c["kind"] == "rotate":
            return dict(bytes=8 * M * _columns(c), flops=8 * turned)
        return dict(bytes=16 * M * _columns(c), flops=24 * turned)
    frame = 2 * c["kv_heads"] * (c["dh"] * _container_bits(c) / 8 + 4)     # keys and values of one frame in the cache
    if c["kind"] == "store":
        new = sum(min(n, c["capacity"]) for n in _counts(c))
        out = c["streams"] * c["T"] * 2 * c["kv_heads"] * c["dh"] * 4
        return dict(bytes=new * (2 * c["kv_heads"] * c["dh"] * 4 + frame) + out, flops=new * 2 * c["kv_heads"] * c["dh"] * 4)
    read = pairs = rows = 0
    for L, n in zip(_lengths(c), _counts(c)):
        lo_all, hi_all, old = None, None, _held(c, L, n)
        for t in range(n):
            lo = max(old, L + t - c["left"]) if c["left"] >= 0 else old
            hi = min(L + n - 1, L + t + c["right"]) if c["right"] >= 0 else L + n - 1
            if hi >= lo:
                pairs += hi - lo + 1
                lo_all, hi_all = min(lo, lo if lo_all is None else lo_all), max(hi, hi if hi_all is None else hi_all)
        read += 0 if lo_all is None else hi_all - lo_all + 1
        rows += n
    return dict(bytes=read * frame + rows * 8 * c["heads"] * c["dh"], flops=4 * pairs * c["heads"] * c["dh"])


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------


def _exact_rotate(c, seed):
    s = _rotate_inputs(c, seed)
    H, G, d, r, M = c["heads"], c["kv_heads"], c["dh"], c["rot"], c["B"] * c["T"]
    rows = s["qkv"].double().view(M, H + 2 * G, d)
    frame = torch.repeat_interleave(s["first"].double(), c["T"]) + torch.arange(c["T"], device="cuda").double().repeat(c["B"])
    i = torch.arange(r // 2, device="cuda").double()
    turn = torch.polar(torch.ones((M, r // 2), dtype=torch.float64, device="cuda"), torch.outer(frame, torch.exp(-2.0 * i / r * math.log(c["base"]))))
    gain = torch.cat([s["gain_q"].double().expand(H, d), s["gain_k"].double().expand(G, d)])

    def rotated(x, by):
        y = x.clone()
        first, second = (slice(0, r // 2), slice(r // 2, r)) if c["pairing"] == HALVES else (slice(0, r, 2), slice(1, r, 2))
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * by[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        return y

    x = rows[:, :H + G]
    n = x / ((x ** 2).sum(-1, keepdim=True) / d + s["eps"]).sqrt() if c["norm"] else x
    out = rows.clone()
    out[:, :H + G] = rotated(n * gain if c["norm"] else n, turn)
    if c["kind"] == "rotate":
        return dict(out=out.view(M, -1))
    back = s["dout"].double().view(M, H + 2 * G, d).clone()
    g = rotated(back[:, :H + G], turn.conj())
    res = dict(out=out.view(M, -1), dqkv=back.view(M, -1))
    if c["norm"]:
        by_head = (g * n).sum(0)
        res.update(dgain_q=by_head[:H].sum(0), dgain_k=by_head[H:].sum(0))
        u = g * gain
        # y = x / rms: dx = (u - n <u, n> / d) / rms, and 1 / rms = n / x
        g = (u - n * ((u * n).sum(-1, keepdim=True) / d)) / ((x ** 2).sum(-1, keepdim=True) / d + s["eps"]).sqrt()
    back[:, :H + G] = g
    return res


def _exact_frames(c, seed):
    """Keys and values of every stream as the cache holds them after the call, in 64 bits: [frames, kv_heads, dh] each, with the
    first frame's number, and the queries."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    L, n = _lengths(c), _counts(c)
    H, G, d = c["heads"], c["kv_heads"], c["dh"]
    parts = [[] for _ in L]
    for rows, T, length, count in _history(c, gen):
        rows = rows.view(c["streams"], T, -1)
        for b, m in enumerate(count.tolist()):
            parts[b].append(rows[b, :m, H * d:])
    new = _rows(c, gen, c["streams"] * c["T"]).view(c["streams"], c["T"], -1)
    for b in range(c["streams"]):
        kv = torch.cat(parts[b] + [new[b, :n[b], H * d:]])[-c["capacity"]:].view(-1, 2 * G, d)
        qmax = 2 ** (c["bits"] - 1) - 1
        top = kv.abs().max(-1).values
        scale = top / torch.full_like(top, qmax)                 # the quantizer is defined by its float32 roundings
        code = torch.floor(kv / scale[..., None] + 0.5).nan_to_num(0.0).clamp(-qmax, qmax).double()
        kv = code * scale[..., None].double()
        yield b, L[b] + n[b] - kv.shape[0], kv[:, :G], kv[:, G:], new[b, :, :H * d].view(c["T"], H, d).double()


def exact(case, seed):
    c = case
    if c["kind"].startswith("rotate"):
        return _exact_rotate(c, seed)
    S, T, G, d = c["streams"], c["T"], c["kv_heads"], c["dh"]
    L, n = _lengths(c), _counts(c)
    if c["kind"] == "store":
        keys, values = (torch.zeros((S, T, G * d), dtype=torch.float64, device="cuda") for _ in range(2))
        for b, _, k, v, _ in _exact_frames(c, seed):
            m = min(T, k.shape[0])
            if m:
                keys[b, T - m:], values[b, T - m:] = k[-m:].flatten(1), v[-m:].flatten(1)
        return dict(keys=keys.view(S * T, -1), values=values.view(S * T, -1))
    ctx = torch.zeros((S, T, c["heads"], d), dtype=torch.float64, device="cuda")
    for b, first, k, v, q in _exact_frames(c, seed):
        at = L[b] + torch.arange(T, device="cuda")
        frame = first + torch.arange(k.shape[0], device="cuda")
        off = frame[None] - at[:, None]
        hidden = (off < -c["left"] if c["left"] >= 0 else torch.zeros_like(off, dtype=torch.bool)) | (off > c["right"] if c["right"] >= 0 else False)
        for h in range(c["heads"]):
            g = h // (c["heads"] // G)
            z = (q[:n[b], h] @ k[:, g].T * d ** -0.5).masked_fill(hidden[:n[b]], -math.inf)
            ctx[b, :n[b], h] = torch.softmax(z, -1).nan_to_num(0.0) @ v[:, g]
    return dict(ctx=ctx.view(S * T, -1))
