"""Measured cases of the operators that a train step over packed documents needs beside a decoder's own.

  attend, attend_grad     causal attention inside the documents of a packed batch (one buffer of T rows, documents of any
                          length one behind the other, rows behind the last one left alone)
  rotary                  rotary positions: half-split and interleaved pairs, part of a head, tables for long contexts,
                          forward and transposed
  adamw                   one AdamW step over many tensors, moments in 32 bits or in 8 with a scale for 256 elements

Every operator has a plain form in elementary torch operations, a 64-bit definition written separately, and the calls a user
of the package makes.  Tensors are laid out as the package's kernels take them: q, k and v heads packed in one
[T, (heads + 2 kv_heads) * d] buffer, document bounds as int32 offsets on the device, parameters and moments in flat arenas.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
MAX_WORK = 2.0e9  # (query, key) pairs of all heads of a drawn attention case, at most
MAX_BAND = 3.6e9  # scores its plain form holds at a time, at most
MAX_CELLS = 1.3e8  # elements of a drawn case of the other operators, at most
BETA1, BETA2, ADAM_EPS, LR, DECAY = 0.9, 0.95, 1e-8, 1e-3, 0.1


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the smallest configuration's tokens as a few short documents: launch latency
        dict(name="packed_tiny", op="attend", T=256, heads=4, kv_heads=4, d=64, mean=48, limit=128, tail=0, mix=1),
        # a 124M decoder's batch of 8 x 1024 tokens, packed from short texts
        dict(name="packed_124m", op="attend", T=8192, heads=12, kv_heads=12, d=64, mean=300, limit=1024, tail=0, mix=2),
        # a 1B decoder's long-context batch: a few documents of thousands of tokens
        dict(name="packed_long", op="attend", T=16384, heads=16, kv_heads=8, d=128, mean=4000, limit=8192, tail=0, mix=3),
        # gradients: all query heads on one kv head, odd lengths, an odd buffer whose last rows are padding
        dict(name="packed_grad_ragged", op="attend_grad", T=1999, heads=6, kv_heads=1, d=64, mean=180, limit=700, tail=13, mix=4, rope=False),
        # gradients of a 1B decoder's batch of 4 x 2048 tokens, packed
        dict(name="packed_grad_1b", op="attend_grad", T=8192, heads=16, kv_heads=8, d=128, mean=500, limit=2048, tail=0, mix=5, rope=True),
        # gradients of the long-context batch
        dict(name="packed_grad_long", op="attend_grad", T=16384, heads=16, kv_heads=8, d=128, mean=4000, limit=8192, tail=0, mix=3, rope=True),
        # the smallest configuration's q and k heads, rotated where they lie
        dict(name="rotary_tiny", op="rotary", rows=256, heads=8, other=4, d=64, rot=64, style="half", dtype="bf16", inverse=False, span=128, build=False, inplace=True),
        # q and k heads of an 8B decoder's sequence inside its qkv rows
        dict(name="rotary_8b", op="rotary", rows=4096, heads=40, other=8, d=128, rot=128, style="half", dtype="bf16", inverse=False, span=4096, build=False, inplace=True),
        # gradients of a decoder that rotates part of a head in interleaved pairs, at the far end of a stretched context whose
        # tables are made anew
        dict(name="rotary_part", op="rotary", rows=8191, heads=16, other=1, d=80, rot=48, style="pairs", dtype="f32", inverse=True, span=131072, build=True, inplace=False),
        # the smallest configuration's tensors
        dict(name="adamw_tiny", op="adamw", layers=1, h=256, ffn=688, vocab=1024, q=256, kv=256, state=32, grad="f32", copy=True),
        # a 124M decoder's tensors, moments in 32 bits
        dict(name="adamw_124m", op="adamw", layers=12, h=768, ffn=2048, vocab=32000, q=768, kv=768, state=32, grad="f32", copy=True),
        # the same with moments in 8 bits and bf16 gradients
        dict(name="adamw_124m_8bit", op="adamw", layers=12, h=768, ffn=2048, vocab=32000, q=768, kv=768, state=8, grad="bf16", copy=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend_grad", "rotary", "adamw"])
    if op.startswith("attend"):
        c = dict(op=op, T=_log_int(rng, 1, 16384), heads=0, kv_heads=rng.choice([1, 2, 3, 4, 8, 12]), d=rng.choice([64, 128]),
                 mean=0, limit=0, tail=0, mix=rng.randrange(1000))
        c["heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 7])
        c["mean"] = _log_int(rng, 1, 8192)
        c["limit"] = max(1, min(c["T"], _log_int(rng, max(1, c["mean"] // 2), 8 * c["mean"])))
        c["tail"] = rng.choice([0, 0, rng.randrange(0, max(1, min(c["T"], 300)))])
        if op == "attend_grad":
            c["rope"] = rng.random() < 0.5
        while c["heads"] * _pairs(c) > MAX_WORK or c["heads"] * 2 * c["T"] * max(1, max(_lengths(c), default=1)) > MAX_BAND:
            c["T"] = c["T"] * 3 // 4
            c["limit"], c["tail"] = max(1, min(c["limit"], c["T"])), min(c["tail"], c["T"] // 2)
        return c
    if op == "rotary":
        d = rng.choice([64, 128, 80, 96, 2 * rng.randint(1, 160)])
        c = dict(op=op, rows=_log_int(rng, 1, 32768), heads=rng.choice([1, 2, 5, 8, 16, 40]), other=rng.choice([0, 1, 8]), d=d,
                 rot=rng.choice([d, d, 2 * rng.randint(1, d // 2)]), style=rng.choice(["half", "pairs"]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                 inverse=rng.random() < 0.4, span=_log_int(rng, 128, 131072), build=rng.random() < 0.3, inplace=rng.random() < 0.5)
        c["rows"] = max(1, min(c["rows"], 33554432 // ((c["heads"] + c["other"]) * d) // (2 if c["dtype"] == "f32" else 1)))
        return c
    kv = rng.choice([64, 128, 256])
    c = dict(op=op, layers=rng.randint(1, 12), h=_log_int(rng, 1, 1024), ffn=_log_int(rng, 1, 4096), vocab=_log_int(rng, 1, 32000),
             q=kv * rng.choice([1, 2, 4]), kv=kv, state=rng.choice([8, 32]), grad=rng.choice(["f32", "bf16"]), copy=rng.random() < 0.7)
    while _spans(c)[-1][1] > MAX_CELLS:
        c["layers"] = max(1, c["layers"] // 2)
        c["vocab"] = c["vocab"] * 3 // 4
    return c


def _lengths(c):
    """Lengths of the documents: log-normal about `mean`, at most `limit`, empty ones among them; the last is cut at T - tail."""
    rng, left, got = random.Random(c["mix"] * 7919 + c["T"]), c["T"] - c["tail"], []
    while left > 0:
        n = min(c["limit"], left, int(c["mean"] * math.exp(rng.gauss(-0.3, 0.8))))
        if rng.random() < 0.05:
            n = 0  # a text that the filter before left empty
        elif n == 0:
            n = 1
        got.append(n)
        left -= n
    return got


def _pairs(c):
    return sum(n * (n + 1) // 2 for n in _lengths(c))


def _tensors(c):
    """(elements, decay) of a decoder's tensors, in the order of the package's models."""
    h, n = c["h"], []
    n.append((c["vocab"] * h, DECAY))
    for _ in range(c["layers"]):
        n += [(h, 0.0), ((c["q"] + 2 * c["kv"]) * h, DECAY), (h * c["q"], DECAY), (h, 0.0), (2 * c["ffn"] * h, DECAY), (h * c["ffn"], DECAY)]
    return n + [(h, 0.0), (c["vocab"] * h, DECAY)]


def _spans(c):
    """(start, end) of every tensor in the arena: each begins at a multiple of 256 elements."""
    got, at = [], 0
    for n, _ in _tensors(c):
        got.append((at, at + n))
        at += -(-n // 256) * 256
    return got


def work(case):
    c = case
    if c["op"].startswith("attend"):
        T, d = c["T"] - c["tail"], c["d"]
        qkv, o, lse = T * (c["heads"] + 2 * c["kv_heads"]) * d * 2, T * c["heads"] * d * 2, T * c["heads"] * 4
        pairs = c["heads"] * _pairs(c)
        if c["op"] == "attend":  # two products of 2 d operations a pair
            return {"bytes": qkv + o + lse, "flops": 4 * d * pairs}
        return {"bytes": 2 * qkv + 2 * o + lse + (max(_lengths(c), default=0) * d * 4 if c["rope"] else 0), "flops": 10 * d * pairs}
    if c["op"] == "rotary":
        e, turned = 4 if c["dtype"] == "f32" else 2, c["rot"] if c["inplace"] else c["d"]
        table = min(c["rows"], c["span"]) * c["rot"] * 4
        if c["build"]:
            table = c["span"] * c["rot"] * 4
        return {"bytes": 2 * c["rows"] * c["heads"] * turned * e + table + 4 * c["rows"], "flops": 3 * c["rows"] * c["heads"] * c["rot"]}
    n = sum(k for k, _ in _tensors(c))
    each = 8 + (4 if c["grad"] == "f32" else 2) + (2 if c["copy"] else 0) + (16 if c["state"] == 32 else 4 + 16 / 256)
    return {"bytes": int(n * each), "flops": 15 * n}


# ------------------------------------------------------------------------------------------------ inputs
def _tables(span, rot, factors, device="cuda"):
    """cos and sin of position / (10000^(2 i / rot) factors[i]), angles in 64 bits."""
    i = torch.arange(rot // 2, dtype=torch.float64, device=device)
    angle = torch.arange(span, dtype=torch.float64, device=device)[:, None] * (10000.0 ** (-2.0 * i / rot) / factors.double())
    return angle.cos().float(), angle.sin().float()


def _stretch(rot, span):
    """Frequency factors of a stretched context: slow frequencies by up to span / 4096, fast ones hardly."""
    i = torch.arange(rot // 2, dtype=torch.float32, device="cuda")
    return 1.0 + (max(1.0, span / 4096.0) - 1.0) * (i + 1) / (rot // 2)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    if c["op"].startswith("attend"):
        T, d, lens = c["T"], c["d"], _lengths(c)
        c["longest"] = max(lens, default=0)
        c["cu"] = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
        c["qkv"] = torch.randn(T, (c["heads"] + 2 * c["kv_heads"]) * d, generator=g, device="cuda").to(torch.bfloat16)
        c["o"], c["lse"] = torch.zeros(T, c["heads"] * d, dtype=torch.bfloat16, device="cuda"), torch.zeros(c["heads"], T, device="cuda")
        c["bounds"] = torch.empty(3, T, dtype=torch.int32, device="cuda")
        if c["op"] == "attend_grad":  # the forward pass has left its output and log-sum-exp
            c["o"], c["lse"] = _plain_attend(c)
            c["do"] = torch.randn(T, c["heads"] * d, generator=g, device="cuda").to(torch.bfloat16)
            c["dqkv"] = torch.zeros_like(c["qkv"])
            c["cos"], c["sin"] = _tables(c["limit"], d, torch.ones(d // 2, device="cuda")) if c["rope"] else (None, None)
        return c
    if c["op"] == "rotary":
        dt, width = DTYPES[c["dtype"]], (c["heads"] + c["other"]) * c["d"]
        c["x"] = torch.randn(c["rows"], width, generator=g, device="cuda").to(dt)
        c["y"] = c["x"] if c["inplace"] else torch.empty(c["rows"], c["heads"] * c["d"], dtype=dt, device="cuda")
        # documents one behind the other: runs of positions, some of them far from the start
        starts = torch.randint(0, c["span"], (c["rows"],), generator=g, device="cuda")
        run = 512
        c["pos"] = ((starts[torch.arange(c["rows"], device="cuda") // run] + torch.arange(c["rows"], device="cuda") % run) % c["span"]).to(torch.int32)
        c["factors"] = _stretch(c["rot"], c["span"])
        c["cos"], c["sin"] = _tables(c["span"], c["rot"], c["factors"])
        return c
    spans = _spans(c)
    n = -(-spans[-1][1] // 256) * 256
    c["spans"] = spans
    decay = torch.zeros(n // 256, device="cuda")  # of each run of 256 elements; the spans begin at multiples of 256
    live = torch.zeros(n, dtype=torch.bool, device="cuda")
    for (a, b), (_, w) in zip(spans, _tensors(c)):
        decay[a // 256:-(-b // 256)] = w
        live[a:b] = True
    c["decay"] = decay
    normal = lambda scale: torch.randn(n, generator=g, device="cuda") * scale * live  # noqa: E731
    c["p"] = normal(0.02)
    size = 1e-3 * torch.exp2(torch.randint(-6, 3, (n // 256,), generator=g, device="cuda").float()).repeat_interleave(256)  # rows differ in scale
    c["g"] = (normal(1.0) * size).to(DTYPES[c["grad"]])
    m, r = normal(0.4) * size, torch.abs(normal(1.0)) * size
    if c["state"] == 8:
        c["m"], c["m_scale"] = _to8(m.double(), None)
        c["v"], c["v_scale"] = _to8(r.double(), None, floor=True)
        c["seed"] = int(seed) * 2654435761 + 23
    else:
        c["m"], c["v"] = m, r * r
    c["copy16"] = c["p"].to(torch.bfloat16) if c["copy"] else None
    c["step"] = torch.full((1,), 5 + int(seed) % 1000, dtype=torch.int64, device="cuda")  # the training step's counter
    c["clip"] = torch.rand(1, generator=g, device="cuda") * 0.5 + 0.5  # the factor of gradient clipping, left by the norm's kernel
    return c


# ------------------------------------------------------------------------------------------------ plain forms
class _Band:
    """Queries in blocks of L rows, each block with the L + longest - 1 rows that hold all its keys."""

    def __init__(self, c):
        self.T, w = c["T"], max(1, c["longest"])
        self.L = min(self.T, max(64, w))
        self.nb = -(-self.T // self.L)
        dev, cu = c["qkv"].device, c["cu"].long()
        row = torch.arange(self.T, device=dev)
        doc = torch.searchsorted(cu, row, right=True) - 1
        self.live = row < cu[-1]
        self.start = torch.where(self.live, cu[doc.clamp(max=cu.numel() - 1)], 1 << 40)  # others see nothing
        first = torch.arange(self.nb, device=dev) * self.L
        keys = first[:, None] - (w - 1) + torch.arange(self.L + w - 1, device=dev)
        rows = first[:, None] + torch.arange(self.L, device=dev)
        start = torch.where(rows < self.T, self.start[rows.clamp(max=self.T - 1)], 1 << 40)
        self.hidden = ~((keys[:, None, :] <= rows[:, :, None]) & (keys[:, None, :] >= start[:, :, None]))
        self.keys, self.rows = keys.clamp(0, self.T - 1), rows.clamp(0, self.T - 1)

    def queries(self, t):  # [G, rep, T, d] -> [G, nb, rep, L, d]
        return t[:, :, self.rows].transpose(1, 2)

    def back(self, t):  # [G, nb, rep, L, n] -> [G, rep, T, n]
        G, _, R, _, n = t.shape
        return t.transpose(1, 2).reshape(G, R, self.nb * self.L, n)[:, :, :self.T]

    def scores(self, q, k, scale):
        s = (q * scale) @ k[:, :, None].transpose(-1, -2)
        return s.masked_fill_(self.hidden[None, :, None], -math.inf)

    def add_back(self, t):  # [G, nb, keys, d] -> [G, T, d], summed over the blocks that hold a key
        G, _, _, d = t.shape
        return torch.zeros(G, self.T, d, device=t.device).index_add_(1, self.keys.reshape(-1), t.reshape(G, -1, d))


def _split(c, t):
    """Packed rows -> float q [kv, rep, T, d], k and v [kv, T, d]."""
    T, H, G, d = c["T"], c["heads"], c["kv_heads"], c["d"]
    t = t.view(T, H + 2 * G, d).transpose(0, 1).float()
    return t[:H].reshape(G, H // G, T, d), t[H:H + G], t[H + G:]


def _plain_attend(c):
    band = _Band(c)
    q, k, v = _split(c, c["qkv"])
    s = band.scores(band.queries(q), k[:, band.keys], 1.0 / math.sqrt(c["d"]))
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)  # rows that see nothing
    p = s.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    o = band.back(p @ v[:, band.keys][:, :, None] / z)
    lse = band.back(m + z.log())
    o = o.reshape(c["heads"], c["T"], c["d"]).transpose(0, 1).reshape(c["T"], -1)
    return torch.where(band.live[:, None], o, 0.0).to(torch.bfloat16), torch.where(band.live, lse.reshape(c["heads"], c["T"]), 0.0)


def _plain_attend_grad(c):
    band, T, H, G, d = _Band(c), c["T"], c["heads"], c["kv_heads"], c["d"]
    scale = 1.0 / math.sqrt(d)
    q, k, v = _split(c, c["qkv"])
    per_row = lambda t: t.view(T, H, d).transpose(0, 1).reshape(G, H // G, T, d).float()  # noqa: E731
    o, do = per_row(c["o"]), per_row(c["do"])
    qb, dob, kb, vb = band.queries(q), band.queries(do), k[:, band.keys], v[:, band.keys]
    lse = band.queries(c["lse"].view(G, H // G, T, 1))
    delta = band.queries((o * do).sum(-1, keepdim=True))
    p = band.scores(qb, kb, scale).sub_(lse).exp_()
    ds = (dob @ vb[:, :, None].transpose(-1, -2)).sub_(delta).mul_(p)
    fold = lambda t: t.flatten(2, 3)  # noqa: E731
    dv = band.add_back(fold(p).transpose(-1, -2) @ fold(dob))
    dk = band.add_back(fold(ds).transpose(-1, -2) @ fold(qb)) * scale
    dq = band.back(ds @ kb[:, :, None]).reshape(H, T, d) * scale
    if c["rope"]:
        pos = torch.where(band.live, torch.arange(T, device=q.device) - band.start, 0)
        cos, sin = c["cos"][pos], c["sin"][pos]
        turn = lambda t: torch.cat([t[..., :d // 2] * cos + t[..., d // 2:] * sin, t[..., d // 2:] * cos - t[..., :d // 2] * sin], -1)  # noqa: E731
        dq, dk = turn(dq), turn(dk)
    out = torch.cat([dq, dk, dv]).transpose(0, 1).reshape(T, -1)
    return torch.where(band.live[:, None], out, 0.0).to(torch.bfloat16)


def _plain_rotary(c):
    cos, sin = _tables(c["span"], c["rot"], c["factors"]) if c["build"] else (c["cos"], c["sin"])
    at = c["pos"].long()
    co, si = cos[at][:, None], sin[at][:, None]
    if c["inverse"]:
        si = -si
    x = c["x"][:, :c["heads"] * c["d"]].view(c["rows"], c["heads"], c["d"])
    turned = x[..., :c["rot"]].float()
    if c["style"] == "half":
        a, b = turned.chunk(2, -1)
        turned = torch.cat([a * co - b * si, b * co + a * si], -1)
    else:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * co - b * si, b * co + a * si], -1).flatten(-2)
    turned = turned.to(c["x"].dtype)
    if c["inplace"]:
        x[..., :c["rot"]] = turned
        out = c["x"]
    else:
        out = torch.cat([turned, x[..., c["rot"]:]], -1).view(c["rows"], -1)
    return [out, cos, sin] if c["build"] else out


_STEP, _GROUP = 0xA24BAED4963EE407, 0x8CB92BA72F3D8DD7


def _i64(v):
    """A 64-bit pattern as the signed number torch keeps."""
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _mix(z):
    """The splitmix64 finaliser on int64 tensors (wrapping arithmetic, logical shifts)."""
    z = z + _i64(0x9E3779B97F4A7C15)
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _i64(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _i64(0x94D049BB133111EB)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _random16(c, n):
    """[n, 2] numbers in [0, 1): 16 bits for the first and 16 for the second moment of each element, a 64-bit word a pair."""
    key = _mix(_mix(torch.full((1,), _i64(c["seed"]), dtype=torch.int64, device="cuda")) ^ (c["step"] * _i64(_STEP)))
    word = _mix(key ^ (torch.arange(n // 2, dtype=torch.int64, device="cuda") * _i64(_GROUP)))
    return ((word[:, None] >> torch.arange(0, 64, 16, device="cuda")) & 0xFFFF).double().view(n, 2) / 65536.0


def _to8(x, u, floor=False):
    """Signed 8-bit floats (4 exponent, 3 mantissa bits, at most 448) and a scale for every 256 elements.  u: what is added to
    the number of steps before it is cut (None: to nearest); floor: what is not 0 stays at least the smallest code."""
    x = x.view(-1, 256)
    top = x.abs().amax(1, keepdim=True)
    scale = torch.where(top >= 2.0 ** -100, top / 448.0, 0.0)
    y = torch.where(scale > 0, x.abs() / scale, 0.0)
    step = torch.exp2(torch.log2(y.clamp(min=2.0 ** -6)).floor() - 3.0)
    q = ((y / step).round() if u is None else (y / step + u.view_as(y)).floor()) * step
    q = q.clamp(max=448.0)
    if floor:
        q = torch.where((x != 0) & (scale > 0), q.clamp(min=2.0 ** -9), q)
    return torch.copysign(q, x).view(-1).float().to(torch.float8_e4m3fn), scale.view(-1).float()


def _plain_adamw(c):
    wide = torch.float64 if c["state"] == 8 else torch.float32  # codes flip where a moment lies on the border between two
    n = c["p"].numel()
    runs = lambda t: t.view(-1, 256)  # noqa: E731
    grad = c["g"].to(wide) * c["clip"].to(wide)
    if c["state"] == 8:
        m = (runs(c["m"].to(wide)) * c["m_scale"].to(wide)[:, None]).view(-1)
        v = (runs(c["v"].to(wide)) * c["v_scale"].to(wide)[:, None]).view(-1).square()
    else:
        m, v = c["m"], c["v"]
    m = BETA1 * m + (1 - BETA1) * grad
    v = BETA2 * v + (1 - BETA2) * grad * grad
    t = c["step"].double()
    mhat, vhat = m / (1 - BETA1 ** t).to(wide), v / (1 - BETA2 ** t).to(wide)
    p = c["p"].to(wide)
    update = mhat / (vhat.sqrt() + ADAM_EPS) + (runs(p) * c["decay"].to(wide)[:, None]).view(-1)
    c["p"].copy_(p - LR * update)
    if c["state"] == 8:
        u = _random16(c, n)
        (qm, sm), (qv, sv) = _to8(m, u[:, 0]), _to8(v.sqrt(), u[:, 1], floor=True)
        c["m"].copy_(qm), c["m_scale"].copy_(sm), c["v"].copy_(qv), c["v_scale"].copy_(sv)
    else:
        c["m"].copy_(m), c["v"].copy_(v)
    if c["copy"]:
        c["copy16"].copy_(c["p"])
    return _adamw_outputs(c)


def _adamw_outputs(c):
    return {k: c[k] for k in ("p", "m", "v", "m_scale", "v_scale", "copy16") if c.get(k) is not None}


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    c = state
    if own:
        return _run_own(c)
    if c["op"] == "attend":
        return _plain_attend(c)
    if c["op"] == "attend_grad":
        return _plain_attend_grad(c)
    return _plain_rotary(c) if c["op"] == "rotary" else _plain_adamw(c)


def _run_own(c):
    from paper_2609_13645_b200 import binding as ft
    if c["op"].startswith("attend"):
        size = (c["T"], c["heads"], c["kv_heads"], c["d"])
        ft.k_packed_bounds(c["cu"], c["bounds"], c["T"], c["limit"])  # of a batch; every layer uses them
        if c["op"] == "attend":
            ft.k_attention_packed_fwd(c["qkv"], c["o"], c["lse"], c["bounds"], *size)
            return c["o"], c["lse"]
        if "scratch" not in c:  # the workspace a user's program allocates once and keeps
            c["scratch"] = torch.empty(ft.attention_packed_scratch_bytes(*size, c["limit"]), dtype=torch.uint8, device="cuda")
        ft.k_attention_packed_bwd(c["qkv"], c["o"], c["do"], c["lse"], c["dqkv"], c["bounds"], c["scratch"], *size, c["limit"],
                                  cos=c["cos"], sin=c["sin"])
        return c["dqkv"]
    if c["op"] == "rotary":
        if c["build"]:
            ft.k_rotary_tables(c["cos"], c["sin"], 10000.0, factors=c["factors"])
        x = c["x"][:, :c["heads"] * c["d"]]
        ft.k_rotary(x, x if c["inplace"] else c["y"], c["cos"], c["sin"], c["heads"], c["d"], positions=c["pos"],
                    interleaved=c["style"] == "pairs", inverse=c["inverse"])
        return [c["y"], c["cos"], c["sin"]] if c["build"] else c["y"]
    if "plan" not in c:  # the list of its tensors, which a user's program hands over once
        part = lambda t: [t[a:b] for a, b in c["spans"]]  # noqa: E731
        scale = lambda t: [t[a // 256:-(-b // 256)] for a, b in c["spans"]]  # noqa: E731
        eight = c["state"] == 8
        c["plan"] = ft.AdamWPlan(part(c["p"]), part(c["g"]), part(c["m"]), part(c["v"]), weight_decay=[w for _, w in _tensors(c)],
                                 m_scales=scale(c["m_scale"]) if eight else None, v_scales=scale(c["v_scale"]) if eight else None,
                                 copies=part(c["copy16"]) if c["copy"] else None)
    ft.k_adamw(c["plan"], LR, BETA1, BETA2, ADAM_EPS, c["step"], grad_scale=c["clip"], seed=c.get("seed", 0))
    return _adamw_outputs(c)


# ------------------------------------------------------------------------------------------------ definitions in 64 bits
def _exact_attend(c):
    """Document by document, head by head, over the whole score matrix."""
    T, H, G, d = c["T"], c["heads"], c["kv_heads"], c["d"]
    grad, f64 = c["op"] == "attend_grad", dict(dtype=torch.float64, device="cuda")
    lens = _lengths(c)
    if len(lens) * H > 12000:
        return None
    x = c["qkv"].double().view(T, H + 2 * G, d)
    o, lse, dx = torch.zeros(T, H, d, **f64), torch.zeros(H, T, **f64), torch.zeros(T, H + 2 * G, d, **f64)
    s0 = 0
    for n in lens:
        s1 = s0 + n
        later = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
        for h in range(H if n else 0):
            kv = h * G // H
            q, k, v = x[s0:s1, h], x[s0:s1, H + kv], x[s0:s1, H + G + kv]
            s = (q @ k.T / math.sqrt(d)).masked_fill_(later, -math.inf)
            p = torch.softmax(s, -1)
            if not grad:
                o[s0:s1, h], lse[h, s0:s1] = p @ v, torch.logsumexp(s, -1)
                continue
            do, oi = (c[t].view(T, H, d)[s0:s1, h].double() for t in ("do", "o"))
            ds = p * (do @ v.T - (do * oi).sum(-1, keepdim=True)) / math.sqrt(d)
            dx[s0:s1, h] = ds @ k
            dx[s0:s1, H + kv] += ds.T @ q
            dx[s0:s1, H + G + kv] += p.T @ do
        if grad and c["rope"]:
            cos, sin = c["cos"][:n].double()[:, None], c["sin"][:n].double()[:, None]
            a, b = dx[s0:s1, :H + G, :d // 2].clone(), dx[s0:s1, :H + G, d // 2:].clone()
            dx[s0:s1, :H + G, :d // 2], dx[s0:s1, :H + G, d // 2:] = a * cos + b * sin, b * cos - a * sin
        s0 = s1
    return dx.view(T, -1) if grad else (o.view(T, H * d), lse)


def _exact_rotary(c):
    """Pairs as complex numbers times exp(i angle)."""
    half, d = c["rot"] // 2, c["d"]
    pos, f = c["pos"].double(), c["factors"].double()
    angle_of = lambda p: torch.outer(p, torch.exp(torch.arange(half, device="cuda").double() * (-2.0 / c["rot"] * math.log(10000.0))) / f)  # noqa: E731
    whole = c["x"].double()
    x = whole[:, :c["heads"] * d].reshape(c["rows"], c["heads"], d)
    if c["style"] == "half":
        z = torch.complex(x[..., :half], x[..., half:c["rot"]])
    else:
        z = torch.view_as_complex(x[..., :c["rot"]].unflatten(-1, (half, 2)).contiguous())
    if c["build"]:
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), angle_of(pos))
    else:  # the tables are inputs
        at = c["pos"].long()
        turn = torch.complex(c["cos"].double()[at], c["sin"].double()[at])
    z = z * (turn.conj() if c["inverse"] else turn)[:, None]
    x = x.clone()
    if c["style"] == "half":
        x[..., :half], x[..., half:c["rot"]] = z.real, z.imag
    else:
        x[..., 0:c["rot"]:2], x[..., 1:c["rot"]:2] = z.real, z.imag
    out = x.view(c["rows"], -1)
    if c["inplace"]:
        out = torch.cat([out, whole[:, c["heads"] * d:]], 1)
    if not c["build"]:
        return out
    angle = angle_of(torch.arange(c["span"], device="cuda").double())
    return [out, torch.cos(angle), torch.sin(angle)]


def _exact_adamw(c):
    """Tensor by tensor; the random numbers of the 8-bit codes on the CPU's unsigned integers."""
    t = int(c["step"][0])
    clip, eight = float(c["clip"][0]), c["state"] == 8
    out = {k: c[k].double().clone() for k in ("p", "m", "v", "m_scale", "v_scale", "copy16") if c.get(k) is not None}

    def mix(z):
        z = z + np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))

    def code(x, scale, u, at_least):
        mant, e = torch.frexp((x.abs() / scale).nan_to_num(0.0, 0.0))  # mant in [1/2, 1)
        step = torch.ldexp(torch.ones_like(x), e.clamp(min=-5) - 4)
        q = torch.minimum(torch.floor(torch.ldexp(mant, e) / step + u) * step, torch.full_like(x, 448.0))
        return torch.sign(x) * torch.maximum(q, torch.where(x != 0, at_least, 0.0) * torch.ones_like(x))

    whole = (1 << 64) - 1
    with np.errstate(over="ignore"):
        key = mix(mix(np.array([c.get("seed", 0) & whole], dtype=np.uint64)) ^ np.array([t * _STEP & whole], dtype=np.uint64))
    for (a, b), (_, decay) in zip(c["spans"], _tensors(c)):
        g = c["g"][a:b].double() * clip
        pad = -(b - a) % 256
        if eight:
            per = lambda s: out[s][a // 256:-(-b // 256)].repeat_interleave(256)[:b - a]  # noqa: E731
            m0, v0 = out["m"][a:b] * per("m_scale"), (out["v"][a:b] * per("v_scale")) ** 2
        else:
            m0, v0 = out["m"][a:b], out["v"][a:b]
        m, v = torch.lerp(g, m0, BETA1), torch.lerp(g * g, v0, BETA2)
        out["p"][a:b] = out["p"][a:b] * (1 - LR * decay) - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + ADAM_EPS)
        if c["copy"]:
            out["copy16"][a:b] = out["p"][a:b]
        if not eight:
            out["m"][a:b], out["v"][a:b] = m, v
            continue
        with np.errstate(over="ignore"):
            words = mix(key ^ (np.arange(a // 2, (b + pad) // 2, dtype=np.uint64) * np.uint64(_GROUP)))
        u = torch.from_numpy(words.astype("<u8").view("<u2").astype(np.int32)).cuda().double()[:2 * (b - a)] / 65536.0
        for k, x, uk, low in (("m", m, u[0::2], 0.0), ("v", v.sqrt(), u[1::2], 2.0 ** -9)):
            top = torch.nn.functional.pad(x.abs(), (0, pad)).view(-1, 256).max(1).values / 448.0
            out[k + "_scale"][a // 256:-(-b // 256)] = top
            out[k][a:b] = code(x, top.repeat_interleave(256)[:b - a], uk, low)
    return out


def exact(case, seed):
    c = prepare(case, seed)
    if c["op"].startswith("attend"):
        return _exact_attend(c)
    return _exact_rotary(c) if c["op"] == "rotary" else _exact_adamw(c)
