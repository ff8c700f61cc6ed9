"""The operators around an 8-bit key/value memory: rotary positions of a layer's queries and keys, rows
quantised into the memory and read back, and the two-view window attention that reads it.

A diffusion decoder with a prefix cache keeps the keys and values of every position and recomputes
the active block's rows only. With the memory in 8 bits a step's layer is: rotate the block's q and k
to their positions, write the block's k and v rows (and the seeds' cached rows) into the memory, and
let the block's queries attend over it.

The memory of a layer holds per row (batch row, KV head, position) D codes in e4m3 and one
exponent byte x in e8m0: the row's values are code * 2^(x - 127), exact in bf16 and in fp32. x is the
smallest for which the row's largest magnitude is at most 448 * 2^(x - 127), held to 17 .. 246 (127
for a row of zeros); a row with an element that is not finite has x = 255 and reads as NaN.

Kinds of cases and their fields:
  rope   q [B, Hq, L, D] and k [B, Hkv, L, D], as a projection leaves them ([B, L, H, D] in memory), to
         positions of their own for each sequence; the first R of D columns turn, in pairs of
         neighbours (``inter``) or of halves; ``yarn`` > 1: frequencies stretched for long contexts.
  write  n rows of every sequence into a memory of L positions: at consecutive positions (``listed``
         false) or at listed ones, of which some are out of range or named twice (the lowest slot is taken).
  read   n rows back, as above (a position out of range reads as zeros).
  attn   Lq queries at q0 over a memory of Lk positions, S seed positions a sequence; ``mask``: the keys that
         a row sees are all of them, its sequence's (lens, of which one may be empty), the prefix and what is
         before it (prefix), its block and those before (blocks) or its document's (docs); ``cap``: scores capped.
"""
import math

import torch

own = False


def listed():
    return [
        # one token of a batch, far into a stretched context: latency is all
        dict(name="rope_token", kind="rope", dtype="bf16", B=4, Hq=28, Hkv=4, L=1, D=128, R=128, inter=False,
             yarn=4.0, far=120000, inverse=False),
        # active blocks of 64 rows, half of each head turned, turned back (the gradient's direction)
        dict(name="rope_blocks_back", kind="rope", dtype="f32", B=8, Hq=32, Hkv=32, L=64, D=64, R=32, inter=True,
             yarn=1.0, far=4000, inverse=True),
        # prompts of a batch, of an odd length
        dict(name="rope_prompt", kind="rope", dtype="bf16", B=4, Hq=32, Hkv=8, L=8191, D=128, R=128, inter=False,
             yarn=1.0, far=0, inverse=False),
        # the active block of one sequence into its memory
        dict(name="write_block", kind="write", dtype="bf16", B=1, Hkv=4, n=32, L=1024, D=128, listed=False),
        # the seeds' cached fp32 rows into the memories of a batch
        dict(name="write_seeds", kind="write", dtype="f32", B=8, Hkv=32, n=64, L=2048, D=64, listed=True),
        # prompts of a batch
        dict(name="write_prompt", kind="write", dtype="bf16", B=4, Hkv=8, n=8191, L=8200, D=128, listed=False),
        # the next seeds' rows, to be cached
        dict(name="read_seeds", kind="read", dtype="bf16", B=8, Hkv=32, n=64, L=2048, D=128, listed=True),
        # whole memories, for a program that goes on in bf16
        dict(name="read_memory", kind="read", dtype="bf16", B=4, Hkv=8, n=8191, L=8191, D=128, listed=False),
        # one token of one short sequence
        dict(name="attn_token", kind="attn", B=1, Hq=28, Hkv=4, Lq=1, Lk=777, q0=776, S=0, mask="none", cap=0.0),
        # the active block of one sequence, verified with seeds
        dict(name="attn_block_seeds", kind="attn", B=1, Hq=28, Hkv=4, Lq=32, Lk=1024, q0=600, S=32, mask="none", cap=0.0),
        # tokens of a padded batch over long memories
        dict(name="attn_token_long", kind="attn", B=4, Hq=32, Hkv=8, Lq=1, Lk=131072, q0=131071, S=0, mask="lens", cap=0.0),
        # a prompt's last part, in blocks that see themselves and those before, scores capped
        dict(name="attn_prompt", kind="attn", B=1, Hq=32, Hkv=8, Lq=2048, Lk=8192, q0=6144, S=64, mask="blocks", cap=30.0),
    ]


HEADS = [(32, 32), (28, 4), (32, 8), (16, 2)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "write", "read", "attn", "attn", "attn"])
    Hq, Hkv = rng.choice(HEADS)
    if kind == "rope":
        D = rng.choice([64, 128])
        while True:
            B, L, dtype = _log(rng, 1, 16), _log(rng, 1, 8192), rng.choice(["bf16", "f32"])
            if B * L * (Hq + Hkv) * D * (2 if dtype == "bf16" else 4) < 320e6:
                break
        return dict(kind=kind, dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, L=L, D=D, R=rng.choice([D, D, D // 2]),
                    inter=rng.random() < 0.5, yarn=rng.choice([1.0, 1.0, 4.0, 16.0]), far=_log(rng, 1, 120000),
                    inverse=rng.random() < 0.3)
    if kind in ("write", "read"):
        D, by = rng.choice([64, 128]), rng.random() < 0.4
        while True:
            B, n, dtype = _log(rng, 1, 16), _log(rng, 1, 512 if by else 8192), rng.choice(["bf16", "f32"])
            L = n + _log(rng, 1, 2000) if by else n + rng.choice([0, 1, 77])
            if B * Hkv * L * D * (2 if dtype == "bf16" else 4) < 67e6:
                break
        return dict(kind=kind, dtype=dtype, B=B, Hkv=Hkv, n=n, L=L, D=D, listed=by)
    while True:
        B = _log(rng, 1, 16)
        Lq = 1 if rng.random() < 0.3 else _log(rng, 2, 1024)
        Lk = Lq + _log(rng, 16, 65536)
        if B * Hkv * Lk < 2.0e6 and 512.0 * B * Hq * Lq * Lk < 2e11 and 4.0 * B * Hq * Lq * Lk < 4e9:
            break
    q0 = rng.randint(0, Lk - Lq)
    return dict(kind="attn", B=B, Hq=Hq, Hkv=Hkv, Lq=Lq, Lk=Lk, q0=q0, S=0 if rng.random() < 0.4 else min(Lk // 2, _log(rng, 1, 64)),
                mask=rng.choice(["none", "lens", "prefix", "blocks", "docs"]), cap=rng.choice([0.0, 0.0, 30.0, 50.0]))


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _frequencies(c):
    """Radians a position of each of the R / 2 pairs, in fp64, and the factor of the turned columns: base
    10000; stretched by ``yarn`` where a pair turns less than once in 4096 positions, not at all where it
    turns 32 times or more, with a ramp between."""
    R = c["R"]
    i = torch.arange(R // 2, dtype=torch.float64, device="cuda")
    f = 10000.0 ** (-2.0 * i / R)
    if c["yarn"] == 1.0:
        return f, 1.0
    turns = 4096 * f / (2 * math.pi)
    keep = ((turns - 1) / (32 - 1)).clamp(0, 1)
    return f * keep + f / c["yarn"] * (1 - keep), 0.1 * math.log(c["yarn"]) + 1.0


def _rows(g, B, H, n, D, dtype):
    """Rows of n tokens as a projection leaves them ([B, n, H, D] in memory), as [B, H, n, D]; a few columns are
    larger than the others, as keys' are."""
    x = torch.randn((B, n, H, D), generator=g, device="cuda")
    return (x * (1 + 6 * (torch.rand(D, generator=g, device="cuda") < 0.04))).to(dtype).transpose(1, 2)


def _power(e):
    """2^e in fp32 for whole numbers e of -126 .. 127, from its bits (pow and exp2 may be a step off)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _encode(x):
    """e4m3 codes and e8m0 bytes of rows x [..., D]."""
    x = x.float()
    amax = x.abs().amax(-1)
    bad = ~torch.isfinite(amax)
    m, e = torch.frexp(torch.where(bad, 0.0, amax))
    byte = torch.where(m <= 0.875, e - 9, e - 8).clamp(-110, 119) + 127
    byte = torch.where(amax == 0, 127, torch.where(bad, 255, byte))
    scaled = torch.where(bad[..., None], 0.0, x * _power(127 - byte.clamp(max=246))[..., None]).clamp(-448, 448)
    return scaled.to(torch.float8_e4m3fn), byte.to(torch.uint8)


def _decode(codes, byte):
    """fp32 values of codes [..., D] with bytes [...]."""
    v = codes.float() * _power(byte.clamp(max=254).int() - 127)[..., None]
    return torch.where((byte == 255)[..., None], math.nan, v)


def _memory(g, B, H, L, D):
    return _encode(_rows(g, B, H, L, D, torch.float32).contiguous())


def _positions(g, c):
    """n listed positions of each sequence: distinct but for two that name another's, two out of range."""
    B, n, L = c["B"], c["n"], c["L"]
    pos = torch.rand((B, L), generator=g, device="cuda").argsort(1)[:, :n].to(torch.int32)
    if n >= 16:
        pos[:, n // 2] = pos[:, 1]
        pos[:, n - 1] = pos[:, n // 3]
        pos[:, 5] = -1
        pos[:, n // 2 + 1] = L + 3
    return pos.contiguous()


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if c["kind"] == "rope":
        dt = _type(c["dtype"])
        start = (torch.rand((c["B"], 1), generator=g, device="cuda") * (c["far"] + 1)).int()
        f, mscale = _frequencies(c)
        return dict(case=c, q=_rows(g, c["B"], c["Hq"], c["L"], c["D"], dt), k=_rows(g, c["B"], c["Hkv"], c["L"], c["D"], dt),
                    pos=start + torch.arange(c["L"], device="cuda", dtype=torch.int32), f=f, mscale=mscale)
    if c["kind"] in ("write", "read"):
        pos = _positions(g, c) if c["listed"] else None
        k8, kx = _memory(g, c["B"], c["Hkv"], c["L"], c["D"])
        v8, vx = _memory(g, c["B"], c["Hkv"], c["L"], c["D"])
        s = dict(case=c, k8=k8, kx=kx, v8=v8, vx=vx, pos=pos, pos0=c["L"] - c["n"])
        if c["kind"] == "write":
            s["k"], s["v"] = (_rows(g, c["B"], c["Hkv"], c["n"], c["D"], _type(c["dtype"])) for _ in range(2))
        return s
    B, Hkv, Lq, Lk, S, q0 = c["B"], c["Hkv"], c["Lq"], c["Lk"], c["S"], c["q0"]
    k8, kx = _memory(g, B, Hkv, Lk, 128)
    v8, vx = _memory(g, B, Hkv, Lk, 128)
    q = torch.randn((B, c["Hq"], Lq, 128), generator=g, device="cuda").to(torch.bfloat16)
    s = dict(case=c, q=q, k8=k8, kx=kx, v8=v8, vx=vx, km=None, vm=None, seeds=None, lo=None, hi=None)
    if S > 0:
        order = torch.rand((B, Lk), generator=g, device="cuda")
        order[:, q0:q0 + Lq] -= 0.7           # most seeds are in the active rows
        s["seeds"] = order.argsort(1)[:, :S].to(torch.int32).contiguous()
        if S >= 4:
            s["seeds"][:, S - 1] = -1         # fewer were selected than the list has room for
        s["km"], s["vm"] = (torch.randn((B, Hkv, S, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    at = q0 + torch.arange(Lq, device="cuda", dtype=torch.int32).repeat(B, 1)
    lens = (Lk * (0.3 + 0.7 * torch.rand((B, 1), generator=g, device="cuda"))).int()
    if c["mask"] == "lens":
        lens[0] = Lk
        if B >= 4:
            lens[B - 1] = 0                   # a place of the batch without a sequence
        s["lo"], s["hi"] = torch.zeros_like(at), lens.expand(B, Lq).contiguous()
    elif c["mask"] == "prefix":
        s["lo"], s["hi"] = torch.zeros_like(at), torch.maximum(at + 1, lens)
    elif c["mask"] == "blocks":
        s["lo"], s["hi"] = torch.zeros_like(at), ((at // 64 + 1) * 64).clamp(max=Lk)
    elif c["mask"] == "docs":
        size = max(1, Lk // 5)
        s["lo"], s["hi"] = at // size * size, (at // size * size + size).clamp(max=Lk)
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------

def _turned(x, c, cos, sin, mscale):
    """x [B, H, L, D] with its first R columns turned by angles whose cos, sin are [B, 1, L, R / 2]."""
    R, f = c["R"], x.float()
    turn, rest = f[..., :R], f[..., R:]
    a, b = (turn[..., 0::2], turn[..., 1::2]) if c["inter"] else (turn[..., :R // 2], turn[..., R // 2:])
    s = -sin if c["inverse"] else sin
    ya, yb = (a * cos - b * s) * mscale, (a * s + b * cos) * mscale
    y = torch.stack((ya, yb), -1).flatten(-2) if c["inter"] else torch.cat((ya, yb), -1)
    return torch.cat((y, rest), -1).to(x.dtype).contiguous()


def _slots(pos, n, L):
    """[B, L]: the lowest slot that names the position, n where none does."""
    at = torch.where((pos >= 0) & (pos < L), pos, L).long()
    slot = torch.arange(n, device=pos.device).expand_as(at)
    return torch.full((pos.shape[0], L + 1), n, device=pos.device).scatter_reduce(1, at, slot, "amin")[:, :L]


def _write(s, x, codes, byte):
    c = s["case"]
    new, new_x = _encode(x)
    if s["pos"] is None:
        codes[:, :, s["pos0"]:s["pos0"] + c["n"]], byte[:, :, s["pos0"]:s["pos0"] + c["n"]] = new, new_x
        return
    slot = _slots(s["pos"], c["n"], c["L"])[:, None]
    named = slot < c["n"]
    take = slot.clamp(max=c["n"] - 1).expand(c["B"], c["Hkv"], c["L"])
    rows = new.view(torch.uint8).gather(2, take[..., None].expand(-1, -1, -1, c["D"]))
    old = codes.view(torch.uint8)
    old.copy_(torch.where(named[..., None], rows, old))
    byte.copy_(torch.where(named, new_x.gather(2, take), byte))


def _read(s, codes, byte):
    c = s["case"]
    dt = _type(c["dtype"])
    if s["pos"] is None:
        return _decode(codes[:, :, s["pos0"]:s["pos0"] + c["n"]], byte[:, :, s["pos0"]:s["pos0"] + c["n"]]).to(dt)
    fine = (s["pos"] >= 0) & (s["pos"] < c["L"])
    at = torch.where(fine, s["pos"], 0).long()[:, None].expand(-1, c["Hkv"], -1)
    rows = codes.view(torch.uint8).gather(2, at[..., None].expand(-1, -1, -1, c["D"])).view(torch.float8_e4m3fn)
    return torch.where(fine[:, None, :, None], _decode(rows, byte.gather(2, at)), 0.0).to(dt)


def _attention(s):
    c = s["case"]
    B, Hq, Hkv, Lq, Lk, S = c["B"], c["Hq"], c["Hkv"], c["Lq"], c["Lk"], c["S"]
    G = Hq // Hkv
    k, v = _decode(s["k8"], s["kx"]), _decode(s["v8"], s["vx"])
    q = s["q"].float().view(B, Hkv, G, Lq, 128)
    z = torch.matmul(q.view(B, Hkv, G * Lq, 128), k.transpose(2, 3)).view(B, Hkv, G, Lq, Lk) / math.sqrt(128)
    at = torch.arange(Lk, device=z.device)
    here = torch.arange(Lq, device=z.device) + c["q0"]
    own_column = (at == here[:, None])                                   # [Lq, Lk]
    if S > 0:
        slot = _slots(s["seeds"], S, Lk)[:, here]                        # [B, Lq]
        is_seed = slot < S
        take = slot.clamp(max=S - 1)[:, None, :, None].expand(B, Hkv, Lq, 128)
        ks, vs = s["km"].float().gather(2, take), s["vm"].float().gather(2, take)
        z_self = (q * ks[:, :, None]).sum(-1) / math.sqrt(128)           # [B, Hkv, G, Lq]
        swap = is_seed[:, None, None, :, None] & own_column              # [B, 1, 1, Lq, Lk]
        z = torch.where(swap, z_self[..., None], z)
    if c["cap"] > 0:
        z = c["cap"] * torch.tanh(z / c["cap"])
    if s["lo"] is not None:
        seen = (at >= s["lo"][..., None]) & (at < s["hi"][..., None])    # [B, Lq, Lk]
        z = z.masked_fill(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    w = p / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total)).view(B, Hq, Lq)
    if S > 0:
        w_self = torch.where(swap, w, 0.0).sum(-1, keepdim=True)
        w = torch.where(swap, 0.0, w)
    o = torch.matmul(w.view(B, Hkv, G * Lq, Lk), v).view(B, Hkv, G, Lq, 128)
    if S > 0:
        o = o + w_self * vs[:, :, None]
    return o.reshape(B, Hq, Lq, 128).to(torch.bfloat16), lse


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2602_06161_gb300 import api
        if c["kind"] == "rope":
            return api.cover_rope_fwd(s["q"], s["k"], s["f"], pos=s["pos"], interleaved=c["inter"], mscale=s["mscale"],
                                      inverse=c["inverse"])
        if c["kind"] == "write":
            api.cover_kv8_write(s["k"], s["v"], s["k8"], s["v8"], s["kx"], s["vx"], pos=s["pos"], pos0=s["pos0"])
            return s["k8"], s["v8"], s["kx"], s["vx"]
        if c["kind"] == "read":
            return api.cover_kv8_read(s["k8"], s["v8"], s["kx"], s["vx"], pos=s["pos"], pos0=s["pos0"], n=c["n"],
                                      dtype=_type(c["dtype"]))
        return api.cover_attn_fwd_prefix8(s["q"], s["k8"], s["v8"], s["kx"], s["vx"], s["km"], s["vm"], s["seeds"],
                                          q0=c["q0"], key_lo=s["lo"], key_hi=s["hi"], softcap=c["cap"])
    if c["kind"] == "rope":
        angle = s["pos"].double()[:, None, :, None] * s["f"]
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        return _turned(s["q"], c, cos, sin, s["mscale"]), _turned(s["k"], c, cos, sin, s["mscale"])
    if c["kind"] == "write":
        _write(s, s["k"], s["k8"], s["kx"])
        _write(s, s["v"], s["v8"], s["vx"])
        return s["k8"], s["v8"], s["kx"], s["vx"]
    if c["kind"] == "read":
        return _read(s, s["k8"], s["kx"]), _read(s, s["v8"], s["vx"])
    return _attention(s)


def work(case):
    c = case
    if c["kind"] == "rope":
        n = c["B"] * c["L"] * (c["Hq"] + c["Hkv"])
        return dict(bytes=2 * n * c["D"] * (2 if c["dtype"] == "bf16" else 4) + 4 * c["B"] * c["L"] + 4 * c["R"],
                    flops=3 * n * c["R"])
    if c["kind"] in ("write", "read"):
        n = c["B"] * c["n"] * c["Hkv"] * 2
        wide = c["D"] * (2 if c["dtype"] == "bf16" else 4)
        return dict(bytes=n * (wide + c["D"] + 1) + (4 * c["B"] * c["n"] if c["listed"] else 0), flops=2 * n * c["D"])
    B, Hq, Hkv, Lq, Lk, q0 = c["B"], c["Hq"], c["Hkv"], c["Lq"], c["Lk"], c["q0"]
    rows = range(q0, q0 + Lq)
    if c["mask"] == "lens":          # as prepare draws them, at their mean
        seen = Lk * (1 + 0.65 * max(0, B - 2) + (0.65 if 1 < B < 4 else 0)) / B
        pairs, keys = seen * Lq, seen
    elif c["mask"] == "prefix":
        pairs, keys = sum(max(r + 1, 0.65 * Lk) for r in rows), max(q0 + Lq, 0.65 * Lk)
    elif c["mask"] == "blocks":
        pairs, keys = sum(min(Lk, (r // 64 + 1) * 64) for r in rows), min(Lk, ((q0 + Lq - 1) // 64 + 1) * 64)
    elif c["mask"] == "docs":
        size = max(1, Lk // 5)
        ends = [(r // size * size, min(Lk, r // size * size + size)) for r in rows]
        pairs, keys = sum(e - b for b, e in ends), ends[-1][1] - ends[0][0]
    else:
        pairs, keys = float(Lq) * Lk, Lk
    return dict(bytes=B * (Hkv * keys * 2 * 129 + Hq * Lq * (128 * 4 + 4) + Hkv * c["S"] * 512), flops=512.0 * B * Hq * pairs)


# ------------------------------------------------------------------------------------------------
# the definitions, in 64 bits
# ------------------------------------------------------------------------------------------------

def _two64(power):
    """2^power in fp64, from its bits."""
    return ((power.long() + 1023) << 52).view(torch.float64)


def _values64(codes, byte):
    power = torch.where(byte == 255, math.nan, _two64(byte.long() - 127))
    return codes.double() * power.unsqueeze(-1)


def _rows64(x):
    """The code values of rows x by their definition: the nearest of e4m3's values, ties to even."""
    x = x.double()
    top = x.abs().max(-1, keepdim=True).values.clamp(min=2.0 ** -60)
    power = torch.frexp(top / 448)[1]                       # 448 * 2^power > top
    power = torch.where(448 * _two64(power - 1) >= top, power - 1, power)
    y = x * _two64(-power)
    step = _two64(torch.clamp(torch.frexp(y)[1] - 1, min=-6) - 3)
    return torch.round(y / step) * step


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "rope":
        i = torch.arange(c["R"] // 2, device="cuda")
        lo, hi = (2 * i, 2 * i + 1) if c["inter"] else (i, i + c["R"] // 2)
        turn = torch.polar(torch.full_like(s["f"], s["mscale"]).expand(c["B"], c["L"], -1).contiguous(),
                           s["pos"].double().unsqueeze(-1) * s["f"] * (-1 if c["inverse"] else 1))
        outs = []
        for x in (s["q"], s["k"]):
            y = x.double().contiguous()
            z = torch.complex(y[..., lo], y[..., hi]) * turn.unsqueeze(1)
            y[..., lo], y[..., hi] = z.real, z.imag
            outs.append(y)
        return tuple(outs)
    if c["kind"] == "write":
        outs = []
        for x, m in ((s["k"], s["k8"]), (s["v"], s["v8"])):
            y, new = m.double(), _rows64(x)
            for b in range(c["B"]):
                at = s["pos"][b].tolist() if c["listed"] else range(s["pos0"], s["pos0"] + c["n"])
                first = {}
                for i, p in enumerate(at):
                    if 0 <= p < c["L"]:
                        first.setdefault(p, i)
                y[b][:, list(first)] = new[b][:, list(first.values())]
            outs.append(y)
        return outs[0], outs[1], None, None
    if c["kind"] == "read":
        outs = []
        for m, x in ((s["k8"], s["kx"]), (s["v8"], s["vx"])):
            rows = _values64(m, x)
            if c["listed"]:
                rows = torch.cat((rows, torch.zeros_like(rows[:, :, :1])), 2)
                at = torch.where((s["pos"] < 0) | (s["pos"] >= c["L"]), torch.full_like(s["pos"], c["L"]), s["pos"]).long()
                outs.append(torch.stack([rows[b][:, at[b]] for b in range(c["B"])]))
            else:
                outs.append(rows[:, :, s["pos0"]:s["pos0"] + c["n"]])
        return tuple(outs)
    B, Hq, Hkv, Lq, Lk, S, q0 = c["B"], c["Hq"], c["Hkv"], c["Lq"], c["Lk"], c["S"], c["q0"]
    out = torch.zeros((B, Hq, Lq, 128), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq, Lq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        where = {}
        for slot, p in enumerate(s["seeds"][b].tolist() if S else []):
            if q0 <= p < q0 + Lq:
                where.setdefault(p, slot)
        rows = torch.tensor([p - q0 for p in where], dtype=torch.long, device="cuda")
        slots = torch.tensor(list(where.values()), dtype=torch.long, device="cuda")
        col = torch.arange(Lk, device="cuda")
        for h in range(Hkv):
            k, v = _values64(s["k8"][b, h], s["kx"][b, h]), _values64(s["v8"][b, h], s["vx"][b, h])
            for hq in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                q = s["q"][b, hq].double()
                z = q @ k.T
                if S:
                    z[rows, rows + q0] = (q[rows] * s["km"][b, h, slots].double()).sum(-1)
                z = z * 128 ** -0.5
                if c["cap"] > 0:
                    z = torch.tanh(z / c["cap"]) * c["cap"]
                if s["lo"] is not None:
                    z[(col < s["lo"][b, :, None]) | (col >= s["hi"][b, :, None])] = -math.inf
                total = torch.logsumexp(z, -1)
                w = torch.exp(z - total[:, None])
                w[total == -math.inf] = 0
                y = w @ v
                if S:
                    y[rows] += w[rows, rows + q0][:, None] * (s["vm"][b, h, slots].double() - v[rows + q0])
                out[b, hq], lse[b, hq] = y, total
    return out, lse
