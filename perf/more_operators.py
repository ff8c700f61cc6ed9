"""Serving from a paged key/value memory, and log probabilities of given tokens with their gradient.

A server keeps the keys and values of many sequences in one pool of pages. A page holds ``page`` consecutive positions of
one sequence, k_pages, v_pages [n_pages, Hkv, page, D] in bf16; table [B, M] names a sequence's pages in order, and an
entry outside the pool (-1) is a page that it does not have. A step's layer appends the new rows (rotated to their
positions on the way) and lets the step's queries attend over the sequence's pages; behind the last layer the log
probabilities of given tokens are read off the logits, with the entropy and the best alternatives, and where the
program learns from them (distillation, policy gradients) their gradient goes back into the logits.

Kinds of cases and their fields:
  append  n new rows k, v [B, Hkv, n, D] of every sequence, as a projection leaves them ([B, n, H, D] in memory), and its
          queries [B, Hq, n, D]: k and q are rotated by R of D columns (``inter``: pairs of neighbours, else of halves; R = 0: not
          at all), k and v written to the pages. Rows lie behind what the sequence has, counts of them a sequence
          (``ragged``: the others are padding), or at ``listed`` positions, of which some are outside the
          pages or named twice (the lowest row is taken).
  attn    Lq queries of every sequence, at its last positions, over its length of at most Lk keys in pages; S seed positions
          with their masked-input pairs; ``mask``: a row sees its sequence's keys (none), those up to itself (causal), its block
          of 64 and those before (blocks), or the 1024 up to itself (window); ``cap``: scores capped. With four
          sequences and more one is empty.
  logp    N rows of V logits, a token each: its log probability, the row's entropy and logsumexp, the K best
          tokens (ties to the lowest index) with theirs.
  grad    the gradient of those in the logits.
"""
import math

import torch

own = False


def listed():
    return [
        # one token of every sequence of a batch: latency is all
        dict(name="append_token", kind="append", dtype="bf16", B=16, Hq=28, Hkv=4, n=1, D=128, R=128, inter=False, page=16,
             far=8000, listed=False, ragged=False),
        # the seeds' cached fp32 rows, put into the memories of a batch at their positions
        dict(name="append_seeds", kind="append", dtype="f32", B=8, Hq=0, Hkv=32, n=63, D=64, R=0, inter=False, page=64,
             far=2000, listed=True, ragged=False),
        # prompts of a batch, padded to the longest
        dict(name="append_prompt", kind="append", dtype="bf16", B=4, Hq=32, Hkv=8, n=8191, D=128, R=128, inter=False, page=64,
             far=100, listed=False, ragged=True),
        # one token of one short sequence
        dict(name="attn_token", kind="attn", B=1, Hq=28, Hkv=4, Lq=1, Lk=777, S=0, page=16, mask="none", cap=0.0),
        # the active block of one sequence, verified with seeds
        dict(name="attn_block_seeds", kind="attn", B=1, Hq=28, Hkv=4, Lq=32, Lk=1024, S=32, page=64, mask="none", cap=0.0),
        # a token of every sequence of a server's batch
        dict(name="attn_batch", kind="attn", B=64, Hq=32, Hkv=8, Lq=1, Lk=8191, S=0, page=16, mask="none", cap=0.0),
        # tokens over long memories
        dict(name="attn_token_long", kind="attn", B=4, Hq=32, Hkv=8, Lq=1, Lk=131072, S=0, page=128, mask="none", cap=0.0),
        # a prompt's last part, in blocks that see themselves and those before, scores capped
        dict(name="attn_prompt", kind="attn", B=1, Hq=32, Hkv=8, Lq=2048, Lk=8192, S=64, page=32, mask="blocks", cap=30.0),
        # what the next token could have been
        dict(name="logp_token", kind="logp", dtype="bf16", N=1, V=152064, K=20),
        # a batch's answers, scored
        dict(name="logp_batch", kind="logp", dtype="bf16", N=2048, V=126464, K=8),
        # a small fp32 head of an odd vocabulary, with the alternatives' gradients
        dict(name="grad_small", kind="grad", dtype="f32", N=64, V=20001, K=5),
        # a training batch
        dict(name="grad_batch", kind="grad", dtype="bf16", N=2048, V=126464, K=0),
    ]


HEADS = [(32, 32), (28, 4), (32, 8), (16, 2)]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attn", "attn", "attn", "logp", "grad"])
    Hq, Hkv = rng.choice(HEADS)
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "append":
        D, by = rng.choice([64, 128]), rng.random() < 0.3
        while True:
            B, n, dtype, far = _log(rng, 1, 64), _log(rng, 1, 512 if by else 8192), rng.choice(["bf16", "f32"]), _log(rng, 1, 60000)
            if B * n * (Hq + Hkv) * D * (2 if dtype == "bf16" else 4) < 160e6 and B * (n + far) * Hkv * D < 134e6:
                break
        return dict(kind=kind, dtype=dtype, B=B, Hq=0 if by else Hq, Hkv=Hkv, n=n, D=D, R=0 if by else rng.choice([D, D, D // 2]),
                    inter=rng.random() < 0.5, page=page, far=far, listed=by, ragged=not by and rng.random() < 0.5)
    if kind == "attn":
        while True:
            B, Lq = _log(rng, 1, 64), 1 if rng.random() < 0.4 else _log(rng, 2, 1024)
            Lk = Lq + _log(rng, 16, 65536)
            if B * Hkv * Lk < 2.0e6 and 512.0 * B * Hq * Lq * Lk < 2e11 and 4.0 * B * Hq * Lq * Lk < 4e9:
                break
        return dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, Lq=Lq, Lk=Lk, S=0 if rng.random() < 0.5 else min(Lk // 2, _log(rng, 1, 64)),
                    page=page, mask=rng.choice(["none", "none", "causal", "blocks", "window"]), cap=rng.choice([0.0, 0.0, 30.0, 50.0]))
    while True:
        N, V, dtype = _log(rng, 1, 4096), _log(rng, 1000, 160000), rng.choice(["bf16", "f32"])
        if N * V * (2 if dtype == "bf16" else 4) < 500e6:
            break
    return dict(kind=kind, dtype=dtype, N=N, V=V, K=rng.choice([0, 1, 5, 20, 64]))


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _rows(g, B, H, n, D, dtype):
    """Rows of n tokens as a projection leaves them ([B, n, H, D] in memory), as [B, H, n, D]; a few columns are
    larger than the others, as keys' are."""
    x = torch.randn((B, n, H, D), generator=g, device="cuda")
    return (x * (1 + 6 * (torch.rand(D, generator=g, device="cuda") < 0.04))).to(dtype).transpose(1, 2)


def _lengths(c):
    """Keys of each sequence: of the first the most, of the others 0.1 to 1 of it; of four and more the last but one is empty."""
    lens = [c["Lk"]] + [max(c["Lq"], int(c["Lk"] * (0.1 + 0.9 * (0.618034 * b % 1)))) for b in range(1, c["B"])]
    if c["B"] >= 4:
        lens[-2] = 0
    return lens


def _pool(g, tokens, H, page, D):
    """A pool of pages that other sequences have used, and a table of pages in no order for sequences of so many tokens."""
    need = [-(-t // page) for t in tokens]
    n_pages, M = sum(need) + 3, max(max(need), 1)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(tokens), M), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    k, v = (torch.randn((n_pages, H, page, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    k *= (1 + 6 * (torch.rand(D, generator=g, device="cuda") < 0.04)).to(torch.bfloat16)
    return k, v, table


def _prepare_append(c, g):
    B, n = c["B"], c["n"]
    start = [int(c["far"] * (0.25 + 0.75 * (0.618034 * (b + 1) % 1))) for b in range(B)]
    counts = [n if not c["ragged"] or b == 0 else int(n * (0.3 + 0.7 * (0.618034 * b % 1))) for b in range(B)]
    kp, vp, table = _pool(g, [s + n for s in start], c["Hkv"], c["page"], c["D"])
    dt = _type(c["dtype"])
    s = dict(case=c, k=_rows(g, B, c["Hkv"], n, c["D"], dt), v=_rows(g, B, c["Hkv"], n, c["D"], dt), q=None, kp=kp, vp=vp,
             table=table, start=None, count=None, at=None, f=None)
    if c["Hq"]:
        s["q"] = _rows(g, B, c["Hq"], n, c["D"], dt)
    if c["R"]:
        s["f"] = 10000.0 ** (-2.0 * torch.arange(c["R"] // 2, dtype=torch.float64, device="cuda") / c["R"])
    if c["listed"]:
        at = torch.stack([torch.randperm(x + n, generator=g, device="cuda")[:n] for x in start]).to(torch.int32)
        if n >= 16:
            at[:, n // 2] = at[:, 1]
            at[:, n - 1] = at[:, n // 3]
            at[:, 5] = -1
            at[:, n // 2 + 1] = table.shape[1] * c["page"] + 3
        s["at"] = at
    else:
        s["start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
        if c["ragged"]:
            s["count"] = torch.tensor(counts, dtype=torch.int32, device="cuda")
    return s


def _prepare_attn(c, g):
    B, Hkv, Lq, Lk, S = c["B"], c["Hkv"], c["Lq"], c["Lk"], c["S"]
    lens = _lengths(c)
    kp, vp, table = _pool(g, lens, Hkv, c["page"], 128)
    lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q0 = (lens - Lq).clamp(min=0)
    s = dict(case=c, kp=kp, vp=vp, table=table, lens=lens, q0=q0, lo=None, hi=None, seeds=None, km=None, vm=None,
             q=torch.randn((B, c["Hq"], Lq, 128), generator=g, device="cuda").to(torch.bfloat16))
    if S > 0:
        order = torch.rand((B, Lk), generator=g, device="cuda")
        at = torch.arange(Lk, device="cuda")
        order = order - 0.7 * ((at >= q0[:, None]) & (at < q0[:, None] + Lq))   # most seeds are in the active rows
        s["seeds"] = order.argsort(1)[:, :S].to(torch.int32).contiguous()
        if S >= 4:
            s["seeds"][:, S - 1] = -1         # fewer were selected than the list has room for
        s["km"], s["vm"] = (torch.randn((B, Hkv, S, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    pos = q0[:, None] + torch.arange(Lq, device="cuda", dtype=torch.int32)
    if c["mask"] in ("causal", "window"):
        s["hi"] = (pos + 1).contiguous()
    if c["mask"] == "window":
        s["lo"] = (pos - 1023).contiguous()
    if c["mask"] == "blocks":
        s["hi"] = ((pos // 64 + 1) * 64).contiguous()
    return s


def _prepare_logits(c, g):
    N, V, K = c["N"], c["V"], c["K"]
    x = torch.randn((N, V), generator=g, device="cuda") * 1.5
    peak = torch.randint(0, V, (N, 4), generator=g, device="cuda")
    x.scatter_add_(1, peak, 14 * torch.rand((N, 4), generator=g, device="cuda"))   # some rows are sure, some are not
    x[:, V - V // 100:] = -math.inf                                                # the vocabulary's padding
    x = x.to(_type(c["dtype"]))
    tok = torch.where(torch.rand(N, generator=g, device="cuda") < 0.5, peak[:, 0],
                      torch.randint(0, V - V // 100, (N,), generator=g, device="cuda"))
    tok = torch.minimum(tok, torch.tensor(V - V // 100 - 1, device="cuda")).to(torch.int32)
    if N >= 8:
        tok[N // 3] = -1                                                           # a row without a token
    s = dict(case=c, x=x, tok=tok)
    if c["kind"] == "grad":
        d = x.double()
        top = d.amax(1, keepdim=True)
        p = torch.exp(d - top)
        total = p.sum(1, keepdim=True)
        p /= total
        s["lse"] = (top + torch.log(total))[:, 0].float()
        s["ent"] = -(p * torch.where(p > 0, torch.log(p.clamp(min=1e-300)), 0.0)).sum(1).float()
        s["g_logp"], s["g_ent"] = (torch.randn(N, generator=g, device="cuda") for _ in range(2))
        s["idx"], s["g_top"] = None, None
        if K:
            s["idx"] = torch.randint(0, V, (N, K), generator=g, device="cuda").to(torch.int32)
            s["idx"][:, 0] = tok.clamp(min=0)
            s["g_top"] = torch.randn((N, K), generator=g, device="cuda")
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"append": _prepare_append, "attn": _prepare_attn, "logp": _prepare_logits, "grad": _prepare_logits}[case["kind"]](case, g)


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------

def _positions(s):
    """[B, n] of the rows in the memory, -1 for those that are not written (not held to the pages)."""
    c = s["case"]
    row = torch.arange(c["n"], device="cuda")
    if s["at"] is not None:
        same = s["at"][:, :, None] == s["at"][:, None, :]
        return torch.where((same & (row[None, :] < row[:, None])).any(-1), -1, s["at"].long())
    at = s["start"].long()[:, None] + row
    return at if s["count"] is None else torch.where(row < s["count"][:, None], at, -1)


def _turned(x, c, cos, sin):
    """x [B, H, n, D] with its first R columns turned by angles whose cos, sin are [B, 1, n, R / 2], in fp32."""
    R, f = c["R"], x.float()
    if R == 0:
        return f
    a, b = (f[..., 0:R:2], f[..., 1:R:2]) if c["inter"] else (f[..., :R // 2], f[..., R // 2:R])
    ya, yb = a * cos - b * sin, a * sin + b * cos
    y = torch.stack((ya, yb), -1).flatten(-2) if c["inter"] else torch.cat((ya, yb), -1)
    return torch.cat((y, f[..., R:]), -1)


def _append(s):
    c = s["case"]
    at, M, n_pages = _positions(s), s["table"].shape[1], s["kp"].shape[0]
    fine = (at >= 0) & (at < M * c["page"])
    page = s["table"].long().gather(1, torch.where(fine, at // c["page"], 0))
    fine = fine & (page >= 0) & (page < n_pages)
    cos = sin = None
    if c["R"]:
        where = s["at"].long() if s["at"] is not None else s["start"].long()[:, None] + torch.arange(c["n"], device="cuda")
        angle = where.double()[:, None, :, None] * s["f"]
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    b, r = fine.nonzero(as_tuple=True)
    for x, pages in ((_turned(s["k"], c, cos, sin), s["kp"]), (s["v"].float(), s["vp"])):
        pages[page[b, r], :, at[b, r] % c["page"]] = x[b, :, r].to(torch.bfloat16)
    q = None if s["q"] is None else _turned(s["q"], c, cos, sin).to(s["q"].dtype).contiguous()
    return tuple(t for t in (q, s["kp"], s["vp"]) if t is not None)


def _gathered(s, pages):
    """[B, Hkv, M * page, D] in fp32: the rows of every sequence's pages (of page 0 where it has none)."""
    n_pages, Hkv, page, D = pages.shape
    t = s["table"].long()
    rows = pages[torch.where((t >= 0) & (t < n_pages), t, 0)]            # [B, M, Hkv, page, D]
    return rows.transpose(1, 2).reshape(t.shape[0], Hkv, -1, D).float()


def _attention(s):
    c = s["case"]
    B, Hq, Hkv, Lq, S = c["B"], c["Hq"], c["Hkv"], c["Lq"], c["S"]
    G = Hq // Hkv
    k, v = _gathered(s, s["kp"]), _gathered(s, s["vp"])
    L = k.shape[2]
    q = s["q"].float().view(B, Hkv, G, Lq, 128)
    z = torch.matmul(q.view(B, Hkv, G * Lq, 128), k.transpose(2, 3)).view(B, Hkv, G, Lq, L) / math.sqrt(128)
    at = torch.arange(L, device=z.device)
    pos = s["q0"].long()[:, None] + torch.arange(Lq, device=z.device)     # [B, Lq]
    if S > 0:
        same = s["seeds"].long()[:, None, :] == pos[:, :, None]           # [B, Lq, S]
        is_seed = same.any(-1)
        slot = same.float().argmax(-1)                                    # the lowest slot of the position
        take = slot[:, None, :, None].expand(B, Hkv, Lq, 128)
        ks, vs = s["km"].float().gather(2, take), s["vm"].float().gather(2, take)
        z_self = (q * ks[:, :, None]).sum(-1) / math.sqrt(128)            # [B, Hkv, G, Lq]
        swap = (is_seed[:, :, None] & (at == pos[:, :, None]))[:, None, None]
        z = torch.where(swap, z_self[..., None], z)
    if c["cap"] > 0:
        z = c["cap"] * torch.tanh(z / c["cap"])
    seen = (at < s["lens"][:, None, None]).expand(B, Lq, L)
    if s["lo"] is not None:
        seen = seen & (at >= s["lo"][..., None])
    if s["hi"] is not None:
        seen = seen & (at < s["hi"][..., None])
    z = z.masked_fill(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    w = p / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total)).view(B, Hq, Lq)
    if S > 0:
        w_self = torch.where(swap, w, 0.0).sum(-1, keepdim=True)
        w = torch.where(swap, 0.0, w)
    o = torch.matmul(w.view(B, Hkv, G * Lq, L), v).view(B, Hkv, G, Lq, 128)
    if S > 0:
        o = o + w_self * vs[:, :, None]
    return o.reshape(B, Hq, Lq, 128).to(torch.bfloat16), lse


def _logp(s):
    c, x = s["case"], s["x"].float()
    top = x.amax(1, keepdim=True)
    t = x - top
    e = torch.exp(t)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    entropy = log_total - torch.where(e > 0, e * t, 0.0).sum(1, keepdim=True) / total
    has = (s["tok"] >= 0) & (s["tok"] < c["V"])
    picked = t.gather(1, torch.where(has, s["tok"], 0).long()[:, None]) - log_total
    out = [torch.where(has, picked[:, 0], 0.0), entropy[:, 0], (top + log_total)[:, 0]]
    if c["K"]:
        best, idx = x.sort(stable=True, dim=1, descending=True)
        out += [idx[:, :c["K"]].to(torch.int32), best[:, :c["K"]] - top - log_total]
    return tuple(out)


def _grad(s):
    c, x = s["case"], s["x"].float()
    logp = x - s["lse"][:, None]
    p = torch.exp(logp)
    has = (s["tok"] >= 0) & (s["tok"] < c["V"])
    g_logp = torch.where(has, s["g_logp"], 0.0)
    given = g_logp if s["g_top"] is None else g_logp + s["g_top"].sum(1)
    d = -p * given[:, None] - s["g_ent"][:, None] * p * (torch.where(p > 0, logp, 0.0) + s["ent"][:, None])
    d.scatter_add_(1, torch.where(has, s["tok"], 0).long()[:, None], g_logp[:, None])
    if s["g_top"] is not None:
        for i in range(c["K"]):
            d.scatter_add_(1, s["idx"][:, i:i + 1].long(), s["g_top"][:, i:i + 1])
    return d.to(s["x"].dtype)


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2602_06161_gb300 import api
        if c["kind"] == "append":
            q, _ = api.cover_paged_append(s["k"], s["v"], s["kp"], s["vp"], s["table"], start=s["start"], count=s["count"], pos=s["at"],
                                          q=s["q"], inv_freq=s["f"], interleaved=c["inter"])
            return tuple(t for t in (q, s["kp"], s["vp"]) if t is not None)
        if c["kind"] == "attn":
            return api.cover_attn_fwd_paged(s["q"], s["kp"], s["vp"], s["table"], s["lens"], s["km"], s["vm"], s["seeds"],
                                            q0=s["q0"], key_lo=s["lo"], key_hi=s["hi"], softcap=c["cap"])
        if c["kind"] == "logp":
            r = api.cover_logprob_fwd(s["x"], s["tok"], topk=c["K"])
            return (r["logp"], r["entropy"], r["lse"]) + ((r["top_idx"], r["top_logp"]) if c["K"] else ())
        return api.cover_logprob_bwd(s["x"], s["lse"], tok=s["tok"], entropy=s["ent"], d_logp=s["g_logp"], d_entropy=s["g_ent"],
                                     top_idx=s["idx"], d_top=s["g_top"])
    return {"append": _append, "attn": _attention, "logp": _logp, "grad": _grad}[c["kind"]](s)


def work(case):
    c = case
    if c["kind"] == "append":
        B, n, e = c["B"], c["n"], 2 if c["dtype"] == "bf16" else 4
        written = sum(n if not c["ragged"] or b == 0 else int(n * (0.3 + 0.7 * (0.618034 * b % 1))) for b in range(B))
        return dict(bytes=2 * c["Hkv"] * written * c["D"] * (e + 2) + 2 * B * n * c["Hq"] * c["D"] * e + 4 * B * (n if c["listed"] else 2) +
                    4 * B * max(1, n // c["page"]) + 4 * c["R"], flops=3 * (B * n * c["Hq"] + written * c["Hkv"]) * c["R"])
    if c["kind"] == "attn":
        pairs = keys = 0
        for L in _lengths(c):
            ends = []
            for r in range(c["Lq"] if L else 0):
                at = L - c["Lq"] + r
                lo = max(0, at - 1023) if c["mask"] == "window" else 0
                hi = {"none": L, "causal": at + 1, "window": at + 1, "blocks": min(L, (at // 64 + 1) * 64)}[c["mask"]]
                ends.append((lo, hi))
            pairs += sum(hi - lo for lo, hi in ends)
            keys += ends[-1][1] - ends[0][0] if ends else 0
        rows = c["B"] * c["Hq"] * c["Lq"]
        return dict(bytes=c["Hkv"] * keys * 512 + rows * (4 * 128 + 4) + c["B"] * c["Hkv"] * c["S"] * 512 + 4 * keys // c["page"],
                    flops=512.0 * c["Hq"] * pairs)
    e, n = 2 if c["dtype"] == "bf16" else 4, c["N"] * c["V"]
    if c["kind"] == "logp":
        return dict(bytes=n * e + c["N"] * (16 + 8 * c["K"]), flops=5 * n)
    return dict(bytes=2 * n * e + c["N"] * (20 + 8 * c["K"]), flops=6 * n)


# ------------------------------------------------------------------------------------------------
# the definitions, in 64 bits
# ------------------------------------------------------------------------------------------------

def _exact_append(c, s):
    B, n, page = c["B"], c["n"], c["page"]
    at = s["at"].tolist() if c["listed"] else [[x + r for r in range(n)] for x in s["start"].tolist()]
    counts = [n] * B if s["count"] is None else s["count"].tolist()
    tables = s["table"].tolist()

    def rotated(x):
        y = x.double().contiguous()
        if c["R"]:
            i = torch.arange(c["R"] // 2, device="cuda")
            a, b = (2 * i, 2 * i + 1) if c["inter"] else (i, i + c["R"] // 2)
            angle = torch.tensor(at, dtype=torch.float64, device="cuda")[:, None, :, None] * s["f"]
            z = torch.complex(y[..., a], y[..., b]) * torch.polar(torch.ones_like(angle), angle)
            y[..., a], y[..., b] = z.real, z.imag
        return y

    outs = [] if s["q"] is None else [rotated(s["q"])]
    for x, pages in ((rotated(s["k"]), s["kp"]), (s["v"].double(), s["vp"])):
        y = pages.double()
        for b in range(B):
            first = {}
            for r in range(counts[b]):
                p = at[b][r]
                if 0 <= p < len(tables[b]) * page and 0 <= tables[b][p // page] < y.shape[0]:
                    first.setdefault(p, r)
            if first:
                where, rows = list(first), list(first.values())
                y[[tables[b][p // page] for p in where], :, [p % page for p in where]] = x[b][:, rows].transpose(0, 1)
        outs.append(y)
    return tuple(outs)


def _exact_attn(c, s):
    B, Hq, Hkv, Lq, S = c["B"], c["Hq"], c["Hkv"], c["Lq"], c["S"]
    out = torch.zeros((B, Hq, Lq, 128), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq, Lq), -math.inf, dtype=torch.float64, device="cuda")
    for b, L in enumerate(s["lens"].tolist()):
        if L == 0:
            continue
        pages = s["table"][b, :-(-L // c["page"])].long()
        first = int(s["q0"][b])
        where = {}
        for slot, p in enumerate(s["seeds"][b].tolist() if S else []):
            if first <= p < first + Lq:
                where.setdefault(p - first, slot)
        rows = torch.tensor(list(where), dtype=torch.long, device="cuda")
        slots = torch.tensor(list(where.values()), dtype=torch.long, device="cuda")
        col = torch.arange(L, device="cuda")
        hidden = torch.zeros((Lq, L), dtype=torch.bool, device="cuda")
        if s["lo"] is not None:
            hidden |= col < s["lo"][b, :, None]
        if s["hi"] is not None:
            hidden |= col >= s["hi"][b, :, None]
        for h in range(Hkv):
            k, v = (x[pages, h].reshape(-1, 128)[:L].double() for x in (s["kp"], s["vp"]))
            for hq in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                q = s["q"][b, hq].double()
                z = q @ k.T
                if len(where):
                    z[rows, rows + first] = (q[rows] * s["km"][b, h, slots].double()).sum(-1)
                z = z * 128 ** -0.5
                if c["cap"] > 0:
                    z = torch.tanh(z / c["cap"]) * c["cap"]
                z[hidden] = -math.inf
                total = torch.logsumexp(z, -1)
                w = torch.exp(z - total[:, None])
                w[total == -math.inf] = 0
                y = w @ v
                if len(where):
                    y[rows] += w[rows, rows + first][:, None] * (s["vm"][b, h, slots].double() - v[rows + first])
                out[b, hq], lse[b, hq] = y, total
    return out, lse


def _exact_logits(c, s):
    outs = []
    V = c["V"]
    for i in range(0, c["N"], 64):
        x, tok = s["x"][i:i + 64].double(), s["tok"][i:i + 64].long()
        lp = torch.log_softmax(x, 1) if c["kind"] == "logp" else x - s["lse"][i:i + 64].double()[:, None]
        p, zero = torch.exp(lp), torch.zeros((), dtype=torch.float64, device="cuda")
        has = (tok >= 0) & (tok < V)
        if c["kind"] == "logp":
            got = [torch.where(has, lp.gather(1, tok.clamp(0, V - 1)[:, None])[:, 0], zero),
                   -torch.special.xlogy(p, p).sum(1), torch.logsumexp(x, 1)]
            if c["K"]:
                idx = torch.argsort(-x, dim=1, stable=True)[:, :c["K"]]
                got += [idx.to(torch.int32), lp.gather(1, idx)]
            outs.append(got)
            continue
        cols = torch.arange(V, device="cuda")
        hit = ((cols == tok[:, None]).double() - p) * torch.where(has, s["g_logp"][i:i + 64].double(), zero)[:, None]
        hit -= (torch.special.xlogy(p, p) + p * s["ent"][i:i + 64].double()[:, None]) * s["g_ent"][i:i + 64].double()[:, None]
        for k in range(c["K"]):
            hit += ((cols == s["idx"][i:i + 64, k:k + 1]).double() - p) * s["g_top"][i:i + 64, k:k + 1].double()
        outs.append([hit])
    whole = [torch.cat(x) for x in zip(*outs)]
    return tuple(whole) if c["kind"] == "logp" else whole[0]


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "logp": _exact_logits, "grad": _exact_logits}[case["kind"]](case, s)
