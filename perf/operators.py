"""Exponential attention and the paged cache that it decodes from, as a program uses them: a forward pass, a training step,
keys and values going into the cache, a prompt taken piece by piece, one new token for every sequence.

Weights are exp(s_ij) with s_ij = scale q_i.k_j, or cap tanh(scale q_i.k_j / cap), minus slope_h |pos_i - j|; query i of T stands
at pos_i = i + Tk - T among Tk keys and sees lo_i <= j < hi_i (documents, prefixes; causal without them) and j > pos_i - window.
Head h of H reads key head h Hk / H of Hk.

Inputs are drawn on the GPU from the seed: k, v ~ N(0, 1), q ~ sharp N(0, 1), dO ~ N(0, 1), scale = d^-1/2.

A case is a dict:
  kind      "fwd" forward pass, "train" forward and backward, "append" rows into the cache and read back as the values held,
            "piece" the last T tokens of a prompt of Tk: into the cache, the whole context read back, attention; "step" one
            token for every sequence
  B, H, Hk, T, Tk, d; cap, window (0: none), bias (slopes 2^(-8 (h + 1) / H)), sharp
  docs      documents that every row of the batch is packed from (0: one, no mask); a tenth of the row is padding behind them
  prefix    share of every document that all of its tokens see
  bits      16 or 4 per cached value; page: tokens per page; ragged: lengths differ by sequence; rot: channels rotated
In "append" and "step" a sequence holds up to Tk tokens, the call's own among them.
"""
import math
import random

import torch

own = False

GROUP = 32      # channels of one scale and minimum of a 4-bit row


def _case(name, kind, B, H, Hk, T, d, Tk=None, cap=0.0, window=0, bias=False, sharp=1.0, docs=0, prefix=0.0, bits=16, page=64,
          ragged=False, rot=0):
    c = dict(kind=kind, B=B, H=H, Hk=Hk, T=T, Tk=T if Tk is None else Tk, d=d, cap=cap, window=window, bias=bias, sharp=sharp,
             docs=docs, prefix=prefix, bits=bits, page=page, ragged=ragged, rot=rot)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a short prompt through one layer of a small model: launches and latency
        _case("fwd_T200_d64", "fwd", 1, 4, 4, 200, 64),
        # prefill of a batch with a sliding window of 1024, the comparison system of the paper at the benchmark's second shape
        _case("fwd_window_T8192_d64", "fwd", 4, 12, 12, 8192, 64, window=1024, sharp=2.0),
        # a batch of texts, each row packed from two and padded: short, odd, rows that see nothing
        _case("train_padded_T1000_d64", "train", 16, 12, 12, 1000, 64, docs=2, sharp=2.0),
        # training on packed documents, capped scores, four query heads to a key head
        _case("train_docs_T8192_d128", "train", 2, 16, 4, 8192, 128, docs=7, cap=20.0, sharp=4.0),
        # a prefix seen by all of its document, distance bias, an odd length
        _case("train_prefix_T4095_d64", "train", 2, 12, 4, 4095, 64, docs=3, prefix=0.25, bias=True, sharp=2.0),
        # the long training step, heads as wide as the benchmark's fifth shape: the largest case
        _case("train_T16384_d128", "train", 1, 16, 8, 16384, 128, sharp=2.0),
        # decoding: one new token of 64 sequences into the cache
        _case("append_B64_T1_d128", "append", 64, 16, 4, 1, 128, Tk=2000, ragged=True, rot=128),
        # prompts of different lengths into a cache of 4 bits
        _case("append_B4_T3000_d128_4bit", "append", 4, 16, 4, 3000, 128, Tk=3500, bits=4, ragged=True, rot=128),
        # a long prompt comes in pieces of 1024 tokens: the last of eight
        _case("piece_T1024_Tk8192_d128", "piece", 1, 16, 4, 1024, 128, Tk=8192, cap=20.0, sharp=4.0, rot=64),
        # decoding for one user, short context: latency
        _case("step_B1_T500_d64", "step", 1, 12, 12, 1, 64, Tk=500, sharp=2.0),
        # decoding for 32 users of different lengths, capped scores with distance bias
        _case("step_B32_T16384_d128", "step", 32, 16, 4, 1, 128, Tk=16384, cap=20.0, bias=True, sharp=4.0, ragged=True),
        # long contexts held in 4 bits, the largest read
        _case("step_B4_T131072_d128_4bit", "step", 4, 32, 8, 1, 128, Tk=131072, sharp=2.0, bits=4, page=128),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    while True:
        kind = rng.choice(["fwd", "train", "train", "append", "piece", "step", "step"])
        d = rng.choice([64, 128]) if kind in ("append", "piece", "step") else rng.choice([32, 64, 128])
        Hk = rng.choice([1, 2, 3, 4, 8])
        H = Hk * rng.choice([1, 2, 3, 4, 8])
        cap = rng.choice([0.0, 0.0, 15.0, 30.0])
        bias, sharp = rng.random() < 0.3, rng.choice([1.0, 2.0, 4.0])
        window = rng.choice([0, 0, int(_log(rng, 16, 4000))])
        bits, page, ragged, rot = rng.choice([16, 4]), rng.choice([32, 64, 128, 256]), rng.random() < 0.6, rng.choice([0, 32, d])
        if kind in ("fwd", "train"):
            T = int(_log(rng, 1, 16384))
            docs = rng.choice([0, 0, 2, 5]) if T >= 40 else 0
            c = _case(None, kind, int(_log(rng, 1, 16)), H, Hk, T, d, cap=cap, window=window, bias=bias, sharp=sharp, docs=docs,
                      prefix=rng.choice([0.0, 0.3]) if docs else 0.0)
        elif kind == "append":
            T = int(_log(rng, 1, 4000))
            c = _case(None, kind, int(_log(rng, 1, 64)), H, Hk, T, d, Tk=T + int(_log(rng, 1, 3000)), bits=bits, page=page, ragged=ragged,
                      rot=rot)
        elif kind == "piece":
            T = int(_log(rng, 1, 2000))
            c = _case(None, kind, 1, H, Hk, T, d, Tk=T + int(_log(rng, 1, 12000)), cap=cap, window=window, bias=bias, sharp=sharp,
                      bits=bits, page=page, rot=rot)
        else:
            c = _case(None, kind, int(_log(rng, 1, 64)), H, Hk, 1, d, Tk=int(_log(rng, 1, 131072)), cap=cap, window=window, bias=bias,
                      sharp=sharp, bits=bits, page=page, ragged=ragged)
        most, w = _most(), work(c)
        held = c["B"] * c["Hk"] * c["Tk"] * c["d"] * 4
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"] and held <= 3 << 30:
            return c


def _most():
    ws = [work(c) for c in listed()]
    return {k: max(w[k] for w in ws) for k in ("flops", "bytes")}


# ---- lengths and masks, from the case alone ------------------------------------------------------------------------------
def _documents(case, b):
    """Lengths of the documents of row b."""
    T, n = case["T"], case["docs"]
    rng = random.Random(1000 * n + b)
    cuts = sorted(rng.sample(range(1, T - T // 10), n - 1))
    return [e - s for s, e in zip([0] + cuts, cuts + [T - T // 10])]


def _rows(case):
    """lo, hi [B, T] int32 on the host, or None, None."""
    if not case["docs"]:
        return None, None
    B, T = case["B"], case["T"]
    lo, hi = torch.zeros(B, T, dtype=torch.int32), torch.zeros(B, T, dtype=torch.int32)
    for b in range(B):
        at = 0
        for n in _documents(case, b):
            lo[b, at:at + n] = at
            hi[b, at:at + n] = torch.arange(at + 1, at + n + 1).clamp(min=at + math.ceil(case["prefix"] * n))
            at += n
    return lo, hi


def _shares(case, salt):
    """One number in (0, 1] for every sequence; 1 where lengths do not differ."""
    rng = random.Random(salt * 7919 + case["B"])
    return [rng.uniform(0.1, 1.0) if case["ragged"] else 1.0 for _ in range(case["B"])]


def _lengths(case):
    """Tokens held before the call, and tokens of the call, by sequence."""
    past = [int((case["Tk"] - case["T"]) * x) for x in _shares(case, 1)]
    count = [max(1, int(case["T"] * x)) for x in _shares(case, 2)]
    return past, count


def work(case):
    B, H, Hk, T, Tk, d, kind = (case[k] for k in ("B", "H", "Hk", "T", "Tk", "d", "kind"))
    held = 2 * d if case["bits"] == 16 else d // 2 + 4 * d // GROUP
    past, count = _lengths(case)
    tokens = sum(count)
    if kind == "append":
        # rows in, rows into the cache, rotated queries and the rows' values out, the angles once
        return {"bytes": 2 * tokens * d * (H + 2 * Hk) + 2 * tokens * Hk * held + 2 * tokens * d * (H + 2 * Hk)
                + 4 * tokens * case["rot"], "flops": 3 * tokens * case["rot"] * (H + Hk)}
    if kind == "step":
        seen = sum(min(p + 1, case["window"]) if case["window"] else p + 1 for p in past)
        return {"bytes": 2 * seen * Hk * held + 4 * B * H * d + 4 * B * H, "flops": 4 * seen * H * d}
    pos = torch.arange(T, dtype=torch.int64) + (Tk - T)
    lo, hi = _rows(case)
    lo = torch.zeros(B, T, dtype=torch.int64) if lo is None else lo.long()
    hi = (pos + 1).expand(B, T) if hi is None else hi.long()
    if case["window"]:
        lo = torch.maximum(lo, pos - case["window"] + 1)
    pairs = int((hi - lo).clamp(min=0).sum())
    qo, kv = 2 * B * H * T * d, 2 * B * Hk * Tk * d
    if kind == "fwd":
        return {"bytes": 2 * qo + 2 * kv + 4 * B * H * T, "flops": 4 * pairs * H * d}
    if kind == "train":     # q, k, v, dO; O, dQ, dK, dV; scores and four products of gradients beside the forward's two
        return {"bytes": 4 * qo + 4 * kv, "flops": 14 * pairs * H * d}
    # piece: its rows in and into the cache, the context out as values, attention over it
    return {"bytes": 3 * qo + 2 * tokens * Hk * (2 * d + held) + 2 * Tk * Hk * held + 2 * kv + 4 * H * T + 4 * tokens * case["rot"],
            "flops": 4 * pairs * H * d}


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _normal(gen, *shape, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).bfloat16()


def _inputs(case, seed):
    """What both sides and the exact form get: a dict of tensors on the GPU."""
    B, H, Hk, T, Tk, d, kind = (case[k] for k in ("B", "H", "Hk", "T", "Tk", "d", "kind"))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = {"q": _normal(gen, B, H, T, d, scale=case["sharp"]), "slopes": None, "lo": None, "hi": None}
    if case["bias"]:
        x["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device="cuda")
    lo, hi = _rows(case)
    if lo is not None:
        x["lo"], x["hi"] = lo.cuda(), hi.cuda()
    if kind in ("fwd", "train"):
        x["k"], x["v"] = _normal(gen, B, Hk, T, d), _normal(gen, B, Hk, T, d)
        if kind == "train":
            x["g"] = _normal(gen, B, H, T, d)
        return x
    page = case["page"]
    x["pages"] = (Tk + page - 1) // page
    x["table"] = torch.randperm(B * x["pages"], generator=gen, device="cuda").int().view(B, x["pages"])
    past, count = _lengths(case)
    x["past"], x["count"] = (torch.tensor(n, dtype=torch.int32, device="cuda") for n in (past, count))
    if kind == "step":
        # the context, the new token's own row (position `past`) among it
        x["ctx_k"], x["ctx_v"] = _normal(gen, B, Hk, Tk, d), _normal(gen, B, Hk, Tk, d)
        return x
    x["k"], x["v"] = _normal(gen, B, Hk, T, d), _normal(gen, B, Hk, T, d)
    if kind == "piece":
        x["ctx_k"], x["ctx_v"] = _normal(gen, B, Hk, Tk - T, d), _normal(gen, B, Hk, Tk - T, d)
    if case["rot"]:
        half = case["rot"] // 2
        turn = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        angle = torch.arange(x["pages"] * page, dtype=torch.float64, device="cuda")[:, None] * turn
        x["cos"], x["sin"] = angle.cos().float(), angle.sin().float()
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    B, H, Hk, T, Tk, d, kind = (case[k] for k in ("B", "H", "Hk", "T", "Tk", "d", "kind"))
    st = {"case": case, "scale": d ** -0.5, **x}
    if kind in ("append", "piece"):
        # rows behind a sequence's last stay what they are: zeros
        st["out_q"] = torch.zeros_like(x["q"])
        st["out_kv"] = tuple(torch.zeros(B, Hk, T if kind == "append" else Tk, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if kind in ("append", "piece", "step"):
        ctx = (x["ctx_k"], x["ctx_v"]) if "ctx_k" in x and x["ctx_k"].shape[2] > 0 else None
        if own:
            from paper_2507_04239_amd import binding
            args = dict(scale=d ** -0.5, cap=case["cap"], window=case["window"])
            st["cache"] = binding.make_cache(B, H, Hk, d, case["page"], x["pages"], B * x["pages"], bits=case["bits"], rot=case["rot"],
                                             rot_rows=x["pages"] * case["page"] if case["rot"] else 0, **args)
            fill = binding.make_cache(B, H, Hk, d, case["page"], x["pages"], B * x["pages"], bits=case["bits"], **args)
            st["pool"] = torch.zeros(binding.power_attn_cache_bytes(st["cache"]), dtype=torch.uint8, device="cuda")
            if ctx:
                binding.power_attn_cache_append(fill, *ctx, st["pool"], x["table"], torch.zeros_like(x["past"]))
            st["start"], st["lens"] = torch.zeros_like(x["past"]), x["past"] + x["count"]
        else:
            st["pool"] = _plain_pool(case, B * x["pages"])
            if ctx:
                _plain_write(st, *(c.float() for c in ctx), torch.zeros_like(x["past"]), torch.full_like(x["past"], ctx[0].shape[2]))
    for name in ("ctx_k", "ctx_v"):
        st.pop(name, None)
    return st


# ---- plain form ----------------------------------------------------------------------------------------------------------
def _plain_attend(case, q, k, v, scale, slopes, lo, hi, g=None):
    """float32 [B, H, T, d] and [B, Hk, Tk, d] -> O, L, and with g the gradients of q, k, v: a head and a block of rows at a time."""
    B, H, T, d = q.shape
    Hk, Tk = k.shape[1], k.shape[2]
    cap, window = case["cap"], case["window"]
    O, L = torch.empty_like(q), torch.empty(B, H, T, device=q.device)
    dq, dk, dv = (torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)) if g is not None else (None, None, None)
    at = torch.arange(T, device=q.device) + (Tk - T)
    keys = torch.arange(Tk, device=q.device)
    step = max(1, min(T, (1 << 27) // Tk))
    for b in range(B):
        first = torch.zeros_like(at) if lo is None else lo[b].long()
        last = at + 1 if hi is None else hi[b].long()
        if window:
            first = torch.maximum(first, at - window + 1)
        for i in range(0, T, step):
            r = slice(i, min(T, i + step))
            see = (keys >= first[r, None]) & (keys < last[r, None])
            far = (at[r, None] - keys).abs().float() if slopes is not None else None
            for h in range(H):
                kh, vh = k[b, h * Hk // H], v[b, h * Hk // H]
                s = (q[b, h, r] @ kh.T) * scale
                if cap:
                    t = torch.tanh(s / cap)
                    s = t * cap
                if slopes is not None:
                    s = s - slopes[h] * far
                s = s.masked_fill(~see, -math.inf)
                m = s.max(1, keepdim=True).values
                m = torch.where(m == -math.inf, 0.0, m)
                p = (s - m).exp()
                z = p.sum(1, keepdim=True)
                p = p / torch.where(z == 0, 1.0, z)
                O[b, h, r] = p @ vh
                L[b, h, r] = (m + z.log())[:, 0]
                if g is None:
                    continue
                gh = g[b, h, r]
                ds = p * (gh @ vh.T - (gh * O[b, h, r]).sum(1, keepdim=True))
                if cap:
                    ds = ds * (1 - t * t)
                ds = ds * scale
                dv[b, h * Hk // H] += p.T @ gh
                dk[b, h * Hk // H] += ds.T @ q[b, h, r]
                dq[b, h, r] = ds @ kh
    return O, L, dq, dk, dv


def _plain_pool(case, pages):
    """Pages of values (16 bits) or of codes with their scale and minimum (4 bits); one page more takes what is not to be kept."""
    shape = (pages + 1, case["page"], case["Hk"], case["d"])
    if case["bits"] == 16:
        return [(torch.zeros(shape, dtype=torch.bfloat16, device="cuda"),) for _ in range(2)]
    held = shape[:3] + (case["d"] // GROUP, 2)
    return [(torch.zeros(shape, dtype=torch.uint8, device="cuda"), torch.zeros(held, dtype=torch.float16, device="cuda"))
            for _ in range(2)]


def _plain_write(st, k, v, past, count):
    """Rows [B, Hk, T, d], rotated already, to positions past .. past + count - 1."""
    case, pool = st["case"], st["pool"]
    B, Hk, T, d = k.shape
    t = torch.arange(T, device="cuda")
    pos = past.long()[:, None] + t
    keep = t < count[:, None]
    page = torch.where(keep, st["table"].long().gather(1, (pos // case["page"]).clamp(max=st["pages"] - 1)), pool[0][0].shape[0] - 1)
    slot = pos % case["page"]
    for x, to in zip((k, v), pool):
        x = x.transpose(1, 2)
        if case["bits"] == 16:
            to[0][page, slot] = x.bfloat16()
            continue
        x = x.clamp(-65024.0, 65024.0).reshape(B, T, Hk, d // GROUP, GROUP)
        least = x.amin(-1)
        unit = ((x.amax(-1) - least) / 15.0).half()
        least = least.half()
        u = unit.float()[..., None]
        code = ((x - least.float()[..., None]) / torch.where(u == 0, 1.0, u)).round().clamp(0, 15)
        code = torch.where(u == 0, 0.0, code)
        to[0][page, slot] = code.to(torch.uint8).reshape(B, T, Hk, d)
        to[1][page, slot] = torch.stack([unit, least], -1)


def _plain_read(st, b, n):
    """The first n tokens of sequence b as values, float32 [Hk, n, d] each."""
    case = st["case"]
    pages = st["table"][b, :(n + case["page"] - 1) // case["page"]].long()
    out = []
    for held in st["pool"]:
        x = held[0][pages].flatten(0, 1)[:n].float()
        if case["bits"] == 4:
            sm = held[1][pages].flatten(0, 1)[:n].float()
            x = (x.unflatten(-1, (-1, GROUP)) * sm[..., :1] + sm[..., 1:]).flatten(-2)
        out.append(x.transpose(0, 1))
    return out


def _plain_rotate(st, x):
    """float32 [B, h, T, d] at positions past ..: channel c < rot / 2 turns with channel c + rot / 2"""
    rot = st["case"]["rot"]
    if not rot:
        return x
    t = st["past"].long()[:, None] + torch.arange(x.shape[2], device="cuda")
    t = t.clamp(max=st["cos"].shape[0] - 1)
    c, s = st["cos"][t][:, None], st["sin"][t][:, None]
    a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    return torch.cat([a * c - b * s, b * c + a * s, x[..., rot:]], -1)


def _plain_append(st):
    """-> rotated q [B, H, T, d], zeros behind the last row of a sequence"""
    _plain_write(st, _plain_rotate(st, st["k"].float()), st["v"].float(), st["past"], st["count"])
    q = _plain_rotate(st, st["q"].float())
    keep = torch.arange(q.shape[2], device="cuda") < st["count"][:, None]
    return torch.where(keep[:, None, :, None], q, 0.0).bfloat16()


def _plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind in ("fwd", "train"):
        q, k, v = (st[n].float() for n in "qkv")
        g = st["g"].float() if kind == "train" else None
        O, L, dq, dk, dv = _plain_attend(case, q, k, v, st["scale"], st["slopes"], st["lo"], st["hi"], g)
        return (O.bfloat16(), L) if g is None else tuple(x.bfloat16() for x in (O, dq, dk, dv))
    past, count = _lengths(case)
    B, H, Hk, T, d = (case[n] for n in ("B", "H", "Hk", "T", "d"))
    if kind == "append":
        q = _plain_append(st)
        out = [torch.zeros(B, Hk, T, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        for b in range(B):
            for to, x in zip(out, _plain_read(st, b, past[b] + count[b])):
                to[b, :, :count[b]] = x[:, past[b]:].bfloat16()
        return q, *out
    if kind == "piece":
        q = _plain_append(st)
        k, v = (x[None].bfloat16() for x in _plain_read(st, 0, case["Tk"]))
        O, L, _, _, _ = _plain_attend(case, q.float(), k.float(), v.float(), st["scale"], st["slopes"], None, None)
        return k, v, O.bfloat16(), L
    o, L = torch.empty(B, H, d, device="cuda"), torch.empty(B, H, device="cuda")
    for b in range(B):
        n = past[b] + count[b]
        k, v = _plain_read(st, b, n)
        s = (st["q"][b, :, 0].float().view(Hk, H // Hk, d) @ k.transpose(1, 2)).view(H, n) * st["scale"]
        if case["cap"]:
            s = torch.tanh(s / case["cap"]) * case["cap"]
        far = torch.arange(n - 1, -1, -1, device="cuda")
        if st["slopes"] is not None:
            s = s - st["slopes"][:, None] * far.float()
        if case["window"]:
            s = s.masked_fill(far >= case["window"], -math.inf)
        m = s.max(1, keepdim=True).values
        p = (s - m).exp()
        z = p.sum(1, keepdim=True)
        o[b] = ((p / z).view(Hk, H // Hk, n) @ v).view(H, d)
        L[b] = (m + z.log())[:, 0]
    return o.bfloat16(), L


# ---- the framework's operators ---------------------------------------------------------------------------------------------
def _own(st):
    from paper_2507_04239_amd import binding as pa
    case = st["case"]
    kind = case["kind"]
    how = dict(scale=st["scale"], cap=case["cap"], window=case["window"], slopes=st["slopes"])
    if kind in ("fwd", "train"):
        how.update(row_lo=st["lo"], row_hi=st["hi"])
        O, L = pa.power_attn_exp_fwd(st["q"], st["k"], st["v"], **how)
        if kind == "fwd":
            return O, L
        return O, *pa.power_attn_exp_bwd(st["q"], st["k"], st["v"], O, L, st["g"], **how)
    if kind == "step":
        return pa.power_attn_cache_step(st["cache"], st["q"][:, :, 0], st["pool"], st["table"], st["lens"], slopes=st["slopes"])
    pa.power_attn_cache_append(st["cache"], st["k"], st["v"], st["pool"], st["table"], st["past"], count=st["count"], Q=st["q"],
                               cos=st.get("cos"), sin=st.get("sin"), out_q=st["out_q"])
    if kind == "append":
        k, v = pa.power_attn_cache_read(st["cache"], st["pool"], st["table"], st["past"], case["T"], count=st["count"], out=st["out_kv"])
        return st["out_q"], k, v
    k, v = pa.power_attn_cache_read(st["cache"], st["pool"], st["table"], st["start"], case["Tk"], out=st["out_kv"])
    return k, v, *pa.power_attn_exp_fwd(st["out_q"], k, v, **how)


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------------
def _exact_head(q, k, v, case, scale, slope, pos, lo, hi, g):
    """One head: float64 q [n, d], k, v [Tk, d] -> O, L and (dq, dk, dv), or None"""
    x = torch.matmul(q, k.t()) * scale
    cap = case["cap"]
    s = cap * torch.tanh(x / cap) if cap else x
    j = torch.arange(k.shape[0], device=q.device)
    dist = pos.unsqueeze(1) - j.unsqueeze(0)
    if slope is not None:
        s = s - slope * dist.abs().double()
    hidden = (j.unsqueeze(0) < lo.unsqueeze(1)) | (j.unsqueeze(0) >= hi.unsqueeze(1))
    if case["window"]:
        hidden |= dist >= case["window"]
    s[hidden] = -math.inf
    L = torch.logsumexp(s, 1)
    w = torch.exp(s - torch.where(torch.isinf(L), 0.0, L).unsqueeze(1))
    O = torch.matmul(w, v)
    if g is None:
        return O, L, None
    e = torch.matmul(g, v.t())
    t = w * (e - (w * e).sum(1, keepdim=True)) * scale
    if cap:
        t = t / torch.cosh(x / cap).square()
    return O, L, (torch.matmul(t, k), torch.matmul(t.t(), q), torch.matmul(w.t(), g))


def _exact_attend(case, q, k, v, slopes, lo, hi, g=None):
    B, H, T, d = q.shape
    Hk, Tk = k.shape[1], k.shape[2]
    O, L = torch.zeros_like(q), torch.zeros(B, H, T, dtype=torch.float64, device=q.device)
    grads = [torch.zeros_like(x) for x in (q, k, v)]
    rows = max(1, min(T, (1 << 26) // Tk))
    for b in range(B):
        for h in range(H):
            kv = h // (H // Hk)
            for i in range(0, T, rows):
                sl = slice(i, min(i + rows, T))
                pos = torch.arange(sl.start, sl.stop, device=q.device) + Tk - T
                o, l, gr = _exact_head(q[b, h, sl], k[b, kv], v[b, kv], case, d ** -0.5, None if slopes is None else slopes[h].double(), pos,
                                       torch.zeros_like(pos) if lo is None else lo[b, sl], pos + 1 if hi is None else hi[b, sl],
                                       None if g is None else g[b, h, sl])
                O[b, h, sl], L[b, h, sl] = o, l
                if gr is not None:
                    grads[0][b, h, sl] = gr[0]
                    grads[1][b, kv] += gr[1]
                    grads[2][b, kv] += gr[2]
    return O, L, grads


def _exact_held(case, x):
    """The values that the cache holds for float64 rows [..., d]."""
    if case["bits"] == 16:
        return x.bfloat16().double()
    g = x.clamp(-65024, 65024).unflatten(-1, (x.shape[-1] // GROUP, GROUP))
    low, high = g.min(-1, keepdim=True).values, g.max(-1, keepdim=True).values
    unit, low = ((high - low) / 15).float().half().double(), low.float().half().double()
    code = torch.where(unit > 0, torch.round((g - low) / unit.clamp(min=1e-30)), 0.0).clamp(0, 15)
    return (low + code * unit).flatten(-2)


def _exact_turned(case, x, rows, cos, sin):
    """float64 [n, h, d] at table rows [n]"""
    half = case["rot"] // 2
    if not half:
        return x
    z = torch.complex(x[..., :half], x[..., half:2 * half]) * torch.complex(cos.double(), sin.double())[rows].unsqueeze(1)
    return torch.cat([z.real, z.imag, x[..., 2 * half:]], -1)


def exact(case, seed):
    x = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("fwd", "train"):
        q, k, v = (x[n].double() for n in "qkv")
        O, L, grads = _exact_attend(case, q, k, v, x["slopes"], x["lo"], x["hi"], x["g"].double() if kind == "train" else None)
        return (O, L) if kind == "fwd" else (O, *grads)
    past, count = _lengths(case)
    if kind == "step":
        B, H, d = case["B"], case["H"], case["d"]
        O, L = torch.zeros(B, H, d, dtype=torch.float64, device="cuda"), torch.zeros(B, H, dtype=torch.float64, device="cuda")
        for b in range(B):
            n = past[b] + 1
            k, v = (_exact_held(case, x[m][b:b + 1, :, :n].double()) for m in ("ctx_k", "ctx_v"))
            o, l, _ = _exact_attend(case, x["q"][b:b + 1].double(), k, v, x["slopes"], None, None)
            O[b], L[b] = o[0, :, 0], l[0, :, 0]
        return O, L
    turned = {}
    for n in "qk":
        to = torch.zeros_like(x[n], dtype=torch.float64)
        for b in range(case["B"]):
            rows = torch.arange(past[b], past[b] + count[b], device="cuda")
            y = _exact_turned(case, x[n][b, :, :count[b]].double().transpose(0, 1), rows, x.get("cos"), x.get("sin"))
            to[b, :, :count[b]] = y.transpose(0, 1)
        turned[n] = to
    if kind == "append":
        if case["bits"] == 4:       # a code next to a border has no one value
            return turned["q"], None, None
        v = torch.zeros_like(x["v"], dtype=torch.float64)
        for b in range(case["B"]):
            v[b, :, :count[b]] = x["v"][b, :, :count[b]].double()
        return turned["q"], turned["k"], v
    k = torch.cat([_exact_held(case, x["ctx_k"].double()), _exact_held(case, turned["k"])], 2)
    v = torch.cat([_exact_held(case, x["ctx_v"].double()), _exact_held(case, x["v"].double())], 2)
    k, v = k.bfloat16().double(), v.bfloat16().double()
    O, L, _ = _exact_attend(case, turned["q"].bfloat16().double(), k, v, x["slopes"], None, None)
    if case["bits"] == 4:
        return None, None, O, L
    return k, v, O, L
