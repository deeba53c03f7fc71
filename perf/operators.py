"""The operators around a paged cache of keys and values, as a serving program calls them: a backbone's heads are normed and
rotated, its new keys and values appended to pages, chunks of new tokens attend over the pages, and a finished prefix is packed
into the ragged cache that the denoising loop reads.

Head shapes are those of ``synth`` (pi0-shaped: 8 query heads on 1 kv head of 256; feature-handoff head: 8 on 2 of 128; the tiny
fp32 expert: 4 on 1 of 64) and generic ones; queries, keys and values are N(0, 1), gains of the head norms N(0, 0.1)."""
import math
import random

import torch

own = False

EPS = 1e-6
THETA = 10000.0


# ------------------------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------------------------
PI0, HANDOFF, TINY = (8, 1, 256), (8, 2, 128), (4, 1, 64)


def _heads(name, tokens, heads, src, dst):
    return dict(name=name, kind="heads", tokens=tokens, hq=heads[0], hkv=heads[1], dh=heads[2], src=src, dst=dst)


def _append(name, batch, q_lo, q_hi, kv_lo, kv_hi, heads, page, src="bf16", dst="bf16"):
    return dict(name=name, kind="append", batch=batch, q_lo=q_lo, q_hi=q_hi, kv_lo=kv_lo, kv_hi=kv_hi, hq=heads[0], hkv=heads[1],
                dh=heads[2], page=page, src=src, dst=dst)


def _attend(name, batch, q_lo, q_hi, kv_lo, kv_hi, heads, page, mask, dst="bf16"):
    return dict(name=name, kind="attend", batch=batch, q_lo=q_lo, q_hi=q_hi, kv_lo=kv_lo, kv_hi=kv_hi, hq=heads[0], hkv=heads[1],
                dh=heads[2], page=page, mask=mask, dst=dst)


def _pack(name, batch, lo, hi, layers, heads, page):
    return dict(name=name, kind="pack", batch=batch, kv_lo=lo, kv_hi=hi, layers=layers, hkv=heads[1], dh=heads[2], page=page)


def listed():
    # kv_lo .. kv_hi: cached tokens of a request with its new ones; q_lo .. q_hi: new tokens of it
    return [
        # one robot, one token of a layer's q | k rows: the smallest call, latency only
        _heads("heads-b1", 1, PI0, "f32", "bf16"),
        # the prefix tokens of eight robots
        _heads("heads-prefix-b8", 8 * 968, PI0, "bf16", "bf16"),
        # one new token for each of 64 robots, appended; its queries normed and rotated in the same pass
        _append("append-token-b64", 64, 1, 1, 601, 969, PI0, 64),
        # the whole prefixes of eight robots, ragged
        _append("append-prefix-b8", 8, 600, 968, 600, 968, PI0, 64),
        # one robot, one token over its prefix: latency
        _attend("token-b1", 1, 1, 1, 969, 969, PI0, 64, "causal"),
        # one token for each of 64 robots over ragged prefixes
        _attend("token-b64", 64, 1, 1, 601, 969, PI0, 64, "causal"),
        # one token each over long histories, grouped heads, small pages
        _attend("token-long-b8", 8, 1, 1, 24576, 32768, HANDOFF, 16, "causal"),
        # the prefixes of eight robots attending to themselves, every token to every other
        _attend("prefix-b8", 8, 968, 968, 968, 968, PI0, 64, "full"),
        # chunks of new tokens over long histories
        _attend("chunk-long-b4", 4, 384, 512, 4096, 8192, HANDOFF, 16, "causal"),
        # the tiny fp32 expert's heads: true fp32 arithmetic
        _attend("tiny-f32-b4", 4, 17, 17, 33, 81, TINY, 16, "causal", "f32"),
        # a finished prefix of one robot into the ragged cache of the denoising loop, all layers
        _pack("pack-b1", 1, 816, 816, 18, PI0, 64),
        # eight robots, ragged prefixes
        _pack("pack-b8", 8, 600, 968, 18, PI0, 64),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["heads", "append", "append", "attend", "attend", "attend", "attend", "attend", "pack"])
    heads = rng.choice([PI0, PI0, HANDOFF, TINY, (8, 1, 128), (32, 8, 128), (6, 2, 128), (16, 1, 64), (4, 4, 256)])
    page = rng.choice([16, 32, 64, 128])
    if kind == "heads":
        src, dst = rng.choice([("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        tokens = _log_int(rng, 1, (1 << 25) // (heads[0] * heads[2]) // (2 if src == "f32" else 1) // (2 if dst == "f32" else 1))
        return dict(_heads("", tokens, heads, src, dst))
    if kind == "pack":
        lo, hi = sorted((rng.randint(1, 968), rng.randint(1, 968)))
        return dict(_pack("", _log_int(rng, 1, 8), lo, hi, rng.randint(2, 18), PI0, page))
    if kind == "append":
        src, dst = rng.choice([("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        batch = _log_int(rng, 1, 64)
        q_hi = _log_int(rng, 1, max(1, min(1024, (8192 if src == "bf16" else 4096) // batch)))
        q_lo = rng.randint(max(0, q_hi // 2), q_hi)
        past = _log_int(rng, 1, 2048)
        return dict(_append("", batch, q_lo, q_hi, q_hi + past // 2, q_hi + past, heads, page, src, dst))
    # attention: one token (half of the cases), a few, or a chunk; the products of new and cached tokens are bounded
    dst = rng.choice(["bf16"] * 5 + ["f32"])
    mask = rng.choice(["causal", "causal", "full", "prefix"])
    batch = _log_int(rng, 1, 64)
    q_hi = 1 if rng.random() < 0.45 else _log_int(rng, 2, 1024)
    room = (1 << 33) // (batch * q_hi * heads[0] * heads[2])          # (multiply-adds of one product: at most the largest listed case's)
    if dst == "f32":
        room //= 16
    room = min(room, (1 << (24 if dst == "f32" else 25)) // (batch * heads[1] * heads[2]) * 3 // 2, 32768)
    q_hi = max(1, min(q_hi, room // 2))
    kv_hi = q_hi + _log_int(rng, 8, max(16, room - q_hi))
    q_lo = rng.randint((q_hi + 1) // 2, q_hi)
    kv_lo = rng.randint(max(q_hi, kv_hi // 2), kv_hi)
    return dict(_attend("", batch, q_lo, q_hi, kv_lo, kv_hi, heads, page, mask, dst))


# ------------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------------
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _spread(batch, lo, hi, salt):
    """One length per request: spread evenly over lo..hi, in a fixed shuffled order; a batch of one takes hi."""
    if batch == 1:
        return [hi]
    order = list(range(batch))
    random.Random(salt).shuffle(order)
    return [lo + (hi - lo) * i // (batch - 1) for i in order]


def _lengths(case):
    """(new tokens, cached tokens with the new ones) of every request."""
    kv = _spread(case["batch"], case["kv_lo"], case["kv_hi"], 1)
    if case["kind"] == "pack":
        return [0] * case["batch"], kv
    q = _spread(case["batch"], case["q_lo"], case["q_hi"], 2)
    if case["q_lo"] == case["kv_lo"]:                     # whole prefixes: every cached token is a new one
        q = kv
    return [min(a, b) for a, b in zip(q, kv)], kv


def _normal(gen, shape, dtype, std=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _rope_table(positions, dh):
    pos = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None]
    ang = pos * THETA ** (-2.0 * torch.arange(dh // 2, dtype=torch.float64, device="cuda") / dh)[None, :]
    return torch.stack([ang.cos(), ang.sin()], dim=-1).float().contiguous()


def _paging(case, kv, seed):
    """Pages of the requests, drawn from the pool without order: (rows of the pool, table [batch, most pages]); the entries
    behind a request's last page name no page."""
    page = case["page"]
    need = [(n + page - 1) // page for n in kv]
    pool = sum(need) + 3
    ids = list(range(pool))
    random.Random(seed).shuffle(ids)
    table, at = [], 0
    for n in need:
        table.append(ids[at:at + n] + [-1] * (max(need) - n))
        at += n
    return pool * page, table


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    if kind == "heads":
        T, hq, hkv, dh = case["tokens"], case["hq"], case["hkv"], case["dh"]
        # rows of a fused projection: q | k | v
        qkv = _normal(gen, (T, (hq + 2 * hkv) * dh), _TYPES[case["src"]])
        longest = min(T, 968)
        s = dict(kind=kind, q=qkv[:, :hq * dh].view(T, hq, dh), k=qkv[:, hq * dh:(hq + hkv) * dh].view(T, hkv, dh),
                 positions=torch.arange(T, dtype=torch.int32, device="cuda") % longest, rope=_rope_table(968, dh),
                 q_gain=_normal(gen, (dh,), torch.float32, 0.1), k_gain=_normal(gen, (dh,), torch.float32, 0.1),
                 dst=_TYPES[case["dst"]])
        if own:
            s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        return s
    q_lens, kv = _lengths(case)
    rows, table = _paging(case, kv, seed)
    hkv, dh, page = case["hkv"], case["dh"], case["page"]
    if kind == "pack":
        s = dict(kind=kind, pages=_normal(gen, (case["layers"], 2, rows, hkv, dh), torch.bfloat16), lens=kv)
    else:
        dst = _TYPES[case["dst"]]
        s = dict(kind=kind, pages=_normal(gen, (2, 2, rows, hkv, dh), dst), layer=1, q_lens=q_lens, lens=kv,
                 cu=_ints([0] + q_lens).cumsum(0).to(torch.int32))
        T, hq = sum(q_lens), case["hq"]
        if kind == "append":
            qkv = _normal(gen, (T, (hq + 2 * hkv) * dh), _TYPES[case["src"]])
            s.update(q=qkv[:, :hq * dh].view(T, hq, dh), k=qkv[:, hq * dh:(hq + hkv) * dh].view(T, hkv, dh),
                     v=qkv[:, (hq + hkv) * dh:].view(T, hkv, dh), rope=_rope_table(max(kv), dh),
                     q_gain=_normal(gen, (dh,), torch.float32, 0.1), k_gain=_normal(gen, (dh,), torch.float32, 0.1))
        else:
            s.update(q=_normal(gen, (T, hq, dh), dst), causal=case["mask"] != "full", prefix_lens=None, prefix=None)
            if case["mask"] == "prefix":      # image and prompt tokens see one another, what follows sees what is before it
                s["prefix"] = [n * 2 // 3 for n in kv]
                s["prefix_lens"] = _ints(s["prefix"])
    s.update(page=page, table=_ints(table), kv_lens=_ints(kv))
    if own:
        from paper_2608_03682_b200 import binding

        s["cache"] = binding.PagedCache(s["pages"], page)
    return s


# ------------------------------------------------------------------------------------------------------------------
# plain forms
# ------------------------------------------------------------------------------------------------------------------
def _plain_heads(x, gain, rope_rows, dst):
    """x [T, heads, dh] -> normed (gain 1 + gain) and rotated: channel j with channel j + dh / 2."""
    x = x.float()
    half = x.shape[-1] // 2
    x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * (1.0 + gain)
    c, s = rope_rows[:, None, :, 0], rope_rows[:, None, :, 1]
    lo, hi = x[..., :half], x[..., half:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], dim=-1).to(dst)


def _plain_rows(s, b, first, last):
    """Rows of the pool that hold cached tokens first .. last - 1 of request b."""
    t = torch.arange(first, last, device="cuda")
    return s["table"][b].long()[t // s["page"]] * s["page"] + t % s["page"]


def _plain_append(s):
    dst, at = s["pages"].dtype, 0
    q_out = torch.empty(s["q"].shape, dtype=dst, device="cuda")
    for b, (n, total) in enumerate(zip(s["q_lens"], s["lens"])):
        if n == 0:
            continue
        tok, rope = slice(at, at + n), s["rope"][total - n:total]
        rows = _plain_rows(s, b, total - n, total)
        s["pages"][s["layer"], 0, rows] = _plain_heads(s["k"][tok], s["k_gain"], rope, dst)
        s["pages"][s["layer"], 1, rows] = s["v"][tok].to(dst)
        q_out[tok] = _plain_heads(s["q"][tok], s["q_gain"], rope, dst)
        at += n
    return q_out, s["pages"]


def _plain_attend(s):
    out, at = torch.zeros_like(s["q"]), 0
    T, hq, dh = s["q"].shape
    hkv = s["pages"].shape[3]
    for b, (n, total) in enumerate(zip(s["q_lens"], s["lens"])):
        if n == 0:
            continue
        rows = _plain_rows(s, b, 0, total)
        k = s["pages"][s["layer"], 0, rows].float().permute(1, 2, 0)                                # [hkv, dh, keys]
        v = s["pages"][s["layer"], 1, rows].float().permute(1, 0, 2)                                # [hkv, keys, dh]
        q = s["q"][at:at + n].float().view(n, hkv, hq // hkv, dh).permute(1, 2, 0, 3).reshape(hkv, -1, dh)
        logits = torch.bmm(q, k) * dh ** -0.5                                                      # [hkv, group * n, keys]
        if s["causal"]:
            limit = torch.arange(total - n + 1, total + 1, device="cuda")
            if s["prefix"] is not None:
                limit = limit.clamp(min=s["prefix"][b])
            hidden = torch.arange(total, device="cuda")[None, :] >= limit[:, None]
            logits.view(hkv, hq // hkv, n, total).masked_fill_(hidden, float("-inf"))
        p = torch.exp(logits - logits.amax(dim=-1, keepdim=True))
        o = torch.bmm(p, v) / p.sum(dim=-1, keepdim=True)
        out[at:at + n] = o.view(hkv, hq // hkv, n, dh).permute(2, 0, 1, 3).reshape(n, hq, dh).to(out.dtype)
        at += n
    return out


def _plain_pack(s):
    L, _, _, hkv, dh = s["pages"].shape
    rows = torch.cat([_plain_rows(s, b, 0, n) for b, n in enumerate(s["lens"])])
    lens = torch.cat([torch.zeros_like(s["kv_lens"][:1]), s["kv_lens"]])
    return s["pages"][:, :, rows], lens.cumsum(0).to(torch.int32)


# ------------------------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if not own:
        if kind == "heads":
            rope = s["rope"][s["positions"].long()]
            return _plain_heads(s["q"], s["q_gain"], rope, s["dst"]), _plain_heads(s["k"], s["k_gain"], rope, s["dst"])
        return {"append": _plain_append, "attend": _plain_attend, "pack": _plain_pack}[kind](s)
    if kind == "heads":
        from paper_2608_03682_b200 import binding

        return binding.norm_rope_heads(s["q"], s["k"], s["positions"], s["rope"], s["q_gain"], s["k_gain"], eps=EPS, dtype=s["dst"],
                                       status=s["status"])
    cache = s["cache"]
    if kind == "append":
        q = cache.append(s["layer"], s["k"], s["v"], s["cu"], s["kv_lens"], s["table"], s["rope"], s["k_gain"], q=s["q"],
                         q_gain=s["q_gain"], eps=EPS)
        return q, cache.pages
    if kind == "attend":
        return cache.attend(s["layer"], s["q"], s["cu"], s["kv_lens"], s["table"], causal=s["causal"], prefix_lens=s["prefix_lens"])
    return cache.pack(s["table"], s["kv_lens"], sum(s["lens"]))


# ------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------
def work(case):
    size = {"bf16": 2, "f32": 4}
    hkv, dh, kind = case["hkv"], case["dh"], case["kind"]
    if kind == "heads":
        T, H = case["tokens"], case["hq"] + hkv
        return {"bytes": T * H * dh * (size[case["src"]] + size[case["dst"]]) + T * 4 + (min(T, 968) + 2) * dh * 4, "flops": 10 * T * H * dh}
    q, kv = _lengths(case)
    table = sum((n + case["page"] - 1) // case["page"] for n in kv) * 4 + 8 * len(kv)
    if kind == "pack":
        return {"bytes": 2 * sum(kv) * case["layers"] * 2 * hkv * dh * 2 + table, "flops": 0}
    T, hq, out = sum(q), case["hq"], size[case["dst"]]
    if kind == "append":
        used = len({p for n, t in zip(q, kv) for p in range(t - n, t)})
        return {"bytes": T * (hq + 2 * hkv) * dh * (size[case["src"]] + out) + (used + 2) * dh * 4 + 12 * len(kv),
                "flops": 10 * T * (hq + hkv) * dh}
    seen = 0
    for n, t in zip(q, kv):
        if case["mask"] == "full":
            seen += n * t
        else:
            p = t * 2 // 3 if case["mask"] == "prefix" else 0
            seen += sum(max(t - n + 1 + i, p) for i in range(n))
    return {"bytes": 2 * T * hq * dh * out + sum(kv) * 2 * hkv * dh * out + table, "flops": 4 * seen * hq * dh}


# ------------------------------------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ------------------------------------------------------------------------------------------------------------------
def _exact_rotate(x, gain, cs):
    """x [..., dh] as complex numbers of channels (j, j + dh / 2), times cos + i sin."""
    d = x.double()
    d = d / d.pow(2).mean(-1, keepdim=True).add(EPS).sqrt() * gain.double().add(1.0)
    half = d.shape[-1] // 2
    z = torch.complex(d[..., :half], d[..., half:]) * torch.view_as_complex(cs.double().contiguous()).unsqueeze(-2)
    return torch.cat([z.real, z.imag], dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "heads":
        cs = s["rope"].index_select(0, s["positions"].long())
        return _exact_rotate(s["q"], s["q_gain"], cs), _exact_rotate(s["k"], s["k_gain"], cs)
    page, table, layer = s["page"], s["table"].tolist(), s.get("layer")
    slots = [torch.tensor([table[b][t // page] * page + t % page for t in range(n)], device="cuda", dtype=torch.long)
             for b, n in enumerate(s["lens"])]
    if kind == "pack":
        cu = [0]
        for n in s["lens"]:
            cu.append(cu[-1] + n)
        return torch.cat([s["pages"].index_select(2, i) for i in slots], dim=2).double(), _ints(cu)
    first = [sum(s["q_lens"][:b]) for b in range(len(s["lens"]))]
    if kind == "append":
        where = torch.cat([slots[b][n - m:] for b, (m, n) in enumerate(zip(s["q_lens"], s["lens"]))])
        pos = torch.cat([torch.arange(n - m, n, device="cuda") for m, n in zip(s["q_lens"], s["lens"])])
        cs = s["rope"].index_select(0, pos)
        pages = s["pages"].double()
        pages[layer, 0].index_copy_(0, where, _exact_rotate(s["k"], s["k_gain"], cs))
        pages[layer, 1].index_copy_(0, where, s["v"].double())
        return _exact_rotate(s["q"], s["q_gain"], cs), pages
    hq, dh = s["q"].shape[1:]
    hkv = s["pages"].shape[3]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, (m, n) in enumerate(zip(s["q_lens"], s["lens"])):
        if m == 0:
            continue
        kv = s["pages"][layer].index_select(1, slots[b]).double()                # [2, n, hkv, dh]
        pos = torch.arange(n - m, n, device="cuda")
        for h in range(hq):
            g = h // (hq // hkv)
            w = s["q"][first[b]:first[b] + m, h].double() @ kv[0, :, g].T / math.sqrt(dh)
            if s["causal"]:
                key = torch.arange(n, device="cuda").expand(m, n)
                seen = key <= pos[:, None]
                if s["prefix"] is not None:
                    seen = seen | (key < s["prefix"][b])
                w = torch.where(seen, w, torch.full_like(w, -math.inf))
            out[first[b]:first[b] + m, h] = torch.softmax(w, dim=-1) @ kv[1, :, g]
    return out
