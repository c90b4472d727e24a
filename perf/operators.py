"""Cases by which the speed of attention and of its 8-bit cache is judged: what they are, their inputs, one pass, the work in it.

A case is one of four kinds of call that a program makes of this package between the qkv layer and the output projection:

  attend   attention_f16: softmax attention on the binary16 rows that the qkv layer leaves, over whole images or packed sequences
  append   daq_kv_append: rotation of queries and keys, and the dynamic quantization of keys and values into a paged 8-bit cache
  cached   attention_kv8: attention over that cache
  step     daq_kv_append followed by attention_kv8, as one layer of a program that extends its sequences runs them

With n_q rows and n_k keys in a sequence, row i stands at position i + n_k - n_q.  Scores are scale * q.k, then cap * tanh(./cap) where
there is a cap, then minus slope * distance where there are slopes.
"""
import math
import random

import torch

own = False

NONE, CAUSAL, PREFIX = "none", "causal", "prefix"
GROUP = 64          # tokens whose value codes the cache keeps together: [D][64] bytes
PARTS = (32, 64, 72, 80, 96, 128, 256)


def _attend(name, B, Sq, Sk, Hq, Hkv, D, mask=NONE, cap=0.0, bias=False, lengths=0, absmax=False):
    return dict(name=name, kind="attend", B=B, Sq=Sq, Sk=Sk, Hq=Hq, Hkv=Hkv, D=D, mask=mask, cap=cap, bias=bias, lengths=lengths, absmax=absmax)


def _cache(name, kind, B, Sq, Sk, Hq, Hkv, D, page, per_scale, mask=CAUSAL, cap=0.0, bias=False, lengths=0, rot=0, values=False):
    return dict(name=name, kind=kind, B=B, Sq=Sq, Sk=Sk, Hq=Hq, Hkv=Hkv, D=D, page=page, per_scale=per_scale, mask=mask, cap=cap, bias=bias,
                lengths=lengths, rot=rot, values=values)


def listed():
    return [
        # one 256-token image through the narrowest block (width 384, 6 heads): the smallest call of a sampling loop
        _attend("attend_image_256", 1, 256, 256, 6, 6, 64, absmax=True),
        # 8 images of 256 tokens, width 1152 with 16 heads of 72, row maxima for the output projection's quantizer
        _attend("attend_images_m2048", 8, 256, 256, 16, 16, 72, absmax=True),
        # the 512-pixel size: 16 images of 1024 tokens
        _attend("attend_images_m16384", 16, 1024, 1024, 16, 16, 72, absmax=True),
        # images of many sizes packed behind each other, capped scores and a bias by distance, shared key heads
        _attend("attend_packed_cap_bias", 24, 1000, 1000, 12, 4, 64, cap=30.0, bias=True, lengths=11),
        # one long sequence whose first 1000 tokens all see each other: text in front of what is generated
        _attend("attend_prefix_8k", 1, 8192, 8192, 16, 2, 128, mask=PREFIX),
        # one new token for each of 64 sequences: the append of a generation step
        _cache("append_tokens_b64", "append", 64, 1, 4000, 16, 2, 128, 64, 64, lengths=12, rot=128),
        # prompts of many lengths entering the cache, with the values it then holds for the dense attention over them
        _cache("append_prompts", "append", 16, 1024, 1500, 32, 8, 128, 128, 64, lengths=13, rot=128, values=True),
        # one token of one sequence over 4096 cached ones: latency
        _cache("cached_one_4k", "cached", 1, 1, 4096, 16, 2, 128, 64, 64),
        # a served batch: 64 sequences of very different lengths, one token each
        _cache("cached_tokens_b64", "cached", 64, 1, 8192, 32, 8, 128, 64, 64, lengths=14),
        # two very long sequences
        _cache("cached_long_128k", "cached", 2, 1, 131071, 32, 8, 128, 128, 32),
        # chunks of 512 prompt rows over what is cached of them so far, capped scores
        _cache("cached_chunks", "cached", 8, 512, 4096, 16, 2, 128, 64, 64, cap=50.0, lengths=15),
        # one layer of a generation step: 32 sequences, heads of 64, a scale for every token
        _cache("step_tokens_b32", "step", 32, 1, 2000, 12, 4, 64, 64, 1, bias=True, lengths=16, rot=64),
    ]


MOST_PAIRS = 16 * 8192 * 8192 * 128     # multiplications of the largest listed dense case
MOST_CACHE = 64 * 8192 * 8 * 128        # padded codes of the largest listed cached case
MOST_CHUNK = 8 * 16 * 512 * 4096 * 128  # multiplications of the largest listed cached case


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _nameless(case):
    del case["name"]
    return case


def draw(rng):
    kind = rng.choice(("attend", "attend", "append", "cached", "cached", "step"))
    Hkv = rng.choice((1, 2, 4, 6, 8, 16))
    Hq = Hkv * rng.choice((1, 1, 2, 3, 4, 8) if Hkv <= 4 else (1, 2, 4) if Hkv <= 8 else (1,))
    lengths = rng.choice((0, rng.randrange(1, 10000)))
    mask = rng.choice((NONE, CAUSAL, PREFIX))
    cap = rng.choice((0.0, 0.0, 20.0, 50.0))
    bias = rng.random() < 0.3
    while True:
        D = rng.choice(PARTS)
        B = _log_int(rng, 1, 64)
        if kind == "attend":
            Sq = _log_int(rng, 1, 8192)
            Sk = Sq if rng.random() < 0.7 else _log_int(rng, 1, 8192)
            if B * Hq * Sq * Sk * D <= MOST_PAIRS and B * (Sq + Sk) <= 65536:
                return _nameless(_attend("", B, Sq, Sk, Hq, Hkv, D, mask, cap, bias, lengths, rng.random() < 0.5))
            continue
        per_scale = rng.choice((1, 16, 32, 64))
        page = rng.choice((64, 128, 256))
        rot = rng.choice((0, D // 32 * 16, D // 16 * 16))
        if kind == "append":
            Sq = _log_int(rng, 1, 2048)
            Sk = Sq + _log_int(rng, 1, 2048)
            if B * Sq <= 16384 and B * Sk * Hkv * D <= MOST_CACHE // 8:
                return _nameless(_cache("", kind, B, Sq, Sk, Hq, Hkv, D, page, per_scale, lengths=lengths, rot=rot, values=rng.random() < 0.5))
            continue
        Sq = _log_int(rng, 1, 1024) if rng.random() < 0.4 else rng.choice((1, 1, 1, 2, 5))
        Sk = Sq + _log_int(rng, 1, 65536)
        if B * Sk * Hkv * D <= MOST_CACHE // 2 and B * Hq * Sq * Sk * D <= MOST_CHUNK:
            return _nameless(_cache("", kind, B, Sq, Sk, Hq, Hkv, D, page, per_scale, mask, cap, bias, lengths, rot if kind == "step" else 0))


def _lengths(case):
    """(rows, keys) of every sequence: all alike, or drawn by the case's own number."""
    B, Sq, Sk = case["B"], case["Sq"], case["Sk"]
    if not case["lengths"]:
        return [Sq] * B, [Sk] * B
    r = random.Random(case["lengths"])
    nq = [Sq] + [max(1, int(round(Sq * r.uniform(0.05, 1.0)))) for _ in range(B - 1)]
    if case["kind"] == "attend" and Sq == Sk:
        return nq, list(nq)
    # a cache holds the new rows too; keys of another sequence may be none at all
    low = [0 if case["kind"] == "attend" else n for n in nq]
    return nq, [Sk] + [lo + int((Sk - lo) * r.random() ** 2) for lo in low[1:]]


def _visible_pairs(case):
    nq, nk = _lengths(case)
    pairs = 0
    for a, b, p in zip(nq, nk, _prefixes(case, nk)):
        if case["mask"] == NONE:
            pairs += a * b
        else:
            # rows see positions up to their own, and what lies in the prefix
            for i0 in range(0, a, 4096):
                i = torch.arange(i0, min(a, i0 + 4096), dtype=torch.int64)
                pairs += int(torch.clamp(torch.clamp(i + b - a + 1, min=p if case["mask"] == PREFIX else 0), 0, b).sum())
    return pairs


def _prefixes(case, nk):
    """Tokens at the front of each sequence that every row sees."""
    return [min(n, 1000 if n > 2000 else n // 3) for n in nk]


def work(case):
    nq, nk = _lengths(case)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    Tq, Tk = sum(nq), sum(nk)
    kind = case["kind"]
    nbytes = flops = 0
    if kind == "attend":
        nbytes += 2 * D * (2 * Tq * Hq + 2 * Tk * Hkv) + (4 * Tq if case["absmax"] else 0)
    if kind in ("append", "step"):
        nbytes += 2 * D * Tq * (2 * Hq + 2 * Hkv) + 2 * D * Tq * Hkv + 4 * Tq * case["rot"]
        nbytes += 4 * D * Tq * Hkv if case["values"] else 0
        flops += 6 * case["rot"] * Tq * (Hq + Hkv) + 4 * D * Tq * Hkv
    if kind in ("cached", "step"):
        nbytes += 2 * D * Tk * Hkv + 8 * Hkv * (Tk // case["per_scale"] + 1) + 2 * D * 2 * Tq * Hq
    if kind != "append":
        flops += 4 * D * Hq * _visible_pairs(case)
    return dict(bytes=nbytes, flops=flops)


def _slot():
    """Where token t of a group of 64 keeps its value codes: 16 * (t % 16 // 4) + 4 * (t // 16) + t % 4."""
    t = torch.arange(GROUP, device="cuda")
    return 16 * (t % 16 // 4) + 4 * (t // 16) + t % 4


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev = dict(device="cuda")
    nq, nk = _lengths(case)
    B, Hq, Hkv, D = case["B"], case["Hq"], case["Hkv"], case["D"]
    Tq, Tk = sum(nq), sum(nk)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, **dev)

    def sums(v):
        c = [0]
        for n in v:
            c.append(c[-1] + n)
        return ints(c)

    def normal(*shape):
        return torch.randn(shape, generator=g, **dev)

    st = dict(case=case, nq=nq, nk=nk, max_q=max(nq), max_k=max(nk), len_k=ints(nk))
    equal = not case["lengths"]
    st["cu_q"] = None if equal else sums(nq)
    st["prefix"] = ints(_prefixes(case, nk)) if case["mask"] == PREFIX else None
    st["slopes"] = torch.rand(Hq, generator=g, **dev) * 0.2 if case["bias"] else None
    st["scale"] = D ** -0.5
    # what the qkv layer leaves: rows of [queries | keys | values], channels of differing size
    gain = 0.25 + 1.5 * torch.rand((Hq + 2 * Hkv) * D, generator=g, **dev)
    if case["kind"] == "attend" and Tq != Tk:
        st["q"] = (normal(Tq, Hq * D) * gain[: Hq * D]).half().view(Tq, Hq, D)
        kv = (normal(Tk, 2 * Hkv * D) * gain[Hq * D:]).half()
        st["k"], st["v"] = kv[:, : Hkv * D].view(Tk, Hkv, D), kv[:, Hkv * D:].view(Tk, Hkv, D)
        st["cu_k"] = None if equal else sums(nk)
    else:
        rows = (normal(Tq, (Hq + 2 * Hkv) * D) * gain).half()
        st["q"] = rows[:, : Hq * D].unflatten(1, (Hq, D))
        st["k"] = rows[:, Hq * D: (Hq + Hkv) * D].unflatten(1, (Hkv, D))
        st["v"] = rows[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D))
        st["cu_k"] = st["cu_q"]
    st["o"] = torch.empty((Tq, Hq, D), dtype=torch.float16, **dev)
    if case["kind"] == "attend":
        st["absmax"] = torch.empty(Tq, dtype=torch.int32, **dev) if case["absmax"] else None
        return st
    # the cache: pages in no order, every sequence's table filled as far as it needs
    page, S = case["page"], case["per_scale"]
    need = [-(-n // page) for n in nk]
    P = sum(need) + 3
    order = torch.randperm(P, generator=g, **dev).int()
    table = torch.full((B, max(max(need), 1)), -1, dtype=torch.int32, **dev)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at: at + n]
        at += n
    st["table"] = table

    def codes(*shape):
        out = torch.empty(shape, dtype=torch.int8, **dev)
        flat = out.view(-1)
        for i in range(0, flat.numel(), 1 << 28):
            part = flat[i: i + (1 << 28)]
            part.copy_((normal(part.numel()) * 36.0).clamp_(-127, 127).round_())
        return out

    st["kc"], st["vc"] = codes(P, Hkv, page, D), codes(P, Hkv, page // GROUP, D, GROUP)
    st["ks"] = 0.02 + 0.03 * torch.rand((P, Hkv, page // S), generator=g, **dev)
    st["vs"] = 0.02 + 0.03 * torch.rand((P, Hkv, page // S), generator=g, **dev)
    st["rot"] = None
    if case["kind"] != "cached":
        half = case["rot"] // 2
        if half:
            angle = torch.arange(max(nk), dtype=torch.float64, **dev)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64, **dev) / half)
            st["rot"] = torch.stack((angle.cos(), angle.sin()), dim=-1).float().contiguous()
        st["q_rot"] = torch.empty((Tq, Hq, D), dtype=torch.float16, **dev)
        for name in ("k_val", "v_val"):
            st[name] = torch.empty((Tq, Hkv, D), dtype=torch.float16, **dev) if case["values"] else None
    return st


# ---- the plain form ---------------------------------------------------------------------------------------------------------

def _rows(st, cu, n, count, T):
    """Which sequence each of T packed rows is of, and its place in it."""
    t = torch.arange(T, device="cuda")
    if cu is None:
        return t // n, t % n
    b = torch.searchsorted(cu[1:].long(), t, right=True)
    return b, t - cu.long()[b]


def _padded(x, cu, count, most):
    """Packed rows [T, H, D] as float32 [count, most, H, D] (rows behind a sequence's end repeat some row)."""
    if cu is None:
        return x.float().unflatten(0, (count, most))
    at = (cu[:-1].long()[:, None] + torch.arange(most, device="cuda")).clamp(max=x.shape[0] - 1)
    return x[at].float()


def _softmax_attention(st, q, k, v):
    """float32 [B, Sq, Hq, D] from padded q, k, v; st says lengths, mask and score form."""
    case = st["case"]
    B, Sq, Hq, D = q.shape
    Sk, Hkv = k.shape[1], k.shape[2]
    G = Hq // Hkv
    q = q.view(B, Sq, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Sq, D)
    s = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(st["scale"]).view(B, Hkv, G, Sq, Sk)
    if case["cap"] > 0:
        s = s.div_(case["cap"]).tanh_().mul_(case["cap"])
    nk = st["len_k"].long()
    nq = (torch.full_like(nk, Sq) if st["cu_q"] is None else st["cu_q"].long().diff())
    j = torch.arange(Sk, device="cuda")
    p = torch.arange(Sq, device="cuda") + (nk - nq)[:, None]           # [B, Sq]
    if st["slopes"] is not None:
        far = (p[:, :, None] - j).abs().float()                          # [B, Sq, Sk]
        s -= st["slopes"].view(1, Hkv, G, 1, 1) * far[:, None, None]
    seen = (j < nk[:, None])[:, None, :].expand(B, Sq, Sk)
    if case["mask"] != NONE:
        back = j <= p[:, :, None]
        if case["mask"] == PREFIX:
            back = back | (j < st["prefix"].long()[:, None])[:, None, :]
        seen = seen & back
    s = s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    w = s.sub_(m.masked_fill(m == -math.inf, 0.0)).exp_()
    total = w.sum(-1).view(B, Hkv, G * Sq, 1)
    o = torch.matmul(w.view(B, Hkv, G * Sq, Sk), v.permute(0, 2, 1, 3).contiguous())
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return o.view(B, Hkv, G, Sq, D).permute(0, 3, 1, 2, 4).reshape(B, Sq, Hq, D)


def _plain_attend(st, q):
    case = st["case"]
    o = _softmax_attention(st, _padded(q, st["cu_q"], case["B"], st["max_q"]), _padded(st["k"], st["cu_k"], case["B"], st["max_k"]),
                           _padded(st["v"], st["cu_k"], case["B"], st["max_k"]))
    b, i = _rows(st, st["cu_q"], st["max_q"], case["B"], q.shape[0])
    return o[b, i].half()


def _plain_cached(st, q):
    case = st["case"]
    at = st["table"].long().clamp(min=0)
    B, S = case["B"], case["per_scale"]
    k = st["kc"][at].float() * st["ks"][at].repeat_interleave(S, dim=-1)[..., None]                   # [B, pages, Hkv, page, D]
    v = st["vc"][at][..., _slot()].float()                                                            # [B, pages, Hkv, page/64, D, 64]
    v = v.transpose(-1, -2).flatten(3, 4) * st["vs"][at].repeat_interleave(S, dim=-1)[..., None]
    k, v = (x.permute(0, 1, 3, 2, 4).flatten(1, 2)[:, : max(st["max_k"], 1)] for x in (k, v))
    o = _softmax_attention(st, _padded(q, st["cu_q"], B, st["max_q"]), k, v)
    b, i = _rows(st, st["cu_q"], st["max_q"], B, q.shape[0])
    return o[b, i].half()


def _turned(x, table, pos):
    """Rotation of the leading channels: halves x1, x2 -> x1 cos - x2 sin, x2 cos + x1 sin."""
    x = x.float()
    if table is None:
        return x.half()
    half = table.shape[1]
    c, s = table[pos, :, 0][:, None], table[pos, :, 1][:, None]
    a, b = x[..., :half], x[..., half: 2 * half]
    return torch.cat((a * c - b * s, b * c + a * s, x[..., 2 * half:]), dim=-1).half()


def _plain_append(st):
    case = st["case"]
    B, S, page, D, Hkv = case["B"], case["per_scale"], case["page"], case["D"], case["Hkv"]
    T = st["k"].shape[0]
    b, i = _rows(st, st["cu_q"], st["max_q"], B, T)
    nk = st["len_k"].long()
    nq = torch.full_like(nk, case["Sq"]) if st["cu_q"] is None else st["cu_q"].long().diff()
    first = nk - nq                                                       # [B] where the new tokens of a sequence begin
    pos = first[b] + i
    table = st["table"].long()
    pg, in_page = table[b, pos // page], pos % page
    q = _turned(st["q"], st["rot"], pos)
    slot, limit = _slot(), torch.tensor(127.0, device="cuda")
    # the block in which a sequence's new tokens begin, and the tokens that are there already
    old_page = table[torch.arange(B, device="cuda"), (first // page).clamp(max=table.shape[1] - 1)].clamp(min=0)
    old_block = first % page // S
    at = old_block[:, None] * S + torch.arange(S, device="cuda")          # [B, S] places in the page
    there = at < (first % page)[:, None]
    out = {}
    for name, x, codes, scales in (("k", _turned(st["k"], st["rot"], pos), st["kc"], st["ks"]), ("v", st["v"], st["vc"], st["vs"])):
        h = x.float()
        blocks = page // S
        flat = scales.permute(0, 2, 1).reshape(-1, Hkv).clone()           # [P * blocks, Hkv]
        block = pg * blocks + in_page // S
        amax = torch.zeros_like(flat).index_reduce_(0, block, h.abs().amax(-1), "amax")
        kept = torch.zeros_like(flat)
        keep = old_page * blocks + old_block
        before = flat[keep]
        kept.index_reduce_(0, keep, torch.where(there[:, :1], before, torch.zeros_like(before)), "amax")
        touched = torch.zeros(flat.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, block, True)
        new = torch.maximum(kept, amax / limit)
        flat = torch.where(touched[:, None], new, flat)
        scales.copy_(flat.view(-1, blocks, Hkv).permute(0, 2, 1))
        alpha = flat[block][..., None]                                    # [T, Hkv, 1]
        c = torch.where(alpha > 0, h / alpha, torch.zeros_like(h)).round_().clamp_(-127, 127)
        after = flat[keep][:, None, :, None]                              # [B, 1, Hkv, 1]
        if name == "k":
            was = codes[old_page[:, None], :, at].float()                 # [B, S, Hkv, D]
        else:
            was = codes[old_page[:, None], :, at // GROUP, :, slot[at % GROUP]].float()
        again = torch.where(after > 0, was * before[:, None, :, None] / after, torch.zeros_like(was)).round_().clamp_(-127, 127)
        again = torch.where((there & (nq > 0)[:, None])[:, :, None, None], again, was).to(torch.int8)
        if name == "k":
            codes[old_page[:, None], :, at] = again
            codes[pg, :, in_page] = c.to(torch.int8)
        else:
            codes[old_page[:, None], :, at // GROUP, :, slot[at % GROUP]] = again
            codes[pg, :, in_page // GROUP, :, slot[in_page % GROUP]] = c.to(torch.int8)
        if case["values"]:
            out[name + "_val"] = (c * alpha).half()
    return dict(out, q_rot=q)


def _outputs(st, o=None, appended=None):
    out = {}
    if o is not None:
        out["o"] = o
    if appended is not None:
        out.update(appended, k_scale=st["ks"], v_scale=st["vs"])
    return out


# ---- the package's calls -----------------------------------------------------------------------------------------------------

def _own(st):
    import paper_2511_11446_amd as ql
    case = st["case"]
    kind = case["kind"]
    mask = dict(none=ql.MASK_NONE, causal=ql.MASK_CAUSAL, prefix=ql.MASK_PREFIX)[case["mask"]]
    form = dict(batch=case["B"], cu_q=st["cu_q"], mask=mask, prefix=st["prefix"], scale=st["scale"], cap=case["cap"], slopes=st["slopes"], o=st["o"])
    if kind == "attend":
        if "ws" not in st:
            st["ws"] = ql.workspace(ql.attention_f16_workspace_bytes(st["q"].shape[0], st["k"].shape[0], case["B"], case["Hq"], case["Hkv"], case["D"]))
        ql.attention_f16(st["q"], st["k"], st["v"], cu_k=st["cu_k"], row_absmax=st["absmax"], ws=st["ws"], **form)
        out = _outputs(st, st["o"])
        if case["absmax"]:
            out["absmax"] = st["absmax"].view(torch.float16).view(-1, 2)[:, 0]
        return out
    if "cache" not in st:
        st["cache"] = ql.KvCache8(st["kc"], st["vc"], st["ks"], st["vs"])
        st["ws"] = ql.workspace(ql.attention_kv8_workspace_bytes(st["q"].shape[0], case["B"], case["Hq"], case["Hkv"], case["D"]))
    q, appended = st["q"], None
    if kind != "cached":
        ql.daq_kv_append(st["cache"], st["k"], st["v"], st["table"], st["len_k"], cu=st["cu_q"], q=q, rot=st["rot"], q_out=st["q_rot"],
                         k_out=st["k_val"], v_out=st["v_val"])
        q = st["q_rot"]
        appended = dict(q_rot=q)
        if case["values"]:
            appended.update(k_val=st["k_val"], v_val=st["v_val"])
    if kind == "append":
        return _outputs(st, None, appended)
    ql.attention_kv8(q, st["cache"], st["table"], st["len_k"], ws=st["ws"], **{k: v for k, v in form.items() if k != "batch"})
    return _outputs(st, st["o"], appended)


def run(st):
    if own:
        return _own(st)
    kind = st["case"]["kind"]
    if kind == "attend":
        o = _plain_attend(st, st["q"])
        out = _outputs(st, o)
        if st["case"]["absmax"]:
            out["absmax"] = o.abs().flatten(1).amax(-1)
        return out
    appended = _plain_append(st) if kind != "cached" else None
    if kind == "append":
        return _outputs(st, None, appended)
    return _outputs(st, _plain_cached(st, st["q"] if appended is None else appended["q_rot"]), appended)


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------------

def _exact_one(case, st, b, q, k, v, n_q, n_k):
    """One sequence: q [n_q, Hq, D], k and v [n_k, Hkv, D] in float64 -> [n_q, Hq, D]."""
    G = case["Hq"] // case["Hkv"]
    o = torch.zeros_like(q)
    if n_k == 0:
        return o
    i = torch.arange(n_q, device="cuda", dtype=torch.float64)[:, None] + (n_k - n_q)
    j = torch.arange(n_k, device="cuda", dtype=torch.float64)[None, :]
    hidden = torch.zeros((n_q, n_k), dtype=torch.bool, device="cuda")
    if case["mask"] == CAUSAL:
        hidden = j > i
    elif case["mask"] == PREFIX:
        hidden = (j > i) & (j >= int(st["prefix"][b]))
    blind = hidden.all(dim=1)
    for h in range(case["Hq"]):
        x = q[:, h] @ k[:, h // G].T.contiguous() * st["scale"]
        if case["cap"] > 0:
            x = case["cap"] * torch.tanh(x / case["cap"])
        if st["slopes"] is not None:
            x = x - float(st["slopes"][h]) * (i - j).abs()
        x[hidden] = -math.inf
        w = torch.softmax(x, dim=1)
        w[blind] = 0.0
        o[:, h] = w @ v[:, h // G]
    return o


def exact(case, seed):
    st = prepare(case, seed)
    nq, nk = st["nq"], st["nk"]
    at_q = [sum(nq[:b]) for b in range(case["B"])]
    at_k = [sum(nk[:b]) for b in range(case["B"])]
    q = st["q"].double()
    if case["kind"] == "attend":
        o = torch.cat([_exact_one(case, st, b, q[at_q[b]: at_q[b] + nq[b]], st["k"][at_k[b]: at_k[b] + nk[b]].double(),
                                  st["v"][at_k[b]: at_k[b] + nk[b]].double(), nq[b], nk[b]) for b in range(case["B"])])
        out = dict(o=o)
        if case["absmax"]:
            out["absmax"] = o.abs().flatten(1).max(dim=1).values
        return out
    page, S, Hkv, D = case["page"], case["per_scale"], case["Hkv"], case["D"]
    t = torch.arange(GROUP)
    where = (t % 4 + 4 * (t // 16) + 16 * (t // 4 % 4)).cuda()

    def held(b, n):
        """What the cache holds of sequence b, as codes and scales a token: [n, Hkv, D] and [n, Hkv, 1]."""
        pages = st["table"][b, : -(-n // page)].long()
        kc = st["kc"][pages].transpose(1, 2).reshape(-1, Hkv, D)[:n].double()
        vc = st["vc"][pages][..., where].permute(0, 2, 4, 1, 3).reshape(-1, Hkv, D)[:n].double()
        ks, vs = (x[pages].double().repeat_interleave(S, dim=2).transpose(1, 2).reshape(-1, Hkv, 1)[:n] for x in (st["ks"], st["vs"]))
        return kc, ks, vc, vs

    out, o = {}, []
    if case["kind"] != "cached":
        ks_all, vs_all = st["ks"].double(), st["vs"].double()
        q_rot, k_val, v_val = [], [], []

        def turn(x, first):
            if st["rot"] is None:
                return x
            half = st["rot"].shape[1]
            z = torch.view_as_complex(st["rot"][first: first + x.shape[0]].double().contiguous())[:, None]
            y = torch.complex(x[..., :half], x[..., half: 2 * half]) * z
            return torch.cat((y.real, y.imag, x[..., 2 * half:]), dim=-1)

    for b in range(case["B"]):
        rows = slice(at_q[b], at_q[b] + nq[b])
        qb = q[rows]
        kc, ks, vc, vs = held(b, nk[b])
        first = nk[b] - nq[b]
        if case["kind"] != "cached":
            qb = turn(qb, first).half().double()
            q_rot.append(qb)
            new = (turn(st["k"][rows].double(), first).half().double(), st["v"][rows].double())
            pages = st["table"][b].long()
            for (codes, scale), x, every in (((kc, ks), new[0], ks_all), ((vc, vs), new[1], vs_all)):
                for lo in range(first // S * S, nk[b], S):
                    hi = min(lo + S, nk[b])
                    a = max(lo, first)
                    alpha = x[a - first: hi - first].abs().amax(dim=(0, 2)) / 127
                    if a > lo:
                        before = scale[lo, :, 0].clone()
                        alpha = torch.maximum(alpha, before)
                        codes[lo:a] = torch.round(codes[lo:a] * (before / alpha)[:, None])
                    codes[a:hi] = torch.round(x[a - first: hi - first] / alpha[:, None])
                    scale[lo:hi] = alpha[:, None]
                    every[pages[lo // page], :, lo % page // S] = alpha
            k_val.append((kc * ks)[first:])
            v_val.append((vc * vs)[first:])
        if case["kind"] != "append":
            o.append(_exact_one(case, st, b, qb, kc * ks, vc * vs, nq[b], nk[b]))
    if o:
        out["o"] = torch.cat(o)
    if case["kind"] != "cached":
        out.update(q_rot=torch.cat(q_rot), k_scale=ks_all, v_scale=vs_all)
        if case["values"]:
            out.update(k_val=torch.cat(k_val), v_val=torch.cat(v_val))
    return out
