"""The serving operators around the prefill path, as cases that can be timed and whose outputs can be compared.

One pass is one call of one operator:
  "extend"  tokens are added to sequences that live in a paged key/value cache: pages off the free list, block tables, slots
  "rope"    queries and keys of a layer on their way into prefill attention: norm of each head, rotation by position
  "write"   the same for tokens whose keys and values go to the paged cache at their slots
  "decode"  attention of one new token per sequence over the paged cache

Shared layout of the paged cases: a cache of pages of `page` tokens, [pages][page][kv heads][128] ("token") or stored
[pages][kv heads][page][128] ("head"), pages of a sequence anywhere in it.
"""
import math
import random

import torch

own = False

HEAD_DIM = 128
EPS = 1e-6
# (query heads, KV heads): the layer shapes of the package's configurations and tests
HEADS = ((32, 4), (64, 8), (40, 8), (16, 16), (8, 2), (4, 2), (16, 1), (3, 1))
PAGES = (16, 24, 64, 128, 256)


def _case(kind, name=None, **more):
    c = {"kind": kind}
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decode step of 64 running requests: a token each, every 64th of them a new page
        _case("extend", "extend_64_seqs_1_token", seqs=64, lo=1, hi=32768, new_lo=1, new_hi=1, page=64, pad=0, mix=1),
        # a prompt batch after an empty cache, small pages, and a fixed buffer that the batch does not fill
        _case("extend", "extend_301_prompts", seqs=301, lo=0, hi=0, new_lo=200, new_hi=16384, page=16, pad=8191, mix=2),
        # the 128K configuration of the 32-head layer shape, on its way into prefill attention
        _case("rope", "rope_128k_32h", tokens=131072, hq=32, hkv=4, rot=128, pairs="half", norm=True, far=131072, packed=False),
        # a packed prompt of odd length whose model rotates half of the head in neighbouring pairs, far positions, no norms
        _case("rope", "rope_1003_40h_part", tokens=1003, hq=40, hkv=8, rot=64, pairs="neighbours", norm=False, far=1000003, packed=True),
        # one decode step of 48 requests: the new keys and values go to the cache
        _case("write", "write_48_tokens_32h", tokens=48, hq=32, hkv=4, rot=128, pairs="half", norm=True, far=32768, page=64, order="token",
              pad=0),
        # a prompt chunk of a 64-head layer into small pages, in a padded buffer
        _case("write", "write_8191_tokens_64h", tokens=8191, hq=64, hkv=8, rot=128, pairs="half", norm=True, far=131072, page=16,
              order="token", pad=257),
        # one request at the shortest length where the cache matters: latency
        _case("decode", "decode_1_seq_4001", seqs=1, lo=4001, hi=4001, hq=32, hkv=4, page=64, order="token", mix=3),
        # one request with the whole 128K context
        _case("decode", "decode_1_seq_128k", seqs=1, lo=131072, hi=131072, hq=32, hkv=4, page=128, order="token", mix=4),
        # a full serving batch of the 64-head layer, ragged lengths
        _case("decode", "decode_64_seqs_64h", seqs=64, lo=500, hi=16384, hq=64, hkv=8, page=64, order="head", mix=5),
        # many short chats, some of them still empty
        _case("decode", "decode_256_short", seqs=256, lo=0, hi=1500, hq=32, hkv=4, page=16, order="token", mix=6),
        # five query heads per KV head, pages that end inside any tile
        _case("decode", "decode_17_seqs_40h_page24", seqs=17, lo=1, hi=9001, hq=40, hkv=8, page=24, order="token", mix=7),
        # a KV head of its own for every query head
        _case("decode", "decode_32_seqs_16_16", seqs=32, lo=300, hi=8192, hq=16, hkv=16, page=256, order="head", mix=8),
    ]


def draw(rng):
    def length(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))
    kind = rng.choice(("extend", "rope", "write", "decode", "decode", "decode"))
    hq, hkv = rng.choice(HEADS)
    page, mix = rng.choice(PAGES), rng.randrange(1, 1 << 20)
    turn = {"rot": rng.choice((128, 128, 64, 96, 32)), "pairs": rng.choice(("half", "half", "neighbours")), "norm": rng.random() < 0.7}
    if kind == "extend":
        seqs = length(1, 512)
        if rng.random() < 0.5:      # a decode step, of one token or a few
            return _case(kind, seqs=seqs, lo=0, hi=length(1, 32768), new_lo=rng.choice((0, 1)), new_hi=rng.choice((1, 1, 5)), page=page,
                         pad=rng.choice((0, 0, 17)), mix=mix)
        return _case(kind, seqs=min(seqs, 300), lo=0, hi=rng.choice((0, 5000)), new_lo=1, new_hi=length(100, 16384), page=page,
                     pad=rng.choice((0, 4099)), mix=mix)
    if kind == "rope":
        return _case(kind, tokens=min(length(1, 131072), 131072 * 36 // (hq + hkv)), hq=hq, hkv=hkv, far=length(4096, 1 << 20),
                     packed=rng.random() < 0.5, **turn)
    if kind == "write":
        return _case(kind, tokens=length(1, 16384), hq=hq, hkv=hkv, far=length(4096, 1 << 20), page=page,
                     order=rng.choice(("token", "head")), pad=rng.choice((0, 0, 33)), **turn)
    seqs = length(1, 300)
    longest = max(1, min(131072, 700000 * 4 // (seqs * hkv)))
    hi = length(min(8, longest), longest)
    return _case(kind, seqs=seqs, lo=rng.choice((0, 1, hi, max(1, hi // 2))), hi=hi, hq=hq, hkv=hkv, page=page,
                 order=rng.choice(("token", "head")), mix=mix)


# ------------------------------------------------------------------------------------------------ sizes of a case


def _spread(rng, lo, hi, count):
    """Lengths between lo and hi, even over their logarithm; zeros among them where lo is zero."""
    low = max(1, lo)
    got = [int(round(math.exp(rng.uniform(math.log(low), math.log(hi))))) if hi > 0 else 0 for _ in range(count)]
    return [0 if lo == 0 and rng.random() < 0.05 else min(max(g, lo), hi) for g in got]


def _lens(case):
    lens = _spread(random.Random(case["mix"]), case["lo"], case["hi"], case["seqs"])
    lens[-1] = case["hi"]
    return lens


def _new_lens(case):
    return _spread(random.Random(case["mix"] + 1), case["new_lo"], case["new_hi"], case["seqs"])


def _ceil(a, b):
    return -(-a // b)


def _extend_sizes(case):
    past, new = _lens(case), _new_lens(case)
    old = sum(_ceil(p, case["page"]) for p in past)
    fresh = sum(_ceil(p + n, case["page"]) - _ceil(p, case["page"]) for p, n in zip(past, new))
    most = max(_ceil(p + n, case["page"]) for p, n in zip(past, new)) + 2
    return past, new, old, fresh, most


def work(case):
    kind = case["kind"]
    row = 2 * HEAD_DIM
    if kind == "extend":
        past, new, old, fresh, most = _extend_sizes(case)
        tokens = sum(new) + case["pad"]
        # lengths in and out, prefix sums, free pages in, table entries out (those of the pages that new tokens share read),
        # position and slot of every token
        return {"bytes": 4 * (4 * case["seqs"] + 2 * fresh + case["seqs"] + 2 * tokens), "flops": 0}
    if kind == "decode":
        lens = _lens(case)
        keys = sum(lens)
        bytes_ = 2 * row * keys * case["hkv"] + 2 * row * case["seqs"] * case["hq"] + 4 * case["seqs"] * case["hq"]
        bytes_ += 4 * case["seqs"] + 4 * sum(_ceil(n, case["page"]) for n in lens)
        return {"bytes": bytes_, "flops": 4 * HEAD_DIM * keys * case["hq"]}
    heads = case["hq"] + case["hkv"] * (2 if kind == "write" else 1)
    flops = case["tokens"] * (case["hq"] + case["hkv"]) * (3 * case["rot"] + (4 * HEAD_DIM if case["norm"] else 0))
    bytes_ = 2 * row * case["tokens"] * heads + 4 * case["tokens"] * (2 if kind == "write" else 1)
    if kind == "write":      # rows of a padded buffer that have no slot: their queries pass too
        bytes_ += case["pad"] * (2 * row * case["hq"] + 8)
        flops += case["pad"] * case["hq"] * (3 * case["rot"] + (4 * HEAD_DIM if case["norm"] else 0))
    return {"bytes": bytes_, "flops": flops}


# ------------------------------------------------------------------------------------------------ inputs


def _bf16(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16).mul_(scale)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _frequencies(rot):
    return (1.0e6 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


def _cache(g, pages, case):
    """Keys and values of recycled pages: whatever stood there before counts as well."""
    p, h = case["page"], case["hkv"]
    shape = (pages, p, h, HEAD_DIM) if case["order"] == "token" else (pages, h, p, HEAD_DIM)
    k, v = _bf16(g, *shape, scale=1.3), _bf16(g, *shape)
    return (k, v) if case["order"] == "token" else (k.transpose(1, 2), v.transpose(1, 2))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, s = case["kind"], {"kind": case["kind"]}
    if kind == "extend":
        past, new, old, fresh, most = _extend_sizes(case)
        page, pages = case["page"], old + fresh + 5
        order = torch.randperm(pages, generator=g, device="cuda").int()
        have = torch.tensor([_ceil(p, page) for p in past], device="cuda")
        at = torch.arange(most, device="cuda")
        first = (have.cumsum(0) - have)[:, None] + at
        table = torch.where(at < have[:, None], order[first.clamp(max=pages - 1)], -1)
        s.update(table=table, past=_ints(past), new=_ints(new), free=order[old:].contiguous(), page=page, pages=pages,
                 tokens=sum(new) + case["pad"])
        return s
    if kind == "decode":
        lens = _lens(case)
        page = case["page"]
        need = [_ceil(n, page) for n in lens]
        pages = sum(need) + 3
        order = torch.randperm(pages, generator=g, device="cuda").int()
        have, most = torch.tensor(need, device="cuda"), max(max(need), 1) + 1
        at = torch.arange(most, device="cuda")
        first = (have.cumsum(0) - have)[:, None] + at
        table = torch.where(at < have[:, None], order[first.clamp(max=pages - 1)], -1)
        k, v = _cache(g, pages, case)
        s.update(q=_bf16(g, case["seqs"], case["hq"], HEAD_DIM, scale=1.5), k=k, v=v, table=table, lens=_ints(lens), longest=max(max(lens), 1))
        return s
    t = case["tokens"] + case.get("pad", 0)
    heads = case["hq"] + 2 * case["hkv"]
    if kind == "write" or case["packed"]:      # slices of the projection's output
        x = _bf16(g, t, heads, HEAD_DIM, scale=2.0)
        q, k, v = x.split((case["hq"], case["hkv"], case["hkv"]), dim=1)
    else:                                      # the [layer][token][head][128] tensors of the prefill calls
        q, k, v = _bf16(g, 1, t, case["hq"], HEAD_DIM, scale=2.0), _bf16(g, 1, t, case["hkv"], HEAD_DIM, scale=2.0), None
    far = case["far"]
    s.update(q=q, k=k, inv_freq=_frequencies(case["rot"]), pairs=case["pairs"], magnitude=1.0 if case["rot"] == HEAD_DIM else 1.07)
    if case["norm"]:
        s["q_norm"], s["k_norm"] = (1.0 + 0.2 * torch.randn(HEAD_DIM, generator=g, device="cuda") for _ in range(2))
    else:
        s["q_norm"] = s["k_norm"] = None
    if kind == "rope" and not case["packed"]:
        start = int(torch.randint(0, max(1, far - t) + 1, (1,), generator=g, device="cuda"))
        s["positions"] = torch.arange(start, start + t, dtype=torch.int32, device="cuda")
    else:
        s["positions"] = torch.randint(0, far, (t,), generator=g, device="cuda", dtype=torch.int32)
    if kind == "write":
        page = case["page"]
        pages = _ceil(case["tokens"], page) + 7
        s["v"] = v
        s["k_cache"], s["v_cache"] = _cache(g, pages, case)
        slots = torch.randperm(pages * page, generator=g, device="cuda")[:t].int()
        slots[case["tokens"]:] = -1
        s["slots"] = slots
    return s


# ------------------------------------------------------------------------------------------------ one pass


def _plain_turn(x, norm, s):
    """Norm of each head and rotation by position: 32 bits, angles in 64."""
    y = x.float()
    if norm is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * norm
    half = s["inv_freq"].numel()
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()
    cos, sin = (angle.cos() * s["magnitude"]).float(), (angle.sin() * s["magnitude"]).float()
    if s["pairs"] == "half":
        a, b, rest = y[..., :half], y[..., half:2 * half], y[..., 2 * half:]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, rest), -1).to(x.dtype)
    a, b, rest = y[..., 0:2 * half:2], y[..., 1:2 * half:2], y[..., 2 * half:]
    return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2), rest), -1).to(x.dtype)


def _plain_extend(s):
    page, table, tokens, pages = s["page"], s["table"], s["tokens"], s["pages"]
    seqs, most = table.shape
    cap, dev = page * most, table.device
    total_new = s["new"].long().clamp(min=0).cumsum(0).clamp(max=tokens)
    cu = torch.cat((torch.zeros(1, dtype=torch.long, device=dev), total_new))
    past = s["past"].long().clamp(0, cap)
    lens = (past + cu.diff()).clamp(max=cap)
    first, last = (past + page - 1) // page, (lens + page - 1) // page
    need = last - first
    at = need.cumsum(0) - need
    index = torch.arange(most, device=dev)
    which = at[:, None] + index - first[:, None]
    entry = torch.where(which < s["free"].numel(), s["free"][which.clamp(0, s["free"].numel() - 1)], -1)
    table.copy_(torch.where((index >= first[:, None]) & (index < last[:, None]), entry, table))
    token = torch.arange(tokens, device=dev)
    seq = torch.searchsorted(cu[1:], token, right=True)
    there, seq = seq < seqs, seq.clamp(max=seqs - 1)
    pos = past[seq] + token - cu[seq]
    inside = table[seq, (pos // page).clamp(0, most - 1)].long()
    good = there & (pos < cap) & (inside >= 0) & (inside < pages)
    return {"table": table, "lens": lens.int(), "cu": cu.int(), "positions": torch.where(there, pos, 0).int(),
            "slots": torch.where(good, inside * page + pos % page, -1).int(), "used": need.sum().int().reshape(1)}


def _plain_decode(s):
    q, k, v, lens = s["q"], s["k"], s["v"], s["lens"]
    page, hkv = k.shape[1], k.shape[2]
    seqs, hq, d = q.shape
    at = torch.arange(s["longest"], device=q.device)
    held = at < lens[:, None]
    pages = torch.where(held, s["table"][:, at // page].long(), 0)
    scores = q.float().view(seqs, hkv, hq // hkv, d) @ k[pages, at % page].permute(0, 2, 3, 1).float() / math.sqrt(d)
    scores.masked_fill_(~held[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top.isinf(), torch.zeros_like(top), top)
    scores.sub_(top).exp_()
    total = scores.sum(-1, keepdim=True)
    out = scores @ v[pages, at % page].permute(0, 2, 1, 3).float() / torch.where(total == 0, torch.ones_like(total), total)
    return {"out": out.reshape(seqs, hq, d).to(q.dtype), "lse": (total.log() + top).reshape(seqs, hq)}


def run(s):
    kind = s["kind"]
    if own:
        import paper_2609_20971_b200 as rbs
        if kind == "extend":
            r = rbs.rbs_paged_extend(s["past"], s["new"], s["table"], s["free"], s["page"], s["pages"], s["tokens"])
            return {"table": s["table"], "lens": r.lens, "cu": r.cu, "positions": r.positions, "slots": r.slots, "used": r.used}
        if kind == "decode":
            out, lse = rbs.rbs_paged_decode(s["q"], s["k"], s["v"], s["table"], s["lens"], return_lse=True)
            return {"out": out, "lse": lse}
        turn = {"q_norm": s["q_norm"], "k_norm": s["k_norm"], "eps": EPS, "interleaved": s["pairs"] == "neighbours", "magnitude": s["magnitude"]}
        if kind == "rope":
            q, k = rbs.rbs_qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], **turn)
            return {"q": q, "k": k}
        q = rbs.rbs_qk_norm_rope_paged(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["inv_freq"], s["k_cache"], s["v_cache"], **turn)
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if kind == "extend":
        return _plain_extend(s)
    if kind == "decode":
        return _plain_decode(s)
    q, k = _plain_turn(s["q"], s["q_norm"], s), _plain_turn(s["k"], s["k_norm"], s)
    if kind == "rope":
        return {"q": q, "k": k}
    page = s["k_cache"].shape[1]
    rows = (s["slots"] >= 0).nonzero()[:, 0]
    slot = s["slots"][rows].long()
    s["k_cache"][slot // page, slot % page] = k[rows]
    s["v_cache"][slot // page, slot % page] = s["v"][rows]
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits


def _exact_turn(x, weight, s):
    """Each pair as a complex number, turned by exp(i * position * frequency)."""
    z = x.double()
    if weight is not None:
        z = z / (z.pow(2).sum(-1, keepdim=True) / HEAD_DIM + EPS).sqrt() * weight.double()
    n = s["inv_freq"].numel()
    phase = torch.outer(s["positions"].double(), s["inv_freq"].double())
    unit = torch.polar(torch.full_like(phase, s["magnitude"]), phase)[:, None]
    if s["pairs"] == "half":
        w = torch.complex(z[..., :n].contiguous(), z[..., n:2 * n].contiguous()) * unit
        z[..., :n], z[..., n:2 * n] = w.real, w.imag
    else:
        z[..., :2 * n] = torch.view_as_real(torch.view_as_complex(z[..., :2 * n].unflatten(-1, (n, 2)).contiguous()) * unit).flatten(-2)
    return z


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "extend":      # whole numbers: nothing to be off by
        return None
    if kind == "decode":
        group = case["hq"] // case["hkv"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
        for b, n in enumerate(_lens(case)):
            if n:
                pages = s["table"][b, :_ceil(n, case["page"])].long()
                k, v = (x[pages].flatten(0, 1)[:n].double().repeat_interleave(group, 1) for x in (s["k"], s["v"]))
                score = torch.einsum("hd,nhd->hn", s["q"][b].double(), k) / HEAD_DIM ** 0.5
                lse[b] = score.logsumexp(-1)
                out[b] = torch.einsum("hn,nhd->hd", score.softmax(-1), v)
        return {"out": out, "lse": lse}
    q, k = _exact_turn(s["q"], s["q_norm"], s), _exact_turn(s["k"], s["k_norm"], s)
    if kind == "rope":
        return {"q": q, "k": k}
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    slot = s["slots"][:case["tokens"]].long()
    k_cache[slot // case["page"], slot % case["page"]] = k[:case["tokens"]]
    v_cache[slot // case["page"], slot % case["page"]] = s["v"][:case["tokens"]].double()
    return {"q": q, "k_cache": k_cache, "v_cache": v_cache}
