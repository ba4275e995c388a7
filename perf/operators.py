"""What the operators around the paged KV cache are measured on.

Four operators of one serving step: `plan` (block tables and slot maps from request lengths), `rope` (rotary positions of
q and k, k and v written to their cache slots), `decode` (one query token per request over the paged cache, requests
in groups that share a prefix) and `prefill` (ragged prompts and chunks over the paged cache, with masks, a cap on the
scores or a bias by distance).  `run` computes them in elementary torch operations, or, with `own`, by the
framework's calls.  Lengths belong to a case; values and the order of pages belong to the seed.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_DEV = "cuda"


def _ceil(a, b):
    return -(-a // b)


# ---- cases ---------------------------------------------------------------------------------------
def listed():
    return [
        # a decode step's bookkeeping: 256 requests, one new token each, caches of the paper's short range
        dict(name="plan_decode_256", op="plan", n_req=256, old_lo=100, old_hi=1024, new_lo=1, new_hi=1, page=16, lens=11),
        # a step that mixes 1024 one-token requests with prompts: many pages handed out at once
        dict(name="plan_mixed_1040", op="plan", n_req=1040, old_lo=0, old_hi=4096, new_lo=1, new_hi=256, one_token=1024,
             page=32, lens=12),
        # rotary positions of a decode step, 7B-shaped: the fp32 projections (base + delta) of 256 tokens, half layout
        dict(name="rope_decode_256", op="rope", n_tok=256, n_q=32, n_kv=32, d=128, rot=128, inter=False, src="fp32", dt="bf16",
             page=16, max_pos=4096, lens=21),
        # rotary positions of a prompt batch (32 x 512 tokens), 70B-shaped heads, half the head rotated, interleaved
        # pairs, a table scaled for long contexts, 16-bit projections read out of one fused [q k v] row
        dict(name="rope_prompt_16384", op="rope", n_tok=16384, n_q=64, n_kv=8, d=128, rot=64, inter=True, src="bf16", dt="bf16",
             page=32, max_pos=32768, fused=True, factor=8.0, lens=22),
        # one request generates a token: nothing but latency
        dict(name="decode_one", op="decode", n_req=1, n_q=32, n_kv=32, d=128, dt="bf16", page=16, own_lo=900, own_hi=1000,
             groups="1:0", cap=0.0, bias=False, lens=31),
        # 7B-shaped decode, 256 requests of one adapter behind the same 4096-token system prompt
        dict(name="decode_shared_256", op="decode", n_req=256, n_q=32, n_kv=32, d=128, dt="bf16", page=16, own_lo=100,
             own_hi=1024, groups="256:4096", cap=0.0, bias=False, lens=32),
        # 70B-shaped heads (8 queries per KV head), adapters of uneven popularity, each with a prompt of its own; IEEE half,
        # capped scores; two requests share nothing
        dict(name="decode_groups_64", op="decode", n_req=64, n_q=64, n_kv=8, d=128, dt="fp16", page=32, own_lo=1, own_hi=1024,
             groups="31:8192 14:4096 9:1984 5:512 3:32 1:0 1:0", cap=30.0, bias=False, lens=33),
        # long caches, nothing shared: the plain single-token form
        dict(name="decode_long_64", op="decode", n_req=64, n_q=64, n_kv=8, d=128, dt="bf16", page=64, own_lo=2048, own_hi=4096,
             groups="64*1:0", cap=0.0, bias=False, lens=34),
        # the prompt batch of the 7B-shaped prefill workload: 32 requests of 512 tokens
        dict(name="prefill_32x512", op="prefill", n_req=32, n_q=32, n_kv=32, d=128, dt="bf16", page=16, new_lo=512, new_hi=512,
             old_lo=0, old_hi=0, docs=0, bidir=0, cap=0.0, bias=False, lens=41),
        # long prompts of the paper's long range, 7B-shaped: the largest case
        dict(name="prefill_long_16", op="prefill", n_req=16, n_q=32, n_kv=32, d=128, dt="bf16", page=64, new_lo=2048, new_hi=4096,
             old_lo=0, old_hi=0, docs=0, bidir=0, cap=0.0, bias=False, lens=42),
        # packed prompts: documents that do not see each other, the first one with a prefix that sees itself both
        # ways, capped scores, IEEE half, 8 queries per KV head, ragged lengths
        dict(name="prefill_docs_8", op="prefill", n_req=8, n_q=64, n_kv=8, d=128, dt="fp16", page=32, new_lo=333, new_hi=2777,
             old_lo=0, old_hi=0, docs=4, bidir=200, cap=30.0, bias=False, lens=43),
        # chunks of a few to some hundred tokens behind long caches, bias by distance, head size 64
        dict(name="prefill_chunks_24", op="prefill", n_req=24, n_q=32, n_kv=8, d=64, dt="bf16", page=16, new_lo=3, new_hi=260,
             old_lo=500, old_hi=9000, docs=0, bidir=0, cap=0.0, bias=True, lens=44),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _group_text(groups):
    return " ".join("%d:%d" % g for g in groups)


def _groups(case):
    """Groups of requests as (requests, shared tokens), from the text "requests:tokens ...", "n*requests:tokens" for n alike."""
    out = []
    for word in case["groups"].split():
        n, _, one = word.rpartition("*")
        k, p = one.split(":")
        out += [(int(k), int(p))] * int(n or 1)
    return out


def draw(rng):
    op = rng.choice(["plan", "rope", "decode", "decode", "prefill", "prefill"])
    lens = rng.randrange(1 << 20)
    page = rng.choice([16, 32, 64, 128])
    dt = rng.choice(["bf16", "fp16"])
    d = rng.choice([64, 128])
    g = rng.choice([1, 1, 2, 3, 4, 5, 8])
    if op == "plan":
        n = _log(rng, 1, 2048)
        return dict(op=op, n_req=n, old_lo=0, old_hi=_log(rng, 16, 8192), new_lo=rng.choice([0, 1]), new_hi=_log(rng, 1, 300),
                    one_token=rng.randrange(n + 1), page=page, lens=lens)
    if op == "rope":
        n_kv = rng.choice([1, 2, 4, 8, 16, 32])
        g = min(g, 64 // n_kv)
        rot = rng.choice([d, d // 2, d // 4, d - 24, 20])
        src = rng.choice(["fp32", dt])
        return dict(op=op, n_tok=_log(rng, 1, 16384), n_q=n_kv * g, n_kv=n_kv, d=d, rot=rot, inter=rng.random() < 0.5, src=src,
                    dt=dt, page=page, max_pos=rng.choice([4096, 32768]), fused=rng.random() < 0.5,
                    factor=rng.choice([1.0, 4.0]), lens=lens)
    cap, bias = rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.3
    if op == "decode":
        n = _log(rng, 1, 256)
        n_kv = rng.choice([1, 2, 4, 8, 8, 32]) if g == 1 else rng.choice([1, 2, 4, 8])
        groups, left = [], n
        while left:
            k = min(left, _log(rng, 1, n))
            groups.append((k, _log(rng, 1, 8192) // page * page if k > 1 and rng.random() < 0.8 else 0))
            left -= k
        hi = _log(rng, 8, 4096 if n <= 64 else 1024)
        case = dict(op=op, n_req=n, n_q=n_kv * g, n_kv=n_kv, d=d, dt=dt, page=page, own_lo=1, own_hi=hi,
                    groups=_group_text(groups), cap=cap, bias=bias, lens=lens)
        while work(case)["bytes"] > 2e9:
            groups = [(k, p // 2 // page * page) for k, p in groups]
            case["groups"], case["own_hi"] = _group_text(groups), max(1, case["own_hi"] * 3 // 4)
        return case
    n = _log(rng, 1, 32)
    n_kv = rng.choice([1, 2, 4, 8])
    g = min(g, 32 // n_kv)
    hi = _log(rng, 1, min(4096, 32768 // n))
    docs = rng.choice([0, 0, 2, 5])
    case = dict(op=op, n_req=n, n_q=n_kv * g, n_kv=n_kv, d=d, dt=dt, page=page, new_lo=max(1, hi // 9), new_hi=hi, old_lo=0,
                old_hi=0 if docs else rng.choice([0, _log(rng, 10, 8192)]), docs=docs, bidir=rng.choice([0, hi // 3]), cap=cap,
                bias=bias, lens=lens)
    while work(case)["flops"] > 6e11:
        case["n_req"] -= case["n_req"] // 2
        case["new_hi"] = max(case["new_lo"], case["new_hi"] * 3 // 4)
    return case


# ---- what a case's lengths are (host side, from the case alone) --------------------------------------
def _span(r, lo, hi, n):
    return [r.randint(lo, hi) for _ in range(n)]


def _plan_lens(case):
    r = random.Random(case["lens"])
    n = case["n_req"]
    old = _span(r, case["old_lo"], case["old_hi"], n)
    new = _span(r, case["new_lo"], case["new_hi"], n)
    one = set(r.sample(range(n), case.get("one_token", 0)))
    return old, [1 if i in one else x for i, x in enumerate(new)]


def _decode_lens(case):
    """Per request: tokens in its cache (its group's prefix included); first request of every group; prefixes."""
    r = random.Random(case["lens"])
    own_len = _span(r, case["own_lo"], case["own_hi"], case["n_req"])
    start, kv = [0], []
    for k, p in _groups(case):
        kv += [p + x for x in own_len[start[-1]:start[-1] + k]]
        start.append(start[-1] + k)
    return kv, start


def _prefill_lens(case):
    """Per request: new tokens, cache length after them; per token: first and one-past-last visible key."""
    r = random.Random(case["lens"])
    n = case["n_req"]
    new, old = _span(r, case["new_lo"], case["new_hi"], n), _span(r, case["old_lo"], case["old_hi"], n)
    lo, hi = [], []
    for q, o in zip(new, old):
        cuts = sorted({0, *(r.randint(0, q) for _ in range(max(0, case["docs"] - 1)))}) if case["docs"] else [0]
        first = cuts[1] if len(cuts) > 1 else q
        b = min(case["bidir"], first)
        j = 0
        for i in range(q):
            while j + 1 < len(cuts) and cuts[j + 1] <= i:
                j += 1
            lo.append(cuts[j] if case["docs"] else 0)
            hi.append(o + max(i + 1, b if i < b else 0))
    return new, [o + q for o, q in zip(old, new)], lo, hi


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=_DEV)


def _gen(seed):
    g = torch.Generator(device=_DEV)
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype, mul=1.0):
    out = torch.empty(shape, dtype=dtype, device=_DEV)
    flat = out.view(-1)
    step = 1 << 27
    for i in range(0, flat.numel(), step):      # in pieces: the fp32 draw of a whole cache would double its memory
        n = min(step, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=g, device=_DEV) * mul
    return out


def _slopes(n):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / n) for h in range(n)], dtype=torch.float32, device=_DEV)


# ---- inputs ----------------------------------------------------------------------------------------
def _plan_inputs(case, seed):
    old, new = _plan_lens(case)
    P, n = case["page"], case["n_req"]
    have, need = [_ceil(o, P) for o in old], [_ceil(o + k, P) for o, k in zip(old, new)]
    used, fresh = sum(have), sum(need) - sum(have)
    g = _gen(seed)
    perm = torch.randperm(used + fresh + 5, generator=g, device=_DEV).to(torch.int32)
    width = max(1, max(need)) + 3
    table = torch.full((n, width), -1, dtype=torch.int32)
    host, at = perm.cpu(), 0
    for r, h in enumerate(have):
        table[r, :h] = host[at:at + h]
        at += h
    return dict(old=_i32(old), new=_i32(new), table=table.to(_DEV), free=perm[used:].contiguous(), max_tokens=sum(new) + 7)


def _rope_freqs(case):
    half = case["rot"] // 2
    return [10000.0 ** (-i / half) / case.get("factor", 1.0) for i in range(half)]


def _rope_table(case):
    ang = torch.arange(case["max_pos"], dtype=torch.float64, device=_DEV)[:, None] * torch.tensor(
        _rope_freqs(case), dtype=torch.float64, device=_DEV)
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()


def _rope_inputs(case, seed):
    g = _gen(seed)
    n, hq, hk, d = case["n_tok"], case["n_q"], case["n_kv"], case["d"]
    src = _DT[case["src"]]
    if case.get("fused"):
        row = _randn(g, (n, hq + 2 * hk, d), src)
        q, k, v = row[:, :hq], row[:, hq:hq + hk], row[:, hq + hk:]
    else:
        q, k, v = _randn(g, (n, hq, d), src), _randn(g, (n, hk, d), src), _randn(g, (n, hk, d), src)
    pages = _ceil(n, case["page"]) + 2
    slots = torch.randperm(pages * case["page"], generator=g, device=_DEV)[:n].to(torch.int32)
    pos = torch.randint(0, case["max_pos"], (n,), generator=g, device=_DEV, dtype=torch.int32)
    cache = (pages, hk, case["page"], d)
    return dict(q=q, k=k, v=v, pos=pos, slots=slots, k_cache=_randn(g, cache, _DT[case["dt"]]),
                v_cache=_randn(g, cache, _DT[case["dt"]]))


def _tables(g, kv, P, shared):
    """Block tables over shuffled pages; shared: per request (first request of the group, shared pages)."""
    need = [_ceil(n, P) for n in kv]
    total = sum(need)
    host = torch.randperm(total, generator=g, device=_DEV).to(torch.int32).cpu()
    table, at = torch.zeros((len(kv), max(1, max(need))), dtype=torch.int32), 0
    for r, n in enumerate(need):
        first, pages = shared[r] if shared else (r, 0)
        keep = pages if first != r else 0
        table[r, :keep] = table[first, :keep]
        table[r, keep:n] = host[at:at + n - keep]
        at += n - keep
    # only the pages in use make up the cache: renumber them
    order = torch.argsort(host[:at]).to(torch.int32)
    rank = torch.zeros(total, dtype=torch.int32)
    rank[host[:at].long()[order.long()]] = torch.arange(at, dtype=torch.int32)
    for r, n in enumerate(need):
        table[r, :n] = rank[table[r, :n].long()]
    return table.to(_DEV), at


def _attn_inputs(case, seed):
    g = _gen(seed)
    P, dt = case["page"], _DT[case["dt"]]
    s = dict(case=case, scale=1.0 / math.sqrt(case["d"]), cap=case["cap"])
    if case["op"] == "decode":
        kv, start = _decode_lens(case)
        shared = []
        for i, (k, p) in enumerate(_groups(case)):
            shared += [(start[i], p // P)] * k
        n_tok, s["h_new"], s["lo"], s["hi"] = len(kv), [1] * len(kv), None, None
        s["group_start"], s["prefix"], s["tok_start"] = _i32(start), _i32([p for _, p in _groups(case)]), None
    else:
        new, kv, lo, hi = _prefill_lens(case)
        shared = None
        n_tok, s["h_new"] = sum(new), new
        s["lo"] = _i32(lo) if case["docs"] else None
        s["hi"] = _i32(hi) if case["bidir"] else None
        at = [0]
        for q in new:
            at.append(at[-1] + q)
        s["tok_start"] = _i32(at)
    s["h_kv"], s["kv_len"] = kv, _i32(kv)
    s["table"], pages = _tables(g, kv, P, shared)
    cache = (max(1, pages), case["n_kv"], P, case["d"])
    s["k_cache"], s["v_cache"] = _randn(g, cache, dt), _randn(g, cache, dt)
    s["q"] = _randn(g, (n_tok, case["n_q"], case["d"]), dt, 2.0)     # scores of a spread of 2, as trained heads have
    s["slopes"] = _slopes(case["n_q"]) if case["bias"] else None
    return s


def prepare(case, seed):
    """Inputs, the rotary table, and the buffers that a server keeps from step to step."""
    op = case["op"]
    if op == "plan":
        s = _plan_inputs(case, seed)
    elif op == "rope":
        s = _rope_inputs(case, seed)
        if own:
            import paper_2608_05483_b200 as P
            f = case.get("factor", 1.0)
            s["table"] = P.rope_table(case["rot"], case["max_pos"], scaling="linear" if f != 1.0 else "none", factor=f)
        else:
            s["table"] = _rope_table(case)
        s["q_out"] = torch.empty((case["n_tok"], case["n_q"], case["d"]), dtype=_DT[case["dt"]], device=_DEV)
    else:
        s = _attn_inputs(case, seed)
        s["out"] = torch.empty_like(s["q"])
        if own:
            import paper_2608_05483_b200 as P
            s["ws"] = P.attn_paged_workspace(s["q"], s["k_cache"], s["kv_len"].numel())
    s["case"] = case
    return s


# ---- the plain forms -------------------------------------------------------------------------------
def _plain_plan(s):
    P, old, new = s["case"]["page"], s["old"].long(), s["new"].long()
    n, T = old.numel(), s["max_tokens"]
    zero = torch.zeros(1, dtype=torch.int64, device=old.device)
    start = torch.cat([zero, torch.cumsum(new, 0)])
    have, need = (old + P - 1) // P, (old + new + P - 1) // P
    fresh = need - have
    first = torch.cumsum(fresh, 0) - fresh
    col = torch.arange(s["table"].shape[1], device=old.device)[None, :]
    take = (col >= have[:, None]) & (col < need[:, None])
    idx = (first[:, None] + col - have[:, None]).clamp(0, s["free"].numel() - 1)
    table = torch.where(take, s["free"][idx], s["table"])
    t = torch.arange(T, device=old.device)
    real = t < start[-1]
    req = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp(max=n - 1)
    pos = old[req] + t - start[req]
    slot = table[req, (pos // P).clamp(0, table.shape[1] - 1)].long() * P + pos % P
    gone = torch.full_like(t, -1)
    pick = lambda x: torch.where(real, x, gone).to(torch.int32)
    return dict(block_table=table, tok_start=start.to(torch.int32), positions=pick(pos), tok_req=pick(req), slots=pick(slot),
                kv_len=(old + new).to(torch.int32), cursor=fresh.sum().reshape(1).to(torch.int32))


def _plain_rotate(x, cos, sin, rot, inter):
    x = x.float()
    r, rest = x[..., :rot], x[..., rot:]
    if inter:
        a, b = r[..., 0::2], r[..., 1::2]
    else:
        a, b = r[..., :rot // 2], r[..., rot // 2:]
    c, s = cos[:, None, :], sin[:, None, :]
    u, w = a * c - b * s, b * c + a * s
    r = torch.stack([u, w], -1).flatten(-2) if inter else torch.cat([u, w], -1)
    return torch.cat([r, rest], -1)


def _plain_rope(s):
    case = s["case"]
    cs = s["table"][s["pos"].long()]
    cos, sin = cs[..., 0], cs[..., 1]
    dt = s["k_cache"].dtype
    page, off = s["slots"].long() // case["page"], s["slots"].long() % case["page"]
    s["q_out"].copy_(_plain_rotate(s["q"], cos, sin, case["rot"], case["inter"]).to(dt))
    s["k_cache"][page, :, off] = _plain_rotate(s["k"], cos, sin, case["rot"], case["inter"]).to(dt)
    s["v_cache"][page, :, off] = s["v"].to(dt)
    return dict(q=s["q_out"], k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_attn(s):
    case = s["case"]
    P, hk = case["page"], case["n_kv"]
    g, at = case["n_q"] // hk, 0
    out = s["out"]
    for r, (n, kv) in enumerate(zip(s["h_new"], s["h_kv"])):
        pages = s["table"][r, :_ceil(kv, P)].long()
        K = s["k_cache"][pages].transpose(0, 1).reshape(hk, -1, case["d"])[:, :kv].float()
        V = s["v_cache"][pages].transpose(0, 1).reshape(hk, -1, case["d"])[:, :kv].float()
        q = s["q"][at:at + n].float().view(n, hk, g, -1).permute(1, 2, 0, 3).reshape(hk, g * n, -1)
        sc = (q @ K.transpose(1, 2) * s["scale"]).view(hk, g, n, kv)
        if s["cap"]:
            sc = s["cap"] * torch.tanh(sc / s["cap"])
        key = torch.arange(kv, device=sc.device)
        pos = torch.arange(kv - n, kv, device=sc.device)
        if s["slopes"] is not None:
            sc = sc - s["slopes"].view(hk, g, 1, 1) * (pos[:, None] - key[None, :]).abs().float()
        hi = s["hi"][at:at + n] if s["hi"] is not None else pos + 1
        see = key[None, :] < hi[:, None]
        if s["lo"] is not None:
            see = see & (key[None, :] >= s["lo"][at:at + n][:, None])
        sc = sc.masked_fill(~see, float("-inf"))
        m = sc.amax(-1, keepdim=True)
        p = torch.exp(sc - torch.where(m == float("-inf"), torch.zeros_like(m), m))
        l = p.sum(-1, keepdim=True)
        o = (p.view(hk, g * n, kv) @ V).view(hk, g, n, -1) / torch.where(l == 0, torch.ones_like(l), l)
        out[at:at + n] = o.permute(2, 0, 1, 3).reshape(n, hk * g, -1).to(out.dtype)
        at += n
    return out


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"plan": _plain_plan, "rope": _plain_rope}.get(op, _plain_attn)(state)
    import paper_2608_05483_b200 as P
    s, case = state, state["case"]
    if op == "plan":
        p = P.kv_plan(s["old"], s["new"], case["page"], s["free"], s["table"], s["max_tokens"])
        return dict(block_table=s["table"], tok_start=p.tok_start, positions=p.positions, tok_req=p.tok_req, slots=p.slots,
                    kv_len=p.kv_len, cursor=p.cursor)
    if op == "rope":
        P.rope_cache(s["q"], s["k"], s["v"], s["pos"], s["slots"], s["table"], s["k_cache"], s["v_cache"], q_out=s["q_out"],
                     interleaved=case["inter"])
        return dict(q=s["q_out"], k_cache=s["k_cache"], v_cache=s["v_cache"])
    if op == "decode":
        P.attn_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["kv_len"], s["scale"], group_start=s["group_start"],
                     prefix_len=s["prefix"], softcap=s["cap"], slopes=s["slopes"], out=s["out"], workspace=s["ws"])
    else:
        P.attn_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["kv_len"], s["scale"], tok_start=s["tok_start"],
                     softcap=s["cap"], slopes=s["slopes"], key_lo=s["lo"], key_hi=s["hi"], out=s["out"], workspace=s["ws"])
    return s["out"]


# ---- what a pass cannot do without ---------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "plan":
        old, new = _plan_lens(case)
        P = case["page"]
        fresh = sum(_ceil(o + k, P) - _ceil(o, P) for o, k in zip(old, new))
        touched = sum(_ceil(o + k, P) - o // P for o, k in zip(old, new))
        n, t = case["n_req"], sum(new) + 7
        return {"bytes": 8 * n + 4 * fresh + 4 * touched + 4 * fresh + 4 * (n + 1) + 12 * t + 4 * n + 4, "flops": 0}
    if op == "rope":
        n, d = case["n_tok"], case["d"]
        i, o = (4 if case["src"] == "fp32" else 2), 2
        heads = case["n_q"] + 2 * case["n_kv"]
        return {"bytes": n * (heads * d * (i + o) + 8 + 4 * case["rot"]),
                "flops": 3 * n * (case["n_q"] + case["n_kv"]) * case["rot"]}
    if op == "decode":
        kv, start = _decode_lens(case)
        tokens = sum(kv) - sum((k - 1) * p for k, p in _groups(case))
        n_tok, pairs = case["n_req"], sum(kv)
    else:
        new, kv, lo, hi = _prefill_lens(case)
        tokens, n_tok = sum(kv), sum(new)
        pairs = sum(max(0, h - l) for l, h in zip(lo, hi))
    row = case["n_kv"] * case["d"] * 2
    return {"bytes": 2 * tokens * row + 2 * n_tok * case["n_q"] * case["d"] * 2, "flops": 4 * pairs * case["n_q"] * case["d"]}


# ---- the definitions in 64 bits ---------------------------------------------------------------------
def _exact_plan(case, s):
    """Token by token, page by page, on the host."""
    P = case["page"]
    old, new = s["old"].tolist(), s["new"].tolist()
    table, free, taken = s["table"].tolist(), s["free"].tolist(), 0
    start, pos, req, slots = [0], [], [], []
    for r in range(len(old)):
        for i in range(new[r]):
            p = old[r] + i
            if p % P == 0:
                table[r][p // P] = free[taken]
                taken += 1
            pos.append(p)
            req.append(r)
            slots.append(table[r][p // P] * P + p % P)
        start.append(start[-1] + new[r])
    pad = [-1] * (s["max_tokens"] - len(pos))
    return dict(block_table=_i32(table), tok_start=_i32(start), positions=_i32(pos + pad), tok_req=_i32(req + pad),
                slots=_i32(slots + pad), kv_len=_i32([o + k for o, k in zip(old, new)]), cursor=_i32([taken]))


def _exact_rope(case, s):
    """A rotation is a complex product with exp(i * position * frequency)."""
    rot, half = case["rot"], case["rot"] // 2
    w = torch.tensor(_rope_freqs(case), dtype=torch.float64, device=_DEV)
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device=_DEV), s["pos"].double()[:, None] * w[None, :])[:, None, :]

    def rotate(x):
        y = x.double().clone()
        re = slice(0, rot, 2) if case["inter"] else slice(0, half)
        im = slice(1, rot, 2) if case["inter"] else slice(half, rot)
        z = torch.complex(y[..., re].contiguous(), y[..., im].contiguous()) * turn
        y[..., re], y[..., im] = z.real, z.imag
        return y

    P = case["page"]
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    flat = lambda c: c.permute(0, 2, 1, 3).reshape(-1, c.shape[1], c.shape[3])
    back = lambda f: f.view(-1, P, f.shape[1], f.shape[2]).permute(0, 2, 1, 3).contiguous()
    fk, fv = flat(kc), flat(vc)
    fk[s["slots"].long()] = rotate(s["k"])
    fv[s["slots"].long()] = s["v"].double()
    return dict(q=rotate(s["q"]), k_cache=back(fk), v_cache=back(fv))


def _exact_attn(case, s):
    """Request by request and KV head by KV head."""
    P, hk = case["page"], case["n_kv"]
    g = case["n_q"] // hk
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=_DEV)
    at = 0
    for r, (n, kv) in enumerate(zip(s["h_new"], s["h_kv"])):
        where = torch.arange(kv, device=_DEV)
        page, off = s["table"][r].long()[where // P], where % P
        own_pos = kv - n + torch.arange(n, device=_DEV)
        first = torch.zeros_like(own_pos) if s["lo"] is None else s["lo"][at:at + n].long()
        end = own_pos + 1 if s["hi"] is None else s["hi"][at:at + n].long()
        hidden = (where[None, :] < first[:, None]) | (where[None, :] >= end[:, None])
        empty = hidden.all(1)
        gap = (own_pos[:, None] - where[None, :]).abs().double()
        for h in range(hk):
            K, V = s["k_cache"][page, h, off].double(), s["v_cache"][page, h, off].double()
            for j in range(h * g, (h + 1) * g):
                z = s["q"][at:at + n, j].double() @ K.T * s["scale"]
                if s["cap"]:
                    z = torch.tanh(z / s["cap"]) * s["cap"]
                if s["slopes"] is not None:
                    z = z - s["slopes"][j].double() * gap
                z[hidden] = -math.inf
                z[empty] = 0.0
                o = torch.softmax(z, -1) @ V
                o[empty] = 0.0
                out[at:at + n, j] = o
        at += n
    return out


def exact(case, seed):
    op = case["op"]
    if op == "plan":
        return _exact_plan(case, _plan_inputs(case, seed))
    if op == "rope":
        return _exact_rope(case, _rope_inputs(case, seed))
    s = _attn_inputs(case, seed)
    if case["op"] == "decode" and case["n_req"] * case["n_q"] > 20000 or work(case)["flops"] > 3e12:
        return None
    return _exact_attn(case, s)
