"""One attention layer of a multi-LoRA server, step by step, on the library's calls.

Requests of several adapters share one batch.  A step is

    plan      pages, slots and positions of the new tokens       kv_plan
    delta     q, k, v += s (x A) B, each with its adapter         bucket + lora_delta_group (fp32 y)
    rotary    q and k to their positions, k and v to the cache    rope_cache (fp32 in, bf16 out)
    attention over the paged cache                                attn_paged
    delta     of the output projection                            lora_delta

The first step takes the prompts; the later ones generate a token per request.  All prompts of an adapter begin with the
same tokens (its system prompt): their pages are shared from the second request on, and the single-token steps read
them once per adapter, the requests being sorted by adapter.

    python examples/serve_layer.py [--steps N]
"""
import argparse
import sys
from pathlib import Path

import torch

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))
import paper_2608_05483_b200 as P  # noqa: E402


class Layer:
    """Base weights and adapter pools of q, k, v, o, and the layer's part of the paged cache."""

    def __init__(self, hidden=512, n_q=4, n_kv=2, head_dim=128, n_adapters=3, rank=16, n_pages=256, page=16, max_tokens=512, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std).bfloat16()
        self.n_q, self.n_kv, self.d, self.page, self.hidden = n_q, n_kv, head_dim, page, hidden
        widths = [n_q * head_dim, n_kv * head_dim, n_kv * head_dim, hidden]
        ins = [hidden, hidden, hidden, n_q * head_dim]
        self.W = [rnd(i, o, std=i ** -0.5) for i, o in zip(ins, widths)]
        self.A = [[rnd(i, rank, std=i ** -0.5) for _ in range(n_adapters)] for i in ins]
        self.B = [[rnd(rank, o, std=rank ** -0.5) for _ in range(n_adapters)] for o in widths]
        self.ctx = P.Context(max_tokens, n_adapters)
        for proj in range(4):
            self.ctx.register_pool(0, proj, ins[proj], widths[proj], [rank] * n_adapters, [0.5] * n_adapters, self.A[proj], self.B[proj])
        self.k_cache = torch.zeros((n_pages, n_kv, page, head_dim), dtype=torch.bfloat16, device="cuda")
        self.v_cache = torch.zeros_like(self.k_cache)
        self.table = P.rope_table(head_dim, 4096)
        self.n_adapters = n_adapters

    def step(self, x, ids, plan, block_table, **attn):
        """x [n_tok, hidden] bf16; ids int32 [n_tok]: every token's adapter.  Returns y [n_tok, hidden], fp32."""
        n = x.shape[0]
        self.ctx.bucket(ids, self.n_adapters)
        q, k, v = ((x @ w).float() for w in self.W[:3])                   # the base projections
        self.ctx.lora_delta_group([x, x, x], ids, [0, 0, 0], [0, 1, 2], [q, k, v])
        heads = lambda y, h: y.view(n, h, self.d)
        q = P.rope_cache(heads(q, self.n_q), heads(k, self.n_kv), heads(v, self.n_kv), plan.positions[:n], plan.slots[:n], self.table,
                         self.k_cache, self.v_cache)
        o, _ = P.attn_paged(q, self.k_cache, self.v_cache, block_table, plan.kv_len, self.d ** -0.5, **attn)
        o = o.view(n, -1)
        y = (o @ self.W[3]).float()
        self.ctx.lora_delta(o, ids, 0, 3, y)
        return y


def serve(layer, system, prompts, adapters, new_tokens):
    """system[a]: the adapter's shared prompt [n, hidden]; prompts[r]: request r's own [n, hidden]; adapters[r], ascending;
    new_tokens: inputs [n_req, hidden] of the single-token steps.  Returns every request's outputs, prompt first."""
    dev, page = "cuda", layer.page
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    n_req, n_ad = len(prompts), len(system)
    # whole pages of a system prompt are shared; the rest of it is each request's own
    shared = [s.shape[0] // page * page for s in system]
    free = torch.arange(layer.k_cache.shape[0], dtype=torch.int32, device=dev)
    width = 64
    outs = [[] for _ in range(n_req)]

    # the system prompts' whole pages, one "request" per adapter
    base = torch.full((n_ad, width), -1, dtype=torch.int32, device=dev)
    x = torch.cat([s[:n] for s, n in zip(system, shared)])
    plan = P.kv_plan(i32([0] * n_ad), i32(shared), page, free, base, x.shape[0])
    ids = torch.repeat_interleave(torch.arange(n_ad, dtype=torch.int32, device=dev), i32(shared).long())
    y_sys = layer.step(x, ids, plan, base, tok_start=plan.tok_start)
    cursor = plan.cursor

    # the requests: the adapter's pages in front, then their own prompt
    table = base[torch.tensor(adapters, device=dev)].contiguous()
    own = [torch.cat([system[a][shared[a]:], p]) for a, p in zip(adapters, prompts)]
    plan = P.kv_plan(i32([shared[a] for a in adapters]), i32([o.shape[0] for o in own]), page, free, table, sum(o.shape[0] for o in own),
                     cursor=cursor)
    ad = i32(adapters)
    y = layer.step(torch.cat(own), ad[plan.tok_req.long()].contiguous(), plan, table, tok_start=plan.tok_start)
    at = [0]
    for s in shared:
        at.append(at[-1] + s)
    for r, part in enumerate(torch.split(y, [o.shape[0] for o in own])):
        outs[r] += [y_sys[at[adapters[r]]:at[adapters[r] + 1]], part]

    # single tokens, the requests of an adapter as a group
    starts = [sum(a < g for a in adapters) for g in range(n_ad)] + [n_req]
    groups, prefix, one = i32(starts), i32(shared), i32([1] * n_req)
    for x in new_tokens:
        plan = P.kv_plan(plan.kv_len, one, page, free, table, n_req, cursor=plan.cursor)
        y = layer.step(x, ad, plan, table, group_start=groups, prefix_len=prefix)
        for r in range(n_req):
            outs[r].append(y[r:r + 1])
    assert int(plan.cursor) <= free.shape[0], "out of pages"
    return [torch.cat(o) for o in outs]


def reference(layer, x, adapter):
    """The same layer over one request's whole sequence, in 64 bits."""
    W = [w.double() + 0.5 * (a[adapter].double() @ b[adapter].double()) for w, a, b in zip(layer.W, layer.A, layer.B)]
    n, d = x.shape[0], layer.d
    q, k, v = (x.double() @ w for w in W[:3])
    pos = torch.arange(n, device=x.device)
    cs = layer.table[pos].double()

    def turn(y, h):
        a, b = y.view(n, h, 2, d // 2).unbind(2)
        c, s = cs[:, None, :, 0], cs[:, None, :, 1]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    g = layer.n_q // layer.n_kv
    q, k = turn(q, layer.n_q), turn(k, layer.n_kv).repeat_interleave(g, 1)
    v = v.view(n, layer.n_kv, d).repeat_interleave(g, 1)
    s = torch.einsum("thd,khd->htk", q, k) * d ** -0.5
    s = s.masked_fill(pos[None, :] > pos[:, None], float("-inf"))
    return torch.einsum("htk,khd->thd", torch.softmax(s, -1), v).reshape(n, -1) @ W[3]


def main(steps=4):
    layer = Layer()
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda n: torch.randn(n, layer.hidden, generator=g, device="cuda").bfloat16()
    system = [rnd(n) for n in (70, 16, 5)]
    adapters = [0, 0, 0, 0, 0, 1, 1, 2]
    prompts = [rnd(n) for n in (7, 1, 30, 12, 3, 25, 2, 40)]
    new = [rnd(len(prompts)) for _ in range(steps)]
    outs = serve(layer, system, prompts, adapters, new)
    worst = 0.0
    for r, a in enumerate(adapters):
        x = torch.cat([system[a], prompts[r], *[t[r:r + 1] for t in new]])
        want = reference(layer, x, a)
        worst = max(worst, float((outs[r].double() - want).abs().max() / want.abs().max()))
    print(f"serve_layer: {len(prompts)} requests, {steps} single-token steps, worst error {worst:.2e} of the largest output")
    layer.ctx.close()
    return worst


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=4)
    main(ap.parse_args().steps)
