"""Attention over the paged cache, rotary positions and the step's plan on the GPU, against 64-bit references."""
import math

import numpy as np
import pytest
import torch

import paper_2608_05483_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")

# Unit roundoff of the 16-bit types.  An output element is off by at most u (rounding of the weights) plus u (rounding of
# the result) times the weighted mean of |v|; fp32 sums and the fast exponentials add a few 1e-5; weights of half
# precision below its normal range are off by up to 2^-25 each.
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


class Batch:
    """A ragged batch over a shuffled paged cache; every slot that no request uses holds NaN."""

    def __init__(self, seed, kv, new=None, hq=4, hk=2, d=128, page=16, dtype=torch.bfloat16, groups=None, prefix=None,
                 q_pad=0, joint_cache=False):
        g = torch.Generator().manual_seed(seed)
        self.kv, self.new, self.page, self.d, self.hq, self.hk, self.dtype = list(kv), new, page, d, hq, hk, dtype
        n_req = len(kv)
        lens = new if new is not None else [1] * n_req
        self.tok = [0]
        for n in lens:
            self.tok.append(self.tok[-1] + n)
        need = [-(-n // page) for n in kv]
        pages = sum(need) + 3
        order = torch.randperm(pages, generator=g).tolist()
        table = torch.full((n_req, max(1, max(need)) + 2), 7 * pages, dtype=torch.int32)     # unused entries: no page at all
        shape = (pages, 2, hk, page, d) if joint_cache else (2, pages, hk, page, d)
        cache = torch.full(shape, NAN, dtype=dtype)
        self.K = cache[:, 0] if joint_cache else cache[0]
        self.V = cache[:, 1] if joint_cache else cache[1]
        self.rows = []
        first_of = {}
        if groups is not None:
            for a, b, p in zip(groups, groups[1:], prefix):
                for r in range(a, b):
                    first_of[r] = (a, p)
        for r, n in enumerate(kv):
            k = torch.randn((n, hk, d), generator=g).to(dtype)
            v = torch.randn((n, hk, d), generator=g).to(dtype)
            first, p = first_of.get(r, (r, 0))
            if first != r:
                p = min(p, n, len(self.rows[first][0]))
                k[:p], v[:p] = self.rows[first][0][:p], self.rows[first][1][:p]
            self.rows.append((k, v))
            for b in range(need[r]):
                if first != r and (b + 1) * page <= p:
                    table[r, b] = table[first, b]
                    continue
                table[r, b] = order.pop()
                m = min(page, n - b * page)
                self.K[table[r, b], :, :m] = k[b * page:b * page + m].transpose(0, 1)
                self.V[table[r, b], :, :m] = v[b * page:b * page + m].transpose(0, 1)
        row = torch.randn((self.tok[-1], hq + q_pad, d), generator=g).to(dtype).to(DEV)
        self.q = row[:, :hq]
        cache = cache.to(DEV)
        self.K = cache[:, 0] if joint_cache else cache[0]
        self.V = cache[:, 1] if joint_cache else cache[1]
        self.table, self.kv_len = table.to(DEV), _ints(kv)
        self.tok_start = _ints(self.tok) if new is not None else None
        self.scale = 1.0 / math.sqrt(d)

    def run(self, groups=None, prefix=None, **kw):
        if groups is not None:
            kw.update(group_start=_ints(groups), prefix_len=_ints(prefix))
        out, ws = P.attn_paged(self.q, self.K, self.V, self.table, self.kv_len, kw.pop("scale", self.scale),
                               tok_start=self.tok_start, **kw)
        torch.cuda.synchronize()
        rc, status = P.plora_attn_status(ws.data_ptr())
        assert rc == 0 and status == 0
        return out

    def reference(self, softcap=0.0, slopes=None, key_lo=None, key_hi=None, scale=None):
        """(output, weighted mean of |v|), 64 bits, token by token's definition."""
        scale = self.scale if scale is None else scale
        G = self.hq // self.hk
        out = torch.zeros((self.tok[-1], self.hq, self.d), dtype=torch.float64, device=DEV)
        mean = torch.zeros_like(out)
        for r, (k, v) in enumerate(self.rows):
            a, b, n = self.tok[r], self.tok[r + 1], self.kv[r]
            if a == b or n == 0:
                continue
            K = k.to(DEV).double().repeat_interleave(G, dim=1)
            V = v.to(DEV).double().repeat_interleave(G, dim=1)
            s = torch.einsum("thd,khd->htk", self.q[a:b].double(), K) * scale
            if softcap:
                s = softcap * torch.tanh(s / softcap)
            pos = torch.arange(n - (b - a), n, device=DEV)
            key = torch.arange(n, device=DEV)
            if slopes is not None:
                s = s - slopes.double()[:, None, None] * (pos[:, None] - key).abs()
            lo = key_lo[a:b].long().clamp(min=0) if key_lo is not None else torch.zeros_like(pos)
            hi = key_hi[a:b].long() if key_hi is not None else pos + 1
            see = (key >= lo[:, None]) & (key < hi[:, None])
            w = torch.softmax(s.masked_fill(~see, -math.inf), -1).nan_to_num(0.0)
            out[a:b] = torch.einsum("htk,khd->thd", w, V)
            mean[a:b] = torch.einsum("htk,khd->thd", w, V.abs())
        return out, mean

    def check(self, got, ref):
        want, mean = ref
        u = ROUND[self.dtype]
        tol = (2 * u + 1e-4) * mean + (max(self.kv) + 1) * 2.0 ** -25 * 5.0 + 1e-6
        err = (got.double() - want).abs()
        assert torch.isfinite(got).all()
        bad = err > tol
        assert not bad.any(), (int(bad.sum()), float((err / tol).max()), bad.nonzero()[0].tolist())


MIXED_NEW = [1, 3, 0, 17, 130, 300, 2, 1]
MIXED_KV = [1, 90, 40, 17, 700, 300, 2, 513]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,page,hq,hk", [(128, 16, 2, 2), (128, 64, 8, 1), (128, 128, 5, 1), (64, 32, 6, 2), (64, 128, 16, 1),
                                          (128, 32, 24, 1), (64, 16, 100, 1)])
def test_ragged_batch(d, page, hq, hk, dtype):
    b = Batch(1, MIXED_KV, MIXED_NEW, hq=hq, hk=hk, d=d, page=page, dtype=dtype)
    b.check(b.run(), b.reference())


@pytest.mark.parametrize("hq,hk", [(3, 3), (16, 2)])
@pytest.mark.parametrize("cap,bias", [(20.0, False), (0.0, True), (5.0, True)])
@pytest.mark.parametrize("d", [64, 128])
def test_capped_and_biased_scores(d, cap, bias, hq, hk):
    b = Batch(2, MIXED_KV, MIXED_NEW, hq=hq, hk=hk, d=d, page=32, dtype=torch.float16)
    slopes = torch.linspace(0.01, 0.7, hq, device=DEV) if bias else None
    kw = dict(softcap=cap, slopes=slopes, scale=0.6)
    b.check(b.run(**kw), b.reference(**kw))


@pytest.mark.parametrize("d,hq,hk", [(128, 2, 2), (64, 12, 2)])
def test_key_intervals_with_empty_rows(d, hq, hk):
    b = Batch(3, MIXED_KV, MIXED_NEW, hq=hq, hk=hk, d=d, page=16)
    rng = np.random.default_rng(5)
    n = b.tok[-1]
    lo = rng.integers(-50, 400, n).astype(np.int32)
    hi = (lo + rng.integers(-60, 500, n)).astype(np.int32)
    lo[:3], hi[:3] = 0, 1000
    kw = dict(key_lo=torch.from_numpy(lo).to(DEV), key_hi=torch.from_numpy(hi).to(DEV))
    got = b.run(**kw)
    ref = b.reference(**kw)
    b.check(got, ref)
    empty = ref[1].sum((1, 2)) == 0
    assert empty.any() and bool((got[empty] == 0).all())
    lo_only = dict(key_lo=torch.from_numpy(np.maximum(0, lo)).to(DEV))
    b.check(b.run(**lo_only), b.reference(**lo_only))


def test_prefix_that_sees_itself_and_documents():
    new = [400, 260]
    b = Batch(4, new, new, hq=8, hk=2, page=64, dtype=torch.float16)
    lo, hi = [], []
    for n in new:
        for i in range(n):
            start = 0 if i < 150 else 150 if i < 151 else 151       # documents of 150, 1 and the rest
            lo.append(start)
            hi.append(max(i + 1, 100 if i < 100 else 0))             # the first 100 tokens see one another
    kw = dict(key_lo=_ints(lo), key_hi=_ints(hi))
    b.check(b.run(**kw), b.reference(**kw))


@pytest.mark.parametrize("kv", [[1], [2, 0, 1], [63, 64, 65, 127, 128, 129, 255, 256, 257, 1000], [5000]])
@pytest.mark.parametrize("hq,hk,d", [(1, 1, 128), (8, 2, 64), (16, 1, 128), (32, 1, 128)])
def test_single_tokens(kv, hq, hk, d):
    b = Batch(6, kv, hq=hq, hk=hk, d=d, page=32)
    got = b.run()
    b.check(got, b.reference())
    for r, n in enumerate(kv):
        if n == 0:
            assert bool((got[r] == 0).all())
        if n == 1:      # weight 1: the value itself
            assert torch.equal(got[r].cpu(), b.rows[r][1][0].repeat_interleave(hq // hk, 0))


GROUPS, PREFIX = [0, 1, 4, 4, 24, 64, 70], [100, 300, 50, 37, 1024, 0]


@pytest.mark.parametrize("hq,hk,d,dtype", [(2, 2, 128, torch.bfloat16), (8, 1, 128, torch.float16), (6, 2, 64, torch.bfloat16),
                                           (20, 1, 64, torch.float16)])
def test_groups_share_their_prefix(hq, hk, d, dtype):
    rng = np.random.default_rng(8)
    kv = []
    for a, b, p in zip(GROUPS, GROUPS[1:], PREFIX):
        kv += [p + int(x) for x in rng.integers(0, 200, b - a)]      # (0: a request whose whole cache is the prefix)
    kv += [33, 0, 5]                                                  # requests of no group
    b = Batch(7, kv, hq=hq, hk=hk, d=d, page=16, dtype=dtype, groups=GROUPS, prefix=PREFIX)
    ref = b.reference()
    got = b.run(GROUPS, PREFIX)
    b.check(got, ref)
    b.check(b.run(), ref)
    # a window that cuts into the prefix, capped scores and a bias, grouped
    lo = torch.from_numpy(np.maximum(0, np.asarray(kv) - rng.integers(0, 400, len(kv))).astype(np.int32)).to(DEV)
    kw = dict(key_lo=lo, softcap=10.0, slopes=torch.linspace(0.02, 0.3, hq, device=DEV))
    b.check(b.run(GROUPS, PREFIX, **kw), b.reference(**kw))


def test_group_with_several_tokens_a_request_is_read_as_requests():
    new = [3, 1, 40]
    b = Batch(9, [100, 90, 140], new, page=16, groups=[0, 3], prefix=[64])
    b.check(b.run([0, 3], [64]), b.reference())


def test_prefix_longer_than_the_caches():
    b = Batch(10, [40] * 20, hq=4, hk=4, page=16, groups=[0, 20], prefix=[40])
    b.check(b.run([0, 20], [1000]), b.reference())


@pytest.mark.parametrize("new", [None, [128], [40]])
def test_long_cache_is_split_and_repeats_bit_for_bit(new):
    b = Batch(11, [9001], new, hq=8, hk=1, page=64)
    first = b.run()
    b.check(first, b.reference())
    for _ in range(5):
        assert torch.equal(b.run(), first)


def test_large_and_negative_scales():
    b = Batch(12, MIXED_KV, MIXED_NEW, hq=4, hk=2)
    for scale in (3.0, -0.3, 0.0):
        got, (want, mean) = b.run(scale=scale), b.reference(scale=scale)
        # scores of several hundred: an exponent is off by their fp32 rounding, 2^-24 * 400
        tol = (2 * ROUND[b.dtype] + 3e-4) * mean + 1e-4
        assert bool(((got.double() - want).abs() <= tol).all())


def test_strides():
    new = [30, 1, 200]
    b = Batch(13, [64, 50, 300], new, hq=4, hk=2, q_pad=3, joint_cache=True)
    assert not b.q.is_contiguous() and not b.K.is_contiguous()
    b.check(b.run(), b.reference())


def test_slots_beyond_32_bits():
    page, hk, d = 128, 8, 128
    pages = (1 << 31) // (page * hk * d) + 40       # the last pages lie beyond 2^31 elements
    K = torch.empty((pages, hk, page, d), dtype=torch.bfloat16, device=DEV)
    V = torch.empty_like(K)
    b = Batch(14, [300, 200], [20, 1], hq=8, hk=hk, d=d, page=page)
    off = pages - b.K.shape[0]
    K[off:], V[off:] = b.K, b.V
    ref = b.reference()
    b.K, b.V, b.table = K, V, b.table + off
    b.check(b.run(), ref)
    # and the cache write
    q = torch.randn(2, 8, d, device=DEV)
    slots = _ints([(pages - 1) * page + 5, 3])
    P.rope_cache(q, q, q, _ints([0, 0]), slots, None, K, V)
    torch.cuda.synchronize()
    assert torch.equal(K[pages - 1, :, 5], q[0].bfloat16()) and torch.equal(V[0, :, 3], q[1].bfloat16())


def test_another_stream_a_graph_and_a_reused_workspace():
    b = Batch(15, MIXED_KV, MIXED_NEW, hq=4, hk=2)
    ref = b.reference()
    ws = P.attn_paged_workspace(b.q, b.K, len(b.kv))
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b.check(b.run(workspace=ws), ref)
        out = torch.zeros_like(b.q, memory_format=torch.contiguous_format)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            P.attn_paged(b.q, b.K, b.V, b.table, b.kv_len, b.scale, tok_start=b.tok_start, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        b.check(out, ref)


def test_no_tokens_and_tokens_of_no_request():
    b = Batch(16, [40, 30], [5, 2])
    out, _ = P.attn_paged(b.q[:0], b.K, b.V, b.table, b.kv_len, 1.0, tok_start=_ints([0, 0, 0]))
    assert out.shape[0] == 0
    b.tok_start = _ints([1, 4, 6])       # token 0 and token 6 belong to nobody
    got = b.run()
    assert bool((got[0] == 0).all()) and bool((got[6] == 0).all()) and bool((got[1:6] != 0).any())


def test_a_page_that_is_none_is_reported():
    for new in (None, [30, 30]):
        b = Batch(17, [40, 50], new)
        b.table[1, 1] = 1 << 20
        out, ws = P.attn_paged(b.q, b.K, b.V, b.table, b.kv_len, b.scale, tok_start=b.tok_start)
        torch.cuda.synchronize()
        assert P.plora_attn_status(ws.data_ptr()) == (0, P.ERR_INVALID_ARG)
        assert P.plora_attn_status(ws.data_ptr()) == (0, 0)


@pytest.mark.parametrize("n_req,new", [(40, None), (1, [300])])
def test_a_wait_that_runs_out_is_reported_and_the_workspace_stays_usable(n_req, new):
    # (single tokens: enough items that every CTA comes back to a stage it has used)
    b = Batch(18, [2000] * n_req, new, hq=16, hk=8)
    ref = b.reference()
    ws = P.attn_paged_workspace(b.q, b.K, n_req)
    assert P.plora_attn_set_debug(ws.data_ptr(), 1 << 20, P.HOOK_WITHHOLD_RELEASE) == 0
    P.attn_paged(b.q, b.K, b.V, b.table, b.kv_len, b.scale, tok_start=b.tok_start, workspace=ws)
    torch.cuda.synchronize()
    assert P.plora_attn_status(ws.data_ptr()) == (0, P.ERR_TIMEOUT)
    assert P.plora_attn_set_debug(ws.data_ptr(), 0, P.HOOK_NONE) == 0
    b.check(b.run(workspace=ws), ref)


# ---- the plan -----------------------------------------------------------------------------------------------
def _plan_by_hand(old, new, page, free, table, max_tokens, cursor=0):
    table, taken = table.copy(), 0
    start, pos, req, slots = [0], [], [], []
    for r, (o, n) in enumerate(zip(old, new)):
        o, n = max(0, int(o)), max(0, int(n))
        for b in range(-(-o // page), -(-(o + n) // page)):
            f = cursor + taken
            if b < table.shape[1]:
                table[r, b] = free[f] if 0 <= f < len(free) else -1
            taken += 1
        for p in range(o, o + n):
            b = p // page
            e = int(table[r, b]) if b < table.shape[1] else -1
            pos.append(p)
            req.append(r)
            slots.append(e * page + p % page if e >= 0 else -1)
        start.append(start[-1] + n)
    pad = lambda x: np.asarray((x + [-1] * max_tokens)[:max_tokens], np.int32)
    return dict(block_table=table, tok_start=start, positions=pad(pos), tok_req=pad(req), slots=pad(slots),
                kv_len=[max(0, int(o)) + max(0, int(n)) for o, n in zip(old, new)], cursor=[cursor + taken])


@pytest.mark.parametrize("n_req,page,hi_old,hi_new", [(1, 16, 1, 1), (1, 1, 5, 40), (7, 16, 100, 1), (300, 32, 500, 60),
                                                      (2500, 8, 40, 6), (1024, 128, 1000, 3), (3, 16, 100, 5000)])
@pytest.mark.parametrize("short", [0, 5])
def test_plan_against_the_loop(n_req, page, hi_old, hi_new, short):
    """short: pages that the free list lacks, and tokens that max_tokens does not cover."""
    rng = np.random.default_rng(n_req + page)
    old = rng.integers(0, hi_old + 1, n_req).astype(np.int32)
    new = rng.integers(0, hi_new + 1, n_req).astype(np.int32)
    width = max(1, int(max(-(-(o + n) // page) for o, n in zip(old, new))) + (1 if not short else -1))
    table = rng.integers(0, 9999, (n_req, width)).astype(np.int32)
    taken = sum(-(-(int(o) + int(n)) // page) - -(-int(o) // page) for o, n in zip(old, new))
    cursor = int(rng.integers(0, 4))
    free = rng.permutation(20000 + taken)[:max(1, cursor + taken - short)].astype(np.int32)
    max_tokens = max(0, int(new.sum()) + (3 if not short else -short))
    want = _plan_by_hand(old, new, page, free, table, max_tokens, cursor)
    t = torch.from_numpy(table).to(DEV)
    got = P.kv_plan(torch.from_numpy(old).to(DEV), torch.from_numpy(new).to(DEV), page, torch.from_numpy(free).to(DEV), t, max_tokens,
                    cursor=_ints([cursor]))
    again = P.kv_plan(torch.from_numpy(old).to(DEV), torch.from_numpy(new).to(DEV), page, torch.from_numpy(free).to(DEV), t, max_tokens,
                      cursor=_ints([cursor]), out=P.KvPlan(*[torch.empty_like(x) for x in got]))
    assert np.array_equal(t.cpu().numpy(), want["block_table"])
    for res in (got, again):
        for name in P.KvPlan._fields:
            assert np.array_equal(getattr(res, name).cpu().numpy(), np.asarray(want[name], np.int32)), name


def test_plan_steps_follow_one_another_without_the_host():
    """Three steps on one free list: each step's cursor and lengths are the next one's."""
    page, n = 16, 5
    free = torch.randperm(60).to(torch.int32).to(DEV)
    table = torch.full((n, 20), -1, dtype=torch.int32, device=DEV)
    kv, cursor, seen = _ints([0] * n), None, []
    for step, add in enumerate(([20, 1, 33, 0, 16], [1, 1, 1, 40, 1], [1] * n)):
        p = P.kv_plan(kv, _ints(add), page, free, table, 100, cursor=cursor)
        slots = p.slots.cpu().numpy()
        seen += [int(s) for s in slots[slots >= 0]]
        kv, cursor = p.kv_len, p.cursor
    assert len(seen) == len(set(seen)) == int(kv.sum())


def test_plan_refusals():
    one, table = _ints([1]), torch.zeros((1, 2), dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError):
        P.kv_plan(one.long(), one, 16, one, table, 4)
    with pytest.raises(P.PloraError) as e:
        P.kv_plan(one, one, 12, one, table, 4)
    assert e.value.status == P.ERR_UNSUPPORTED
    p = P.kv_plan(one, one, 16, one, table, 4)
    with pytest.raises(P.PloraError) as e:
        P.kv_plan(one, one, 16, one, table, 4, out=p._replace(kv_len=one))
    assert e.value.status == P.ERR_INVALID_ARG
    with pytest.raises(P.PloraError):
        P.kv_plan(one, one, 16, one, table, 4, cursor=p.cursor, out=p)


# ---- rotary positions -------------------------------------------------------------------------------------------
def _freqs(rot, base, scaling, factor, orig, low, high):
    i = np.arange(rot // 2, dtype=np.float64)
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2 * i / rot)
    if scaling == "linear":
        return f / factor
    if scaling == "bands":
        turns = orig * f / (2 * np.pi)
        s = np.clip((turns - low) / (high - low), 0, 1)
        return (1 - s) * f / factor + s * f
    if scaling == "ramp":
        dim = lambda n: rot * np.log(orig / (n * 2 * np.pi)) / (2 * np.log(base))
        a, b = max(np.floor(dim(high)), 0), min(np.ceil(dim(low)), rot - 1)
        s = np.clip((i - a) / max(b - a, 0.001), 0, 1)
        return f / factor * s + f * (1 - s)
    return f


@pytest.mark.parametrize("rot", [64, 128, 20, 2])
@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "bands", "ramp"])
def test_rope_table(rot, scaling):
    if scaling == "ntk" and rot == 2:
        return
    kw = dict(base=10000.0, factor=4.0 if scaling != "none" else 1.0, orig_len=2048.0, low=1.0, high=4.0 if scaling == "bands" else 32.0)
    table = P.rope_table(rot, 5000, scaling=scaling, magnitude=1.25, **kw).cpu().numpy()
    f = _freqs(rot, kw["base"], scaling, kw["factor"], kw["orig_len"], kw["low"], kw["high"])
    ang = np.arange(5000, dtype=np.float64)[:, None] * f
    want = 1.25 * np.stack([np.cos(ang), np.sin(ang)], -1)
    # one fp32 rounding, and the frequency's 64-bit rounding times the position
    assert np.max(np.abs(table - want)) <= 1.25 * 2.0 ** -24 + 1e-10


def _rotate(x, cos, sin, rot, inter):
    y = x.double().clone()
    a = (slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))
    u, w = x[..., a[0]].double(), x[..., a[1]].double()
    y[..., a[0]] = u * cos - w * sin
    y[..., a[1]] = w * cos + u * sin
    return y


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (64, 40), (80, 20), (64, 2), (96, 0), (130, 26)])
@pytest.mark.parametrize("src,dst", [(torch.float32, torch.bfloat16), (torch.float32, torch.float16), (torch.bfloat16, torch.bfloat16),
                                     (torch.float16, torch.float16)])
def test_rope_cache(d, rot, inter, src, dst):
    n, hq, hk, page, pages, max_pos = 37, 5, 2, 16, 6, 300
    g = torch.Generator().manual_seed(d + rot)
    row = torch.randn((n, hq + 2 * hk, d), generator=g).to(src).to(DEV)
    q, k, v = row[:, :hq], row[:, hq:hq + hk], row[:, hq + hk:]
    pos = torch.randint(0, max_pos, (n,), generator=g).to(torch.int32)
    slots = torch.randperm(page * pages, generator=g)[:n].to(torch.int32)
    pos[3], slots[3] = -1, 2              # padding: a zero query row, nothing written
    slots[5] = -1                          # nothing written, the query still turns
    table = P.rope_table(rot, max_pos) if rot else None
    kc = torch.full((pages, hk, page, d), 9.0, dtype=dst, device=DEV)
    vc = torch.full_like(kc, 7.0)
    status = _ints([0])
    got = P.rope_cache(q, k, v, pos.to(DEV), slots.to(DEV), table, kc, vc, interleaved=inter, status=status)
    p = pos.clamp(min=0).long().to(DEV)
    cos, sin = (table[p][..., 0].double()[:, None], table[p][..., 1].double()[:, None]) if rot else (0.0, 0.0)
    want_q, want_k = (_rotate(x, cos, sin, rot, inter) if rot else x.double() for x in (q, k))
    want_q[3] = 0
    wk, wv = torch.full(kc.shape, 9.0, dtype=torch.float64, device=DEV), torch.full(kc.shape, 7.0, dtype=torch.float64, device=DEV)
    for t in range(n):
        if t not in (3, 5):
            wk[slots[t] // page, :, slots[t] % page] = want_k[t]
            wv[slots[t] // page, :, slots[t] % page] = v[t].double()
    # a rotated value: two fp32 products of values up to |x|, then one rounding to the type
    for got_x, want_x in ((got, want_q), (kc, wk), (vc, wv)):
        tol = ROUND[dst] * want_x.abs() + 4e-6
        assert bool(((got_x.double() - want_x).abs() <= tol).all())
    assert int(status) == 0


def test_rope_in_place_unaligned_and_out_of_range():
    n, h, d = 9, 3, 64
    table = P.rope_table(d, 50)
    base = torch.randn(n * h * d + 1, device=DEV).bfloat16()
    q = base[1:].view(n, h, d)                       # two-byte alignment only
    kc, vc = torch.zeros((2, h, 16, d), dtype=torch.bfloat16, device=DEV), torch.zeros((2, h, 16, d), dtype=torch.bfloat16, device=DEV)
    pos = _ints(range(n))
    want = P.rope_cache(q.clone(), q.clone(), q.clone(), pos, pos, table, kc, vc)
    k2, v2 = torch.zeros_like(kc), torch.zeros_like(vc)
    keep = q.clone()
    got = P.rope_cache(q, keep, keep, pos, pos, table, k2, v2, q_out=q)
    assert got.data_ptr() == q.data_ptr() and torch.equal(q, want) and torch.equal(kc, k2) and torch.equal(vc, v2)
    status = _ints([0])
    pos[4] = 50
    slots = _ints(range(n))
    slots[6] = 32
    before = k2.clone()
    out = P.rope_cache(keep, keep, keep, pos, slots, table, k2, v2, status=status)
    assert int(status) == P.ERR_INVALID_ARG and bool((out[4] == 0).all()) and torch.equal(k2[0, :, 4], before[0, :, 4])


def test_rope_refusals():
    q = torch.zeros((2, 2, 64), device=DEV)
    kc = torch.zeros((1, 2, 16, 64), dtype=torch.bfloat16, device=DEV)
    pos, table = _ints([0, 1]), P.rope_table(64, 8)
    with pytest.raises(ValueError):
        P.rope_cache(q.half(), q.half(), q.half(), pos, pos, table, kc, kc.clone())
    with pytest.raises(ValueError):
        P.rope_cache(q, q, q[:, :1], pos, pos, table, kc, kc.clone())
    with pytest.raises(P.PloraError) as e:
        P.rope_cache(q, q, q, pos, pos, P.rope_table(128, 8), kc, kc.clone())
    assert e.value.status == P.ERR_UNSUPPORTED
    for kw in (dict(rot_dim=3, max_pos=4), dict(rot_dim=1024, max_pos=4), dict(rot_dim=64, max_pos=4, base=1.0),
               dict(rot_dim=64, max_pos=4, scaling="linear", factor=0.5), dict(rot_dim=64, max_pos=4, scaling="bands", factor=2.0),
               dict(rot_dim=64, max_pos=0)):
        with pytest.raises(P.PloraError):
            P.rope_table(**kw)
    with pytest.raises(ValueError):
        P.rope_table(64, 4, scaling="other")


def test_attention_refusals():
    b = Batch(19, [40, 30], [5, 2])
    ok = lambda **kw: P.attn_paged(kw.get("q", b.q), kw.get("K", b.K), b.V, kw.get("table", b.table), b.kv_len, kw.get("scale", 0.1),
                                   **{k: v for k, v in kw.items() if k not in ("q", "K", "table", "scale")})
    ok(tok_start=b.tok_start)
    for kw in (dict(K=b.K.half()), dict(table=b.table.long()), dict(tok_start=_ints([0, 5])), dict(key_lo=_ints([0])),
               dict(group_start=_ints([0, 2])), dict(slopes=torch.zeros(3, device=DEV)), dict(q=b.q.float()),
               dict(q=b.q[:, :3]), dict(out=torch.empty_like(b.q).half())):
        with pytest.raises(ValueError):
            ok(**{"tok_start": b.tok_start, **kw})
    for kw, status in ((dict(tok_start=None), P.ERR_INVALID_ARG), (dict(softcap=-1.0), P.ERR_INVALID_ARG),
                       (dict(softcap=NAN), P.ERR_INVALID_ARG), (dict(scale=NAN), P.ERR_INVALID_ARG),
                       (dict(workspace=torch.zeros(512, dtype=torch.uint8, device=DEV)), P.ERR_WORKSPACE),
                       (dict(group_start=_ints([0, 1, 1, 2]), prefix_len=_ints([1, 1, 1])), P.ERR_INVALID_ARG)):
        with pytest.raises(P.PloraError) as e:
            ok(**{"tok_start": b.tok_start, **kw})
        assert e.value.status == status, kw
    small = torch.zeros((4, 2, 8, 128), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(P.PloraError) as e:
        P.attn_paged(b.q, small, small.clone(), b.table, b.kv_len, 0.1, tok_start=b.tok_start)
    assert e.value.status == P.ERR_UNSUPPORTED
    torch.cuda.synchronize()


def test_the_example_serves_requests_of_several_adapters():
    """examples/serve_layer.py: plan, deltas, rotary positions, cache, prompt and grouped single-token attention together."""
    import importlib.util
    from pathlib import Path
    path = Path(__file__).resolve().parent.parent / "examples" / "serve_layer.py"
    spec = importlib.util.spec_from_file_location("serve_layer", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    # bf16 base products, q, K, V, weights and output, each rounded at 2^-8, behind one another, against 64 bits throughout
    assert mod.main(steps=5) <= 6 * 2.0 ** -8
