"""The paged cache's calls at their edges: plans of any size, ranges and numbers at their limits, accuracy, streams, empty steps."""
import pytest
import torch

import paper_2608_05483_b200 as P
from test_gpu_paged import DEV, ROUND, Batch, _ints

pytestmark = pytest.mark.gpu


def _status(ws):
    rc, status = P.plora_attn_status(ws.data_ptr())
    assert rc == 0
    return status


def test_caches_longer_than_the_longest_split():
    """Blocks of a prompt behind nine million keys are cut into three pieces each, more of them than items aimed at."""
    n, hq, d, page, kv, window = 3000, 64, 64, 128, 9_000_000, 200
    g = torch.Generator(device=DEV).manual_seed(0)
    pages = -(-kv // page)
    cache = torch.randn((2, pages, 1, page, d), generator=g, device=DEV, dtype=torch.bfloat16)
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    q = torch.randn((n, hq, d), generator=g, device=DEV, dtype=torch.bfloat16)
    pos = torch.arange(kv - n, kv, device=DEV)
    lo = (pos + 1 - window).to(torch.int32)
    lo[::7] = 0                                       # (some see the other pieces too, if only by weights that vanish)
    ws = P.attn_paged_workspace(q, cache[0], 1)
    slopes = torch.full((hq,), 1.0, device=DEV)
    got, _ = P.attn_paged(q, cache[0], cache[1], table, _ints([kv]), d ** -0.5, tok_start=_ints([0, n]), key_lo=lo, slopes=slopes,
                          workspace=ws)
    torch.cuda.synchronize()
    assert _status(ws) == 0
    K, V = (c.view(-1, d)[kv - n - window:kv].double() for c in cache)
    key = torch.arange(kv - n - window, kv, device=DEV)
    for a in range(0, n, 500):
        s = torch.einsum("thd,kd->thk", q[a:a + 500].double(), K) * d ** -0.5 - (pos[a:a + 500, None, None] - key).abs()
        see = (key >= (pos[a:a + 500, None, None] + 1 - window)) & (key <= pos[a:a + 500, None, None])
        w = torch.softmax(s.masked_fill(~see, float("-inf")), -1)
        want, mean = w @ V, w @ V.abs()
        # (distances of up to 2^24 are rounded to 1 at most, where their weights are nothing)
        assert bool(((got[a:a + 500].double() - want).abs() <= (2 * 2.0 ** -8 + 1e-4) * mean + 1e-5).all())


@pytest.mark.parametrize("what", ["tokens", "groups"])
def test_ranges_that_do_not_ascend_are_refused(what):
    """Ranges that jump back may want any number of units.  The call says so, and runs nothing that an earlier, larger batch left
    in the workspace."""
    big = Batch(30, [900] * 4, [900] * 4, hq=8, hk=1, d=64)          # leaves units of up to 3600 tokens behind
    n, n_req = (600, 400) if what == "tokens" else (40, 40)
    ws = P.attn_paged_workspace(big.q, big.K, 400)
    big.check(big.run(workspace=ws), big.reference())
    b = Batch(31, [600] + [1] * (n_req - 1), [n] + [0] * (n_req - 1), hq=8, hk=1, d=64)
    guard = torch.full((n + 8, 8, 64), 77.0, dtype=b.dtype, device=DEV)
    table, kv = b.table[:1].expand(n_req, -1).contiguous(), _ints([600] * n_req)
    if what == "tokens":
        kw = dict(tok_start=_ints([0 if r % 2 == 0 else n for r in range(n_req + 1)]))
    else:
        kw = dict(group_start=_ints([0, 30, 10, 40]), prefix_len=_ints([100, 100, 100]))
    P.attn_paged(b.q, b.K, b.V, table, kv, b.scale, out=guard[4:4 + n], workspace=ws, **kw)
    torch.cuda.synchronize()
    assert _status(ws) == P.ERR_INVALID_ARG
    assert bool((guard[:4] == 77).all()) and bool((guard[-4:] == 77).all())
    b.check(b.run(workspace=ws), b.reference())                          # and the workspace stays usable
    # equal entries are none of this: requests without tokens, groups without requests
    c = Batch(32, [40, 7, 90, 9], [20, 0, 0, 9], hq=8, hk=1, d=64)
    c.check(c.run(workspace=ws, groups=[0, 0, 2, 2, 4], prefix=[5, 0, 9, 3]), c.reference())


@pytest.mark.parametrize("d", [64, 128])
def test_prompts_whose_waits_run_out_leave_nothing_behind(d):
    """Every CTA stops with copies under way; it waits for them before its shared memory goes to the next one, call after call."""
    b = Batch(33, [4000, 3000], [700, 600], hq=8, hk=8, d=d, page=16)       # (items of more tiles than the ring has stages)
    ref = b.reference()
    ws = P.attn_paged_workspace(b.q, b.K, 2)
    for _ in range(3):
        assert P.plora_attn_set_debug(ws.data_ptr(), 1 << 20, P.HOOK_WITHHOLD_RELEASE) == 0
        P.attn_paged(b.q, b.K, b.V, b.table, b.kv_len, b.scale, tok_start=b.tok_start, workspace=ws)
        torch.cuda.synchronize()
        assert _status(ws) == P.ERR_TIMEOUT
        assert P.plora_attn_set_debug(ws.data_ptr(), 0, P.HOOK_NONE) == 0
        b.check(b.run(workspace=ws), ref)


@pytest.mark.parametrize("new", [[300, 40, 3], None])
def test_intervals_at_the_limits_of_their_type(new):
    """Ends of key intervals may be any int32: the lowest for "nothing", the highest for "no limit"."""
    b = Batch(34, [900, 700, 300], new, hq=4, hk=2, page=32)
    n = b.tok[-1]
    low, high = -2 ** 31, 2 ** 31 - 1
    ends = [low, high, low + 1, 200, -1, 0, 1]
    starts = [low, low, 0, low, high, high, 0, -1]
    kw = dict(key_lo=_ints(starts[i % len(starts)] for i in range(n)), key_hi=_ints(ends[i % len(ends)] for i in range(n)))
    got, ref = b.run(**kw), b.reference(**kw)
    b.check(got, ref)
    empty = ref[1].sum((1, 2)) == 0
    assert empty.any() and bool((got[empty] == 0).all())


@pytest.mark.parametrize("n_req,hq,hk", [(3, 4, 2), (2, 8, 1), (40, 4, 2)])
def test_a_window_behind_released_pages_of_the_prefix(n_req, hq, hk):
    """Sliding windows: pages that no token of a group sees any more may be gone from its table, grouped or not."""
    prefix, window = 700, 150
    own = [(7 * i) % 90 for i in range(n_req)]
    b = Batch(35, [prefix + x for x in own], hq=hq, hk=hk, page=16, groups=[0, n_req], prefix=[prefix])
    lo = [prefix + x - window for x in own]
    b.table[:, :min(lo) // 16] = -1
    kw = dict(key_lo=_ints(lo))
    ref = b.reference(**kw)
    b.check(b.run(**kw), ref)
    b.check(b.run([0, n_req], [prefix], **kw), ref)
    # a window that leaves nothing of the prefix, with all of its pages gone
    b.table[:, :prefix // 16] = -1
    kw = dict(key_lo=_ints([prefix] * n_req))
    ref = b.reference(**kw)
    b.check(b.run([0, n_req], [prefix], **kw), ref)


@pytest.mark.parametrize("new", [[300, 1, 40, 3], None])
@pytest.mark.parametrize("cap", [1e-30, 0.01, 2.0, 1e4, 1e6, 1e12, 3e38])
def test_caps_of_any_size(cap, new):
    """A cap far above the scores changes nothing, one far below them makes all weights of a row alike; and a row of large scores
    takes no accuracy from its neighbours."""
    b = Batch(36, [500, 700, 400, 90], new, hq=4, hk=2, dtype=torch.float16)
    n = b.tok[-1]
    huge = 2 if new is None else 25
    b.q = b.q.clone()
    b.q[huge] *= 3000.0
    got, (want, mean) = b.run(softcap=cap), b.reference(softcap=cap)
    assert torch.isfinite(got).all()
    keep = torch.arange(n, device=DEV) != huge        # (scores of 10^4: half an fp32 unit of them is 5e-4 in the exponent)
    tol = (2 * 2.0 ** -11 + 1e-5) * mean + 701 * 2.0 ** -25 * 5.0 + 1e-6
    assert bool(((got.double() - want).abs() <= tol)[keep].all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hk,new,groups", [(1, 1, None, False), (8, 1, None, False), (8, 2, None, True), (16, 1, None, False),
                                              (12, 1, None, False), (4, 2, [2, 1, 2, 1], False), (10, 2, [3, 1, 3, 2], False)])
def test_units_of_few_rows_keep_their_weights(hq, hk, new, groups, dtype):
    """Up to 16 rows: an output is off by its own rounding (the type's unit roundoff) and next to nothing else.  The weights keep
    16 bits or more, the scores of up to 10 and the exponentials are off by some 2^-20, fp32 sums by less."""
    group = dict(groups=[0, 2, 4], prefix=[1500, 300]) if groups else {}
    b = Batch(37, [3000, 1700, 400, 4097], new, hq=hq, hk=hk, d=128, page=64, dtype=dtype, **group)
    got, (want, mean) = b.run(*group.values()), b.reference()
    tol = 1.02 * ROUND[dtype] * want.abs() + 2.0 ** -16 * mean + 2.0 ** -25      # (half a unit below the normal range: 2^-25)
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


def test_what_a_call_allocates_belongs_to_its_stream(monkeypatch):
    """With `stream` given, the workspace is zeroed and the outputs are made on that stream, whatever the current one is doing."""
    made = []
    for name in ("zeros", "empty"):
        make = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, _make=make, **k: (made.append(torch.cuda.current_stream()), _make(*a, **k))[1])
    b = Batch(38, [900, 50], [30, 1], hq=4, hk=2)
    one = Batch(39, [900, 50], hq=4, hk=2)
    refs = b.reference(), one.reference()
    table, lens, free, blocks = P.rope_table(128, 8), _ints([3, 0]), _ints(range(9)), torch.zeros((2, 4), dtype=torch.int32, device=DEV)
    y, pos = torch.randn(3, 4, 128, device=DEV), _ints([0, 1, 2])
    kc = torch.zeros((1, 4, 16, 128), dtype=torch.bfloat16, device=DEV)
    vc = torch.zeros_like(kc)
    qd, kd = torch.randn(2, 4, 128, device=DEV).bfloat16(), torch.randn(2, 4, 64, 128, device=DEV).bfloat16()
    len_d = _ints([64, 10])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    made.clear()
    torch.cuda._sleep(200_000_000)                   # (the current stream is busy for a tenth of a second)
    outs = [P.attn_paged(x.q, x.K, x.V, x.table, x.kv_len, x.scale, tok_start=x.tok_start, stream=s) for x in (b, one)]
    P.rope_table(128, 8, stream=s)
    P.kv_plan(lens, lens, 16, free, blocks, 8, stream=s)
    P.rope_cache(y, y, y, pos, pos, table, kc, vc, stream=s)
    dec, _ = P.attn_decode(qd, kd, kd, len_d, 0.1, stream=s)
    assert len(made) >= 9 and all(m == s for m in made)
    s.synchronize()
    for (out, ws), x, ref in zip(outs, (b, one), refs):
        with torch.cuda.stream(s):
            x.check(out, ref)
        rc, status = P.plora_attn_status(ws.data_ptr(), s.cuda_stream)
        assert rc == 0 and status == 0
    torch.cuda.synchronize()
    assert torch.equal(dec, P.attn_decode(qd, kd, kd, len_d, 0.1)[0])


def test_each_scaling_has_its_own_default_turns():
    kw = dict(rot_dim=128, max_pos=4000, factor=8.0, orig_len=4096.0)
    for scaling, high in (("bands", 4.0), ("ramp", 32.0)):
        assert torch.equal(P.rope_table(scaling=scaling, **kw), P.rope_table(scaling=scaling, low=1.0, high=high, **kw))
    assert not torch.equal(P.rope_table(scaling="ramp", **kw), P.rope_table(scaling="ramp", low=1.0, high=4.0, **kw))


@pytest.mark.parametrize("ragged", [False, True])
def test_a_step_without_requests(ragged):
    none, table = _ints([]), torch.zeros((0, 5), dtype=torch.int32, device=DEV)
    cache = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16, device=DEV)
    q = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    p = P.kv_plan(none, none, 16, _ints([0, 1, 2]), table, 4)
    assert p.tok_start.tolist() == [0] and p.cursor.tolist() == [0] and p.positions.tolist() == [-1] * 4
    y = torch.zeros((0, 4, 64), device=DEV)
    assert P.rope_cache(y, y[:, :2], y[:, :2], none, none, None, cache, cache.clone()).shape == (0, 4, 64)
    out, _ = P.attn_paged(q, cache, cache.clone(), table, none, 1.0, tok_start=_ints([0]) if ragged else None)
    torch.cuda.synchronize()
    assert out.shape == (0, 4, 64)


def _check_norms(b, got, ref):
    """Per token and head, the error against the output's norm: at most the output's rounding, u, and that of the weights, which
    by random signs stays below u.  (Element by element the bound grows with the mean of |v|, while the output of n random
    keys shrinks as n^-1/2: sixteen keys lost or doubled among nine thousand are 4 % of the norm, and within that bound.)"""
    b.check(got, ref)
    want = ref[0]
    err, size = (got.double() - want).norm(dim=-1), want.norm(dim=-1)
    # (weights below half's normal range are off by up to 2^-25 each, of either sign)
    floor = (want.shape[-1] * max(b.kv)) ** 0.5 * 2.0 ** -25 if b.dtype is torch.float16 else 0.0
    worst = ((err - floor) / size.clamp(min=1e-30)).max()
    assert float(worst) <= 2 * ROUND[b.dtype], float(worst)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kv,new,hq,hk,d,page", [
    ([9001], None, 8, 1, 128, 64), ([9001], None, 32, 1, 64, 16), ([5000, 4999, 5008, 1], None, 2, 2, 128, 32),
    ([9001], [128], 8, 1, 128, 64), ([9001, 4097], [40, 3], 8, 8, 64, 16), ([4200, 6000], [700, 2], 4, 1, 128, 128)])
def test_no_key_of_a_long_cache_is_lost_or_read_twice(kv, new, hq, hk, d, page, dtype):
    b = Batch(40, kv, new, hq=hq, hk=hk, d=d, page=page, dtype=dtype)
    got = b.run()
    _check_norms(b, got, b.reference())
    with pytest.raises(AssertionError):      # (that the check would notice: sixteen keys fewer)
        _check_norms(b, got, b.reference(key_lo=_ints([16] * b.tok[-1])))


@pytest.mark.parametrize("n", [3, 60])
def test_no_key_of_a_long_prefix_is_lost_or_read_twice(n):
    prefix = 5003
    b = Batch(41, [prefix + 37 * r for r in range(n)], hq=4, hk=2, page=32, groups=[0, n], prefix=[prefix])
    _check_norms(b, b.run([0, n], [prefix]), b.reference())


@pytest.mark.parametrize("n", [255, 256, 257, 1024, 1100])
def test_many_single_tokens(n):
    """Up to 256 the attention kernel deals them out itself, beyond that the plan does, and from 1025 on in two rounds."""
    b = Batch(42, [(r * 29) % 41 for r in range(n)], hq=4, hk=2, d=64, page=16)
    _check_norms(b, b.run(), b.reference())


@pytest.mark.parametrize("masked", [False, True])
def test_more_ragged_requests_than_the_plan_has_threads(masked):
    n = 1500
    new = [r % 4 for r in range(n)]
    kv = [x + (r * 7) % 30 for r, x in enumerate(new)]
    for r in (3, 1023, 1024, 1300, 1499):                # long ones on both sides of the rounds' border
        new[r], kv[r] = 150, 400
    b = Batch(43, kv, new, hq=4, hk=2, d=64, page=16)
    kw = {}
    if masked:
        pos = torch.cat([torch.arange(k - x, k) for x, k in zip(new, kv)])
        kw = dict(key_lo=(pos - 20).clamp(min=0).to(torch.int32).to(DEV), key_hi=(pos + 3).to(torch.int32).to(DEV))
    _check_norms(b, b.run(**kw), b.reference(**kw))


def test_more_prompts_than_the_plan_writes_by_warps():
    n = 300
    b = Batch(44, [20 + r % 50 for r in range(n)], [17 + r % 4 for r in range(n)], hq=2, hk=1, d=64, page=16)
    _check_norms(b, b.run(), b.reference())


def test_more_groups_than_the_plan_holds():
    starts, prefix = [0], []
    for g in range(2100):
        starts.append(starts[-1] + (40 if g in (5, 1500, 2099) else 2 + g % 2))
        prefix.append(16 * (g % 3) + g % 5)
    kv = [p + (r * 13) % 23 for g, p in enumerate(prefix) for r in range(starts[g], starts[g + 1])]
    b = Batch(45, kv, hq=2, hk=1, d=64, page=16, groups=starts, prefix=prefix)
    _check_norms(b, b.run(starts, prefix), b.reference())
