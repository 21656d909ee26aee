"""GPU: the handle-free calls against plain float64 implementations: rotary
positions of several axes, block tables and slot maps, exact attention of packed
prompts and of new tokens over pages, and a run of them together with the
readout of the video memory.  Each test prints its case before any GPU step.

Tolerances.  u = 2^-24, float32's rounding; h = 2^-8, bfloat16's.  With
a = sum_k |q_k| |k_k| / sqrt(D) of a score (its largest over the row below) the
float32 products and sums leave it within 130 u a, and the scaling, the
subtraction of the running reference and the exponential within 8 u (|s| + 8):
e = 130 u a + 8 u (|s| + 8) bounds the relative error of every weight.  Sums of
n positive float32 terms are within n u.  Then, with A = sum_k w_k |v_k|,
  float32: |o - o*| <= (2 e + 2 (n + 130) u) A + u |o*|
  bfloat16: the weights are rounded for the PV product, and their sum with them:
           h (A + |o*|) more, and the rounding of o, h |o*|
  lse:     e + (n + 16) u + 8 u |lse|.
A prior (p, lse_p) joins with weights whose exponents carry the lse's error t
and 16 u (|lse| + |lse_p|): 2 (t + 16 u (...)) (|o*| + |p|) more, and t on lse.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U, HB = 2.0 ** -24, 2.0 ** -8
D = 128


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_26762_amd import protokv as pk
    pk.lib()
    yield


def PK():
    from paper_2606_26762_amd import protokv as pk
    return pk


def log(msg):
    print(msg, flush=True)


def _dt(name):
    import torch
    return torch.float32 if name == "fp32" else torch.bfloat16


def _randn(g, *shape, dtype, scale=1.0):
    import torch
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _g(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def attend64(q, k, v, seen):
    """q [m][D], k, v [n][D], seen [m][n] -> o, lse and the bounds' ingredients, all
    in float64; hidden values do not take part, whatever they are."""
    import torch
    q, k, v = q.double(), k.double(), v.double()
    if k.shape[0] == 0:
        z = q.new_zeros(q.shape)
        return z, q.new_full((q.shape[0],), -math.inf), z, q.new_zeros(q.shape[0]), q.new_zeros(q.shape[0])
    s = (q @ k.t() / math.sqrt(D)).masked_fill(~seen, -math.inf)
    a = (q.abs() @ k.abs().t() / math.sqrt(D)).masked_fill(~seen, 0.0).amax(1)
    smax = s.masked_fill(~seen, 0.0).abs().amax(1)
    lse = torch.logsumexp(s, 1)
    w = torch.where(seen, torch.exp(s - torch.where(lse.isfinite(), lse, 0.0)[:, None]), 0.0)
    # a value that is hidden from every row must not reach a product
    o, A = torch.zeros_like(q), torch.zeros_like(q)
    if bool(v.isfinite().all()):
        return w @ v, lse, w @ v.abs(), a, smax
    for r in range(q.shape[0]):
        vr = v[seen[r]]
        o[r], A[r] = w[r][seen[r]] @ vr, w[r][seen[r]] @ vr.abs()
    return o, lse, A, a, smax


def check(o, lse, ref, n, dtype, prior=None, what=""):
    """o, lse [m][...] of one (sequence, head) against attend64's."""
    import torch
    wo, wl, A, a, smax = ref
    e = 130 * U * a + 8 * U * (smax + 8)
    t = e + (n + 16) * U + 8 * U * torch.where(wl.isfinite(), wl.abs(), 0.0)
    tol = (2 * e + 2 * (n + 130) * U)[:, None] * A + U * wo.abs()
    if dtype == torch.bfloat16:
        tol = tol + HB * (A + wo.abs())
    if prior is not None:
        p, pl = prior[0].double(), prior[1].double()
        both = torch.logaddexp(wl, pl)
        x, y = torch.exp(wl - both), torch.exp(pl - both)
        x, y = torch.where(wl.isinf(), 0.0, x), torch.where(pl.isinf(), 0.0, y)
        t = t + 16 * U * (torch.where(wl.isinf(), 0.0, wl.abs()) + torch.where(pl.isinf(), 0.0, pl.abs()))
        p = torch.where(pl.isinf()[:, None], 0.0, p)
        tol = tol * x[:, None] + 2 * t[:, None] * (wo.abs() + p.abs())
        wo = x[:, None] * wo + y[:, None] * p
        wl = torch.where(wl.isinf(), pl, torch.where(pl.isinf(), wl, both))
    if dtype == torch.bfloat16:
        tol = tol + HB * wo.abs()
    tol = tol + 1e-30
    err = (o.double() - wo).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), f"{what}: o off by {float((err / tol).nan_to_num(math.inf).max()):.2f} of its bound"
    empty = wl == -math.inf
    assert torch.equal(lse.double()[empty], wl[empty]), what
    le = (lse.double() - wl).abs()[~empty]
    lt = t[~empty]
    assert bool((le <= lt).all()), f"{what}: lse off by {float((le / lt).max()):.2f} of its bound"


# -- packed prompts -------------------------------------------------------------


def _prompt(lens, hq, hk, dtype, seed, fused=True, prior=False, tail=3, odd=None):
    import torch
    pk, g = PK(), _g(seed)
    total = sum(lens) + tail
    dt = _dt(dtype)
    if fused:
        qkv = _randn(g, total, (hq + 2 * hk) * D, dtype=dt, scale=1.5)
        q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([hq * D, hk * D, hk * D], dim=1))
    else:
        q, k, v = (_randn(g, total, h, D, dtype=dt, scale=1.5) for h in (hq, hk, hk))
    if odd is not None:
        odd(q, k, v)
    cu = _i32(np.cumsum([0] + list(lens)).tolist())
    o = torch.full((total, hq, D), 7.5, dtype=dt, device="cuda")
    lse = torch.full((total, hq), 8.5, device="cuda")
    pr = None
    if prior:
        pr = (_randn(g, total, hq, D, dtype=dt), torch.randn(total, hq, generator=g, device="cuda") * 2 + 3)
        pr[1][::5] = -math.inf
        pr[0][::5] = math.nan   # an unread prior may hold anything
    pk.prompt_attend(q, k, v, cu, out=o, lse=lse, prior=pr)
    torch.cuda.synchronize()
    n = sum(lens)
    assert bool((o[n:] == 7.5).all()) and bool((lse[n:] == 8.5).all()), "rows behind the last sequence"
    at = 0
    for L in lens:
        seen = torch.ones(L, L, dtype=torch.bool, device="cuda").tril()
        for h in range(hq):
            kv = h // (hq // hk)
            sl = slice(at, at + L)
            if L:
                ref = attend64(q[sl, h], k[sl, kv], v[sl, kv], seen)
                check(o[sl, h], lse[sl, h], ref, L, dt, (pr[0][sl, h], pr[1][sl, h]) if prior else None,
                      f"sequence of {L}, head {h}")
        at += L
    return q, k, v, cu, o, lse


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,hq,hk", [
    ([1], 1, 1), ([1, 0, 2, 0], 2, 1), ([31, 33, 1, 64], 7, 1), ([63, 64, 65], 6, 2), ([255, 257, 3], 4, 4),
    ([129], 40, 1), ([500, 13], 14, 2), ([300], 3, 3), ([5] * 70, 8, 2)])
def test_prompt(lens, hq, hk, dtype):
    log(f"case: prompt {lens} heads {hq}/{hk} {dtype}")
    _prompt(lens, hq, hk, dtype, 1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prompt_with_prior_and_own_tensors(dtype):
    log(f"case: prompt with prior {dtype}")
    _prompt([40, 1, 97], 14, 2, dtype, 2, fused=False, prior=True)


def test_prompt_long():
    """Many key tiles to a row, more than one row block to a head."""
    log("case: prompt long")
    _prompt([2100, 700], 8, 2, "bf16", 3)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prompt_odd_values_stay_where_they_are_seen(dtype):
    """inf and NaN in keys and values reach the rows that see them and no others,
    though they share tiles, row blocks and matrix products with them."""
    import torch
    log(f"case: prompt odd values {dtype}")
    pk, g = PK(), _g(4)
    dt = _dt(dtype)
    L, hq, hk = 150, 6, 2
    q, k, v = (_randn(g, 2 * L, h, D, dtype=dt) for h in (hq, hk, hk))
    clean = pk.prompt_attend(q, k, v, _i32([0, L, 2 * L]))
    v2, k2 = v.clone(), k.clone()
    v2[100, 0, 5] = math.inf
    v2[131, 1, 77] = math.nan
    k2[140, 0, 3] = math.nan
    v2[L + 149, 0, :] = math.nan
    o, lse = pk.prompt_attend(q, k2, v2, _i32([0, L, 2 * L]))
    torch.cuda.synchronize()
    same = torch.ones(2 * L, hq, D, dtype=torch.bool, device="cuda")
    same[100:L, :3, 5] = False
    same[131:L, 3:, 77] = False
    same[140:L, :3] = False
    same[L + 149, :3] = False
    # the products of a tile that holds such a value are summed in another order
    tol = 2 * HB if dt == torch.bfloat16 else 1e-5
    d = (o.double() - clean[0].double()).abs()
    assert bool((d[same] <= tol * (clean[0].double().abs()[same] + 0.05)).all())
    assert bool((o[100:140, :3, 5] == math.inf).all())
    assert bool(o[131:L, 3:, 77].isnan().all()) and bool(o[140:L, :3].isnan().all())
    assert bool(o[L + 149, :3].isnan().all())
    keep = torch.ones(2 * L, hq, dtype=torch.bool, device="cuda")
    keep[140:L, :3] = False
    assert torch.equal(lse[keep], clean[1][keep])


def test_prompt_first_row_returns_its_value():
    """A row with one key returns that key's value exactly, whatever the score."""
    import torch
    log("case: prompt of single tokens")
    pk, g = PK(), _g(5)
    n, hq, hk = 50, 4, 2
    q, k, v = (_randn(g, n, h, D, dtype=torch.bfloat16, scale=3.0) for h in (hq, hk, hk))
    o, lse = pk.prompt_attend(q, k, v, _i32(list(range(n + 1))))
    assert torch.equal(o, v.repeat_interleave(2, dim=1))
    want = (q.double().unflatten(1, (hk, 2)) * k.double()[:, :, None]).sum(-1).flatten(1) / math.sqrt(D)
    assert bool(((lse.double() - want).abs() <= 1e-4).all())


@pytest.mark.parametrize("lens,hq,hk", [([1300], 28, 4), ([700, 90], 16, 2)])
def test_prompt_in_few_blocks(lens, hq, hk):
    """So few rows that two waves share a row's keys; values of the first keys that
    are infinite reach every row, one of a late key only those behind it."""
    import torch
    log(f"case: prompt in few blocks {lens}")
    q, k, v, cu, o, lse = _prompt(lens, hq, hk, "bf16", 6)
    _prompt(lens, hq, hk, "bf16", 7, prior=True)
    v2 = v.clone()
    v2[3, 0, 9] = -math.inf
    v2[600, 0, 11] = math.nan
    o2, lse2 = PK().prompt_attend(q, k, v2, cu)
    g, L = hq // hk, lens[0]
    assert torch.equal(lse2[:L], lse[:L])
    assert bool((o2[3:L, :g, 9] == -math.inf).all()) and bool(o2[600:L, :g, 11].isnan().all())
    assert bool(o2[:3, :g, 9].isfinite().all()) and bool(o2[:600, :g, 11].isfinite().all())
    o2[:, :g, 9], o2[:, :g, 11] = o[:, :g, 9], o[:, :g, 11]
    d = (o2[:L].double() - o[:L].double()).abs()
    assert bool((d <= 2 * HB * (o[:L].double().abs() + 0.05)).all())


@pytest.mark.parametrize("n", [3, 70])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_that_make_no_sense_stay_inside(dtype, n):
    """cu that falls, is negative or passes the rows: whatever comes out, nothing
    outside the results is written, and sequences that are in order are right."""
    import torch
    log(f"case: senseless cu {dtype} {n}")
    pk, g = PK(), _g(8)
    dt = _dt(dtype)
    total, hq, hk, P = 200, 4, 2, 16
    wild = [0, 60, 20, 900, -5, 2 ** 31 - 1, -2 ** 31, 130]
    cu = _i32([wild[i % 8] for i in range(n + 1)])
    q, k, v = (_randn(g, total, h, D, dtype=dt) for h in (hq, hk, hk))
    big = torch.full((total + 400, hq, D), 7.5, dtype=dt, device="cuda")
    bl = torch.full((total + 400, hq), 8.5, device="cuda")
    o, lse = big[200:200 + total], bl[200:200 + total]
    pk.prompt_attend(q, k, v, cu, out=o, lse=lse)
    pages = tuple(_randn(g, 20, hk, P, D, dtype=dt) for _ in range(2))
    table = torch.randint(-3, 25, (n, 9), generator=g, device="cuda").int()
    lens = torch.randint(-50, 400, (n,), generator=g, device="cuda").int()
    for add in (1, 200):
        pk.page_attend(q, pages, table, cu, lens, add, out=o, lse=lse)
    torch.cuda.synchronize()
    for x, s in ((big, 7.5), (bl, 8.5)):
        assert bool((x[:200] == s).all()) and bool((x[200 + total:] == s).all())


# -- pages ------------------------------------------------------------------------


def _paged(reqs, hq, hk, P, dtype, seed, prior=False, tail=2, bad=(), width=None, lens=None, max_add=None,
           workspace=None):
    """reqs: (context, new); everything that no token fills is NaN; bad: (request, page)
    entries set outside the pages.  lens: kv_len where it is not context + new."""
    import torch
    pk, g = PK(), _g(seed)
    dt = _dt(dtype)
    kv = [c + a for c, a in reqs] if lens is None else lens
    need = [(max(x, 0) + P - 1) // P for x in kv]
    width = width or max(max(need), 1)
    need = [min(x, width) for x in need]
    pages = sum(need) + 2
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(reqs), width), -7, dtype=torch.int32, device="cuda")
    kp, vp = (torch.full((pages, hk, P, D), math.nan, dtype=dt, device="cuda") for _ in range(2))
    at, ks, vs = 0, [], []
    for i, n in enumerate(need):
        own = order[at:at + n].long()
        at += n
        table[i, :n] = own.int()
        m = min(max(kv[i], 0), width * P)
        k, v = (_randn(g, hk, m, D, dtype=dt, scale=1.2) for _ in range(2))
        idx = torch.arange(m, device="cuda")
        kp[own[idx // P], :, idx % P] = k.transpose(0, 1)
        vp[own[idx // P], :, idx % P] = v.transpose(0, 1)
        ks.append(k)
        vs.append(v)
    gone = [set() for _ in reqs]
    for i, p in bad:
        table[i, p] = [-1, pages, 2 ** 31 - 1, -2 ** 31][(i + p) % 4]
        gone[i].add(p)
    add = [a for _, a in reqs]
    total = sum(add) + tail
    q = _randn(g, total, hq, D, dtype=dt, scale=2.0)
    o = torch.full((total, hq, D), 7.5, dtype=dt, device="cuda")
    lse = torch.full((total, hq), 8.5, device="cuda")
    pr = (_randn(g, total, hq, D, dtype=dt), torch.randn(total, hq, generator=g, device="cuda") + 3) if prior else None
    pk.page_attend(q, (kp, vp), table, _i32(np.cumsum([0] + add).tolist()), _i32(kv), max_add or max(max(add), 1), out=o,
                   lse=lse, prior=pr, workspace=workspace)
    torch.cuda.synchronize()
    n = sum(add)
    assert bool((o[n:] == 7.5).all()) and bool((lse[n:] == 8.5).all()), "rows behind the last request"
    at = 0
    for i, a in enumerate(add):
        m = ks[i].shape[1]
        key = torch.arange(m, device="cuda")
        last = min(max(kv[i], 0), width * P) - a + torch.arange(a, device="cuda")
        here = torch.tensor([int(x) // P not in gone[i] for x in range(m)], dtype=torch.bool, device="cuda")
        seen = (key[None] <= last[:, None]) & here[None]
        sl = slice(at, at + a)
        for h in range(hq if a else 0):
            ref = attend64(q[sl, h], ks[i][h // (hq // hk)], vs[i][h // (hq // hk)], seen)
            check(o[sl, h], lse[sl, h], ref, m, dt, (pr[0][sl, h], pr[1][sl, h]) if prior else None,
                  f"request {i} {reqs[i]}, head {h}")
        at += a
    return o, lse


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("reqs,hq,hk,P", [
    ([(0, 1)], 1, 1, 16), ([(1, 1), (0, 1), (63, 1), (64, 1), (65, 1)], 4, 2, 16), ([(700, 1)], 7, 1, 1),
    ([(2500, 1), (31, 1)], 28, 4, 16), ([(100, 5), (0, 33), (1000, 1), (5, 0), (255, 64)], 6, 2, 8),
    ([(1500, 40)], 14, 2, 64), ([(300, 300), (7, 2)], 3, 3, 128), ([(900, 3)], 40, 1, 1024), ([(50, 1)] * 70, 2, 1, 32)])
def test_pages(reqs, hq, hk, P, dtype):
    log(f"case: pages {reqs[:6]} heads {hq}/{hk} page {P} {dtype}")
    _paged(reqs, hq, hk, P, dtype, 11)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("reqs", [[(400, 1), (77, 1)], [(400, 30), (77, 9)]])
def test_pages_with_prior(reqs, dtype):
    log(f"case: pages with prior {reqs} {dtype}")
    _paged(reqs, 14, 2, 16, dtype, 12, prior=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("add", [1, 25])
def test_pages_that_are_none_hold_no_tokens(dtype, add):
    """Entries outside the pages leave their tokens out: in the first and last
    tile, across a whole tile, and of a whole request (its rows see nothing)."""
    log(f"case: bad pages {dtype} add {add}")
    bad = [(0, 0), (0, 5), (0, 6), (0, 7), (0, 8), (0, 9), (0, 10), (1, 0), (1, 1), (1, 2), (1, 3), (2, 20)]
    _paged([(300, add), (64 - add, add), (320, add)], 6, 2, 16, dtype, 13, bad=bad)
    _paged([(300, add), (64 - add, add), (320, add)], 6, 2, 16, dtype, 13, bad=bad, prior=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("prior", [False, True])
def test_rows_before_the_first_token_see_nothing(dtype, prior):
    """kv_len below the number of new rows, 0, negative, or beyond the table."""
    log(f"case: short kv_len {dtype} prior {prior}")
    _paged([(0, 10), (0, 3), (0, 40), (0, 2), (0, 1)], 6, 2, 16, dtype, 14, prior=prior, lens=[4, 0, -9, 300, 0], width=19)


def test_pages_beyond_the_table_are_not_read():
    log("case: kv_len beyond the table row")
    _paged([(0, 5), (0, 2)], 4, 2, 16, "bf16", 15, lens=[100, 33], width=4)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_beyond_max_add_are_left(dtype):
    import torch
    log(f"case: max_add {dtype}")
    pk, g = PK(), _g(16)
    dt = _dt(dtype)
    kp, vp = (_randn(g, 4, 1, 16, D, dtype=dt) for _ in range(2))
    q = _randn(g, 12, 2, D, dtype=dt)
    args = ((kp, vp), _i32([[0, 1], [2, 3]]), _i32([0, 8, 12]), _i32([20, 30]))
    full, _ = pk.page_attend(q, *args, 8)
    o = torch.full_like(full, 7.5)
    pk.page_attend(q, *args, 4, out=o)
    torch.cuda.synchronize()
    assert bool((o[4:8] == 7.5).all())
    got, want = torch.cat([o[:4], o[8:]]).double(), torch.cat([full[:4], full[8:]]).double()
    assert bool(((got - want).abs() <= 2 * HB * (want.abs() + 0.05)).all())


@pytest.mark.parametrize("reqs", [[(5000, 1)], [(2000, 1), (9000, 1), (10, 1)], [(6000, 50)], [(4000, 1), (4500, 200)]])
def test_pages_split_over_the_context(reqs):
    log(f"case: split context {reqs}")
    _paged(reqs, 7, 1, 16, "bf16", 17, prior=True)
    _paged(reqs, 4, 2, 32, "fp32", 17)


def test_pages_of_many_requests():
    """Thousands of requests, most with a token, some with none, a few with a chunk."""
    log("case: pages of many requests")
    rng = np.random.default_rng(21)
    reqs = [(int(rng.integers(0, 90)), int(rng.choice([0, 1, 1, 1, 1, 2]))) for _ in range(2500)]
    reqs[700], reqs[2400] = (300, 40), (10, 70)
    _paged(reqs, 2, 1, 8, "bf16", 21)


@pytest.mark.parametrize("P", [1, 2])
def test_pages_more_than_staged_at_a_time(P):
    """Small pages: the page ids of one context come in several parts."""
    log(f"case: {P} tokens to a page")
    _paged([(4500, 1), (4300, 70)], 2, 1, P, "bf16", 18)


def test_cache_beyond_4_gib():
    """Pages whose byte offsets pass 32 bits, unsigned too."""
    import torch
    log("case: large cache")
    pk, g = PK(), _g(19)
    P, hk = 64, 8
    pages = (5 << 30) // (hk * P * D * 2)
    kp, vp = (torch.empty(pages, hk, P, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    top = [pages - 1, pages - 2, pages // 2 + 3, 0]
    small = tuple(_randn(g, 4, hk, P, D, dtype=torch.bfloat16) for _ in range(2))
    for x, s in zip((kp, vp), small):
        x[torch.tensor(top, device="cuda")] = s
    for add in (1, 20):
        q = _randn(g, add, 16, D, dtype=torch.bfloat16)
        args = (_i32([0, add]), _i32([230]), add)
        o, lse = pk.page_attend(q, (kp, vp), _i32([top]), *args)
        o2, lse2 = pk.page_attend(q, small, _i32([[0, 1, 2, 3]]), *args)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    # and written there
    k, v = (_randn(g, 3, hk, D, dtype=torch.bfloat16) for _ in range(2))
    slots = [(pages - 1) * P + 63, (pages // 2 + 3) * P, 5]
    pk.rotate(None, k, _i32([0, 0, 0]), pk.pair_axes((64,)), 1e4, v=v, pages=(kp, vp), slots=_i32(slots))
    for t, s in enumerate(slots):
        assert torch.equal(vp[s // P, :, s % P], v[t]) and torch.equal(kp[s // P, :, s % P], k[t])


def test_prompt_rows_beyond_4_gib():
    """Row strides that carry offsets past 32 bits."""
    import torch
    log("case: far rows")
    pk, g = PK(), _g(20)
    L = 70
    far = (1 << 31) // L // 8 * 8 + (1 << 26)   # elements from row to row
    rows = {}
    for name, h in (("q", 2), ("k", 1), ("v", 1)):
        buf = torch.empty(far * (L - 1) + 2 * D, dtype=torch.bfloat16, device="cuda")
        rows[name] = buf.as_strided((L, h, D), (far, D, 1))
        rows[name].copy_(_randn(g, L, h, D, dtype=torch.bfloat16))
    near = {n: x.contiguous() for n, x in rows.items()}
    cu = _i32([0, L])
    a = pk.prompt_attend(rows["q"], rows["k"], rows["v"], cu)
    b = pk.prompt_attend(near["q"], near["k"], near["v"], cu)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# -- rotary positions -----------------------------------------------------------------


def rotate64(x, pos, axes, theta):
    import torch
    i = torch.arange(D // 2, dtype=torch.float64, device=x.device)
    w = pos.double()[torch.tensor(list(axes), device=x.device)].t() * theta ** (-2 * i / D)
    x = x.double()
    c, s = torch.cos(w)[:, None], torch.sin(w)[:, None]
    a, b = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], -1), torch.cat([a.abs() + b.abs()] * 2, -1)


def check_turned(got, x, pos, axes, theta):
    """float64 angles of up to 2^31: the power (2^-52), the product (2^-53) and the
    whole turns taken off leave them within 2^31 x 2^-51.3 on each side, 2e-6 in all;
    cos, sin, products and sum in float32: 6 u (|a| + |b|); the rounding of the result."""
    import torch
    want, size = rotate64(x, pos, axes, theta)
    tol = (6 * U + 2e-6) * size + (HB if got.dtype == torch.bfloat16 else U) * want.abs()
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol.clamp(min=1e-300)).max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,hq,hk", [(1, 28, 4), (3, 1, 1), (65, 7, 1), (700, 6, 3), (9000, 2, 1)])
@pytest.mark.parametrize("store", [False, True])
def test_rotate(n, hq, hk, dtype, store):
    import torch
    log(f"case: rotate {n} tokens, heads {hq}/{hk} {dtype} store {store}")
    pk, g = PK(), _g(31)
    dt = _dt(dtype)
    qkv = _randn(g, n, (hq + 2 * hk) * D, dtype=dt)
    q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([hq * D, hk * D, hk * D], dim=1))
    pos = torch.stack([torch.randint(0, m, (n,), generator=g, device="cuda") for m in (2 ** 31 - 1, 100, 5000)]).int()
    pos[1, 0] = -3
    axes = pk.pair_axes((16, 24, 24), interleaved=n % 2 == 1)
    theta = 1e6
    if not store:
        qo, ko = pk.rotate(q, k, pos, axes, theta)
        torch.cuda.synchronize()
        check_turned(qo, q, pos, axes, theta)
        check_turned(ko, k, pos, axes, theta)
        return
    P = 16
    pages = (n + P - 1) // P + 2
    kp, vp = (torch.full((pages, hk, P, D), 3.0, dtype=dt, device="cuda") for _ in range(2))
    slots = torch.randperm(pages * P, generator=g, device="cuda")[:n].int()
    out = torch.arange(n, device="cuda") % 7 == 3   # not stored: below and beyond the pages
    slots[out] = torch.where(torch.arange(n, device="cuda") % 2 == 0, -1 - slots, pages * P + slots)[out].int()
    ko = torch.empty(n, hk, D, dtype=dt, device="cuda")
    qo, _ = pk.rotate(q, k, pos, axes, theta, v=v, pages=(kp, vp), slots=slots, k_out=ko)
    torch.cuda.synchronize()
    check_turned(qo, q, pos, axes, theta)
    check_turned(ko, k, pos, axes, theta)
    want_k, want_v = (torch.full((pages, hk, P, D), 3.0, dtype=dt, device="cuda") for _ in range(2))
    s = slots[~out].long()
    want_k[s // P, :, s % P] = ko[~out]
    want_v[s // P, :, s % P] = v[~out]
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rotate_in_place_and_alone(dtype):
    """In place on strided rows; q or k alone; one position for every axis."""
    import torch
    log(f"case: rotate in place {dtype}")
    pk, g = PK(), _g(32)
    dt = _dt(dtype)
    n, hq, hk = 37, 6, 2
    x = _randn(g, n, (hq + hk) * D + 64, dtype=dt)
    y = x.clone()
    q, k = (t[:, a * D:b * D].unflatten(1, (-1, D)) for t, a, b in ((x, 0, hq), (x, hq, hq + hk)))
    pos = torch.randint(0, 10 ** 6, (n,), generator=g, device="cuda").int()
    axes = pk.pair_axes((20, 44))
    a, b = pk.rotate(q, None, pos, axes, 1e4)
    assert b is None
    a2, b2 = pk.rotate(None, k, pos, axes, 1e4)
    assert a2 is None
    pk.rotate(q, k, pos, axes, 1e4, q_out=q, k_out=k)
    torch.cuda.synchronize()
    assert torch.equal(q, a) and torch.equal(k, b2) and torch.equal(x[:, (hq + hk) * D:], y[:, (hq + hk) * D:])
    check_turned(a, y[:, :hq * D].unflatten(1, (-1, D)), torch.stack([pos, pos]), axes, 1e4)


def test_rotate_values_are_copied_as_they_are():
    """v's rows go to their slots bit for bit, NaN payloads and infinities too."""
    import torch
    log("case: rotate copies values")
    pk = PK()
    bits = torch.arange(1 << 16, device="cuda").to(torch.int32).to(torch.int16).view(-1, 2, D)
    v = bits.view(torch.bfloat16)
    n = v.shape[0]
    kp, vp = (torch.zeros(n // 8, 2, 8, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pk.rotate(None, v, torch.zeros(n, dtype=torch.int32, device="cuda"), pk.pair_axes((64,)), 1e4, v=v, pages=(kp, vp),
              slots=torch.arange(n, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(vp.view(torch.int16).transpose(1, 2).reshape(n, 2, D), bits)


# -- block tables ---------------------------------------------------------------------


def plan_ref(ctx, add, base, table, stack, count, P, most):
    """The definition, request by request, on lists."""
    width, pages = len(table[0]), len(stack)
    table, stack = [list(r) for r in table], list(stack)
    ctx = [min(max(c, 0), width * P) for c in ctx]
    up = lambda x: -(-x // P)  # noqa: E731
    count = min(max(count, 0), pages)
    for i, a in enumerate(add):
        if a < 0:
            for j in range(up(ctx[i])):
                if count < pages:
                    stack[count] = table[i][j]
                    count += 1
    top, asked, used, refused, row = count, 0, 0, 0, 0
    cu, kv, slots, positions = [0], [], [-1] * most, [0] * most
    for i, a in enumerate(add):
        first, row = row, row + max(a, 0)
        fits = ctx[i] + a <= width * P and row <= most
        need = up(ctx[i] + a) - up(ctx[i]) if a > 0 and fits else 0
        asked += need
        ok = a == 0 or (a > 0 and fits and (need == 0 or asked <= top))
        if ok:
            for j in range(need):
                table[i][up(ctx[i]) + j] = stack[top - 1 - (asked - need + j)]
            used += need
        refused += a > 0 and not ok
        kv.append(ctx[i] + a if ok else 0)
        cu.append(min(row, most))
        for t in range(first, min(row, most)):
            p = ctx[i] + t - first
            positions[t] = base[i] + p
            if ok and 0 <= table[i][p // P] < pages:
                slots[t] = table[i][p // P] * P + p % P
    return table, stack, top - used, cu, kv, slots, positions, refused


def _plan(ctx, add, P, pages, width, most, free, seed, base=True, held_order=None):
    import torch
    pk = PK()
    rng = np.random.default_rng(seed)
    order = rng.permutation(pages).tolist()
    table, at = [], 0
    for c in ctx:
        n = -(-min(max(c, 0), width * P) // P)
        table.append(order[at:at + n] + [-5] * (width - n))
        at += n
    assert at + free <= pages
    stack = order[at:at + free] + [-9] * (pages - free)
    bs = [int(x) for x in rng.integers(0, 10 ** 6, len(ctx))] if base else [0] * len(ctx)
    t, s = _i32(table), _i32(stack)
    count = _i32([free])
    p = pk.page_plan(_i32(ctx), _i32(add), t, s, count, P, most, base=_i32(bs) if base else None)
    torch.cuda.synchronize()
    want = plan_ref(ctx, add, bs, table, stack, free, P, most)
    got = (t.tolist(), s.tolist(), int(p.count), p.cu.tolist(), p.kv_len.tolist(), p.slots.tolist(),
           p.positions.tolist(), int(p.refused))
    for name, x, y in zip(("table", "stack", "count", "cu", "kv_len", "slots", "positions", "refused"), got, want):
        assert x == y, name
    assert int(count) == free
    return p


@pytest.mark.parametrize("case", [
    ("one", [0], [1], 16, 4, 2, 1, 4), ("full page", [16], [1], 16, 4, 3, 2, 2), ("nothing", [5, 0], [0, 0], 16, 4, 2, 3, 3),
    ("ends", [33, 5, 0, 40], [-1, 20, 7, -1], 16, 12, 4, 40, 2), ("none left", [0, 3, 16, 0, 2], [40, 2, 1, 5, 3], 16, 8, 4, 60, 3),
    ("row too short", [60, 0], [5, 4], 16, 8, 4, 9, 3), ("tokens too few", [0, 0, 0], [4, 5, 6], 8, 9, 3, 10, 9),
    ("single tokens", [3, 0, 9], [4, 2, 1], 1, 30, 12, 8, 18), ("ctx out of range", [-4, 1000], [3, 0], 8, 20, 4, 9, 6)])
def test_page_plan(case):
    name, ctx, add, P, pages, width, most, free = case
    log(f"case: page_plan {name}")
    _plan(ctx, add, P, pages, width, most, free, 1)
    _plan(ctx, add, P, pages, width, most, free, 2, base=False)


@pytest.mark.parametrize("n,P,top,most_add,short", [
    (64, 16, 900, 1, 1.0), (1023, 8, 300, 20, 0.7), (1024, 32, 600, 3, 1.0), (1025, 16, 100, 40, 0.5), (5000, 4, 60, 9, 0.9),
    (8192, 2, 20, 5, 1.0), (3, 64, 5000, 30000, 1.0)])
def test_page_plan_many(n, P, top, most_add, short):
    log(f"case: page_plan {n} requests")
    rng = np.random.default_rng(n)
    ctx = rng.integers(0, top, n)
    add = np.where(rng.random(n) < 0.2, -1, rng.integers(0, most_add + 1, n))
    width = -(-(top + most_add) // P)
    need = int((-(-(ctx + np.maximum(add, 0)) // P) + (-ctx // P)).sum())
    free = max(1, int(need * short))
    pages = int((-(-ctx // P)).sum()) + free
    rows = int(np.maximum(add, 0).sum())
    _plan([int(x) for x in ctx], [int(x) for x in add], P, pages, width, rows + 5, free, n)
    _plan([int(x) for x in ctx], [int(x) for x in add], P, pages, width, max(1, rows // 2), free, n)


def test_page_plan_sums_that_pass_32_bits_are_refused():
    """New tokens of 2^31 - 1 each: every such request is refused, the small one before is not."""
    log("case: page_plan huge requests")
    import torch
    pk = PK()
    t, s = torch.full((4, 2), -5, dtype=torch.int32, device="cuda"), _i32([3, 1, 0, 2])
    p = pk.page_plan(_i32([0, 0, 0, 0]), _i32([2, 2 ** 31 - 1, 2 ** 31 - 1, 1]), t, s, _i32([4]), 16, 6)
    torch.cuda.synchronize()
    assert p.kv_len.tolist() == [2, 0, 0, 0] and p.cu.tolist() == [0, 2, 6, 6, 6] and int(p.refused) == 3
    assert p.slots.tolist() == [32, 33, -1, -1, -1, -1] and int(p.count) == 3


# -- streams, graphs, together -----------------------------------------------------------


def test_two_streams_at_once():
    """Calls on two streams, each with its own workspace, against the same calls alone."""
    import torch
    log("case: two streams")
    pk, g = PK(), _g(41)
    made = []
    for add in (1, 60):
        kp, vp = (_randn(g, 400, 4, 16, D, dtype=torch.bfloat16) for _ in range(2))
        table = torch.randperm(400, generator=g, device="cuda").int()[:380].view(1, 380)
        q = _randn(g, add, 28, D, dtype=torch.bfloat16)
        made.append((q, (kp, vp), table, _i32([0, add]), _i32([6000]), add))
    alone = [pk.page_attend(*m) for m in made]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(5):
        both = [pk.page_attend(*m, stream=s) for m, s in zip(made, streams)]
        torch.cuda.synchronize()
        for (o, l), (o2, l2) in zip(both, alone):
            assert torch.equal(o, o2) and torch.equal(l, l2)


def _step_tensors(g, n, hq, hk, P, pages, width, most):
    import torch
    st = {"ctx": torch.zeros(n, dtype=torch.int32, device="cuda"), "add": torch.zeros(n, dtype=torch.int32, device="cuda"),
          "table": torch.full((n, width), -1, dtype=torch.int32, device="cuda"),
          "stack": torch.randperm(pages, generator=g, device="cuda").int(), "count": _i32([pages]), "next": _i32([0]),
          "kp": torch.full((pages, hk, P, D), math.nan, dtype=torch.bfloat16, device="cuda"),
          "vp": torch.full((pages, hk, P, D), math.nan, dtype=torch.bfloat16, device="cuda"),
          "qkv": torch.zeros(most, (hq + 2 * hk) * D, dtype=torch.bfloat16, device="cuda")}
    return st


def _step(st, hq, hk, P, most, max_add):
    """One step of a server: pages, positions, rotation and store, attention."""
    pk = PK()
    q, k, v = (x.unflatten(1, (-1, D)) for x in st["qkv"].split([hq * D, hk * D, hk * D], dim=1))
    p = pk.page_plan(st["ctx"], st["add"], st["table"], st["stack"], st["count"], P, most, count_out=st["next"])
    qr, _ = pk.rotate(q, k, p.positions, pk.pair_axes((64,)), 1e4, v=v, pages=(st["kp"], st["vp"]), slots=p.slots)
    o, lse = pk.page_attend(qr, (st["kp"], st["vp"]), st["table"], p.cu, p.kv_len, max_add)
    st["count"].copy_(st["next"])
    return p, o, lse


def test_dialogue_steps_captured_and_eager():
    """Dialogues of several requests step by step: questions of different lengths,
    single tokens, padded rows, an end that frees pages which others take up.  The
    same steps through a captured graph, replayed with eager work in between, give
    the same bits, and both the float64 attention over what was said so far."""
    import torch
    log("case: dialogue, eager and captured")
    n, hq, hk, P, pages, width, most, top = 5, 14, 2, 16, 40, 12, 128, 64
    g = _g(42)
    eager, graphed = (_step_tensors(_g(43), n, hq, hk, P, pages, width, most) for _ in range(2))
    steps = [[40, 7, 0, 64, 1], [1, 1, 1, 1, 1], [1, 1, 30, 0, 1], [1, 9, 1, -1, 1], [3, 1, 1, 60, 1], [1, 1, 1, 1, -1],
             [1, 1, 1, 1, 17]]
    graph = torch.cuda.CUDAGraph()
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):   # a warm-up step of no tokens
        _step(graphed, hq, hk, P, most, top)
    torch.cuda.current_stream().wait_stream(warm)
    with torch.cuda.graph(graph):
        gout = _step(graphed, hq, hk, P, most, top)
    said = [[] for _ in range(n)]
    for si, add in enumerate(steps):
        qkv = _randn(g, most, (hq + 2 * hk) * D, dtype=torch.bfloat16)
        for st in (eager, graphed):
            st["qkv"].copy_(qkv)
            st["add"].copy_(_i32(add))
        ep, eo, el = _step(eager, hq, hk, P, most, top)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        gp, go, gl = gout
        rows = sum(max(a, 0) for a in add)
        for x, y in ((ep.slots, gp.slots), (ep.cu, gp.cu), (ep.kv_len, gp.kv_len), (ep.positions, gp.positions),
                     (eo[:rows], go[:rows]), (el[:rows], gl[:rows]), (eager["table"], graphed["table"]),
                     (eager["count"], graphed["count"])):
            assert torch.equal(x, y), f"step {si}"
        assert int(ep.refused) == 0
        # float64 over everything said
        q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([hq * D, hk * D, hk * D], dim=1))
        qr, kr = PK().rotate(q, k, ep.positions, PK().pair_axes((64,)), 1e4)
        at = 0
        for i, a in enumerate(add):
            if a < 0:
                said[i] = []
                continue
            said[i] += [(kr[t], v[t]) for t in range(at, at + a)]
            if a:
                K, V = (torch.stack([x[j] for x in said[i]]) for j in (0, 1))
                m = len(said[i])
                seen = torch.arange(m, device="cuda")[None] <= (m - a + torch.arange(a, device="cuda"))[:, None]
                for h in (0, hq - 1):
                    ref = attend64(qr[at:at + a, h], K[:, h // (hq // hk)], V[:, h // (hq // hk)], seen)
                    check(eo[at:at + a, h], el[at:at + a, h], ref, m, torch.bfloat16, None, f"step {si} request {i}")
            at += a
        for st in (eager, graphed):
            st["ctx"].copy_(_i32([len(x) for x in said]))


def test_question_and_answer_over_the_video_memory():
    """A stream's readout as the prior of the dialogue's exact attention: layer by
    layer, question tokens (a prompt of their own) and answer tokens (over pages)
    get the attention over [near window ; pseudo-tokens ; dialogue] that one
    float64 softmax over all of them gives."""
    import torch
    from tests import gpu_harness as h
    from paper_2606_26762_amd import workloads as W
    log("case: question and answer over the video memory")
    pk = PK()
    wl = W.WORKLOADS["7b"].with_(num_layers=2, num_kv_heads=2, num_q_heads=8, grid_h=7, grid_w=7, frames=14,
                                 window_frames=3, capacity=40, query_tokens=16)
    pair = h.Pair(wl)
    for _ in range(wl.frames):
        pair.step()
    pair.gpu.synthesize(0)
    # the readout alone, in float64: weights of the oracle's attention
    pseudo = pair.oracle[0].synthesize()
    g = _g(44)
    hq, hk, P = 8, 2, 16
    pages = [tuple(torch.full((4, hk, P, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
             for _ in range(2)]
    table, stack, count = torch.full((1, 4), -1, dtype=torch.int32, device="cuda"), _i32([2, 0, 3, 1]), _i32([4])
    said = [[] for _ in range(2)]
    done = 0
    for add in (16, 1, 1):
        p = pk.page_plan(_i32([done]), _i32([add]), table, stack, count, P, add)
        count = p.count
        q = _randn(g, 2, add, hq, D, dtype=torch.bfloat16, scale=2.0)
        o, lse = pair.gpu.attend(0, q.contiguous())
        oo, ol = pair.oracle[0].attend(q.float().cpu().numpy(), hk, pseudo)
        for l in range(2):
            k, v = (_randn(g, add, hk, D, dtype=torch.bfloat16) for _ in range(2))
            qr, kr = pk.rotate(q[l], k, p.positions * 0, pk.pair_axes((64,)), 1e4)   # position 0: as they are
            assert torch.equal(qr, q[l]) and torch.equal(kr, k)
            pk.rotate(None, k, p.positions * 0, pk.pair_axes((64,)), 1e4, v=v, pages=pages[l], slots=p.slots)
            prior = (o[l], lse[l])
            fo, fl = pk.page_attend(qr, pages[l], table, p.cu, p.kv_len, add, prior=prior)
            if done == 0:   # the question: the same as a prompt
                po, pl = pk.prompt_attend(qr, kr, v, p.cu, prior=prior)
                assert float((po.float() - fo.float()).abs().max()) <= 2e-2 and float((pl - fl).abs().max()) <= 2e-3
            torch.cuda.synchronize()
            said[l] += [(k[t], v[t]) for t in range(add)]
            K, V = (torch.stack([x[j] for x in said[l]]).double().cpu() for j in (0, 1))
            m = len(said[l])
            seen = torch.arange(m)[None] <= (m - add + torch.arange(add))[:, None]
            for head in range(hq):
                so, sl, _, _, _ = attend64(q[l, :, head].cpu(), K[:, head // 4], V[:, head // 4], seen)
                rl = torch.from_numpy(np.asarray(ol[l, :, head])).double()
                ro = torch.from_numpy(np.asarray(oo[l, :, head])).double()
                both = torch.logaddexp(sl, rl)
                want = torch.exp(sl - both)[:, None] * so + torch.exp(rl - both)[:, None] * ro
                # the readout's own tolerance, and this attention's
                assert float((fo[:, head].double().cpu() - want).abs().max()) <= h.READOUT_ATOL + 2e-2
                assert float((fl[:, head].double().cpu() - both).abs().max()) <= h.LSE_ATOL + 1e-4
        done += add


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("reqs,hq,hk", [
    ([(40, 1)], 4, 2), ([(9000, 1), (5, 2)], 7, 1), ([(9000, 1)] * 2, 1, 1), ([(700, 150)], 6, 2), ([(12000, 40)], 4, 1),
    ([(0, 600)] * 20, 8, 4)])
def test_result_in_the_prior_s_own_arrays(reqs, hq, hk, dtype):
    """o and lse written over the prior: one wave's rows, joined runs, row blocks,
    context splits; the same bits as beside it."""
    import torch
    log(f"case: in place {reqs[:2]} heads {hq}/{hk} {dtype}")
    pk, g = PK(), _g(51)
    dt, P = _dt(dtype), 16
    need = [(c + a + P - 1) // P for c, a in reqs]
    width, pages = max(need), sum(need)
    table = torch.full((len(reqs), width), -1, dtype=torch.int32, device="cuda")
    order = torch.randperm(pages, generator=g, device="cuda").int()
    for i, n in enumerate(need):
        table[i, :n] = order[sum(need[:i]):sum(need[:i]) + n]
    kv = tuple(_randn(g, pages, hk, P, D, dtype=dt) for _ in range(2))
    add = [a for _, a in reqs]
    total = sum(add)
    cu, lens = _i32(np.cumsum([0] + add).tolist()), _i32([c + a for c, a in reqs])
    q, po = (_randn(g, total, hq, D, dtype=dt) for _ in range(2))
    pl = torch.randn(total, hq, generator=g, device="cuda") + 4
    want_o, want_l = pk.page_attend(q, kv, table, cu, lens, max(add), prior=(po, pl))
    o, lse = po.clone(), pl.clone()
    pk.page_attend(q, kv, table, cu, lens, max(add), prior=(o, lse), out=o, lse=lse)
    k, v = (_randn(g, total, hk, D, dtype=dt) for _ in range(2))
    want_o2, want_l2 = pk.prompt_attend(q, k, v, cu, prior=(po, pl))
    o2, lse2 = po.clone(), pl.clone()
    pk.prompt_attend(q, k, v, cu, prior=(o2, lse2), out=o2, lse=lse2)
    torch.cuda.synchronize()
    assert torch.equal(o, want_o) and torch.equal(lse, want_l)
    assert torch.equal(o2, want_o2) and torch.equal(lse2, want_l2)


def test_no_rows_are_no_error():
    """Empty tensors through the binding: nothing is launched, nothing is refused."""
    import torch
    log("case: no rows")
    pk = PK()
    bf = dict(dtype=torch.bfloat16, device="cuda")
    q, k = torch.empty(0, 4, D, **bf), torch.empty(0, 2, D, **bf)
    kv = tuple(torch.full((3, 2, 16, D), 2.0, **bf) for _ in range(2))
    axes = pk.pair_axes((64,))
    qo, ko = pk.rotate(q, k, _i32([]), axes, 1e4)
    assert qo.shape == q.shape and ko.shape == k.shape
    pk.rotate(q, k, _i32([]), axes, 1e4, v=k, pages=kv, slots=_i32([]))
    for cu in (_i32([0]), _i32([0, 0])):
        n = cu.shape[0] - 1
        for o, lse in (pk.prompt_attend(q, k, k, cu),
                       pk.page_attend(q, kv, torch.zeros(n, 2, dtype=torch.int32, device="cuda"), cu, _i32([5] * n), 1)):
            assert o.shape == q.shape and lse.shape == (0, 4)
    one = torch.ones(2, 4, D, **bf)
    o = torch.full_like(one, 7.5)
    pk.prompt_attend(one, one[:, :2], one[:, :2], _i32([0, 0]), out=o)   # rows, of no sequence
    torch.cuda.synchronize()
    assert bool((o == 7.5).all()) and all(bool((x == 2.0).all()) for x in kv)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_prompts_captured_and_replayed_with_other_lengths(dtype):
    """A graph of a rotation and a prompt's attention on a side stream, padded to its
    sizes; lengths and rows change between the replays, with eager work in between."""
    import torch
    log(f"case: captured prompts {dtype}")
    pk, g = PK(), _g(52)
    dt, hq, hk, n, most = _dt(dtype), 6, 2, 3, 400
    axes = pk.pair_axes((16, 24, 24))
    qkv = torch.zeros(most, (hq + 2 * hk) * D, dtype=dt, device="cuda")
    pos, cu = torch.zeros(3, most, dtype=torch.int32, device="cuda"), _i32([0] * (n + 1))
    o = torch.empty(most, hq, D, dtype=dt, device="cuda")
    lse = torch.empty(most, hq, device="cuda")

    def step(out, l):
        q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([hq * D, hk * D, hk * D], dim=1))
        qr, kr = pk.rotate(q, k, pos, axes, 1e6)
        return pk.prompt_attend(qr, kr, v, cu, out=out, lse=l)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(o, lse)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(o, lse)
    for lens in ([400, 0, 0], [1, 70, 129], [0, 0, 0], [33, 300, 2]):
        qkv.copy_(_randn(g, *qkv.shape, dtype=dt))
        pos.copy_(torch.randint(0, 4000, pos.shape, generator=g, device="cuda").int())
        cu.copy_(_i32(np.cumsum([0] + lens).tolist()))
        o.fill_(7.5)
        lse.fill_(8.5)
        want, wl = torch.full_like(o, 7.5), torch.full_like(lse, 8.5)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step(want, wl)
        side.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want) and torch.equal(lse, wl), f"lengths {lens}"
        assert bool((o[sum(lens):] == 7.5).all())


def test_plan_and_rotation_on_a_stream_of_their_own():
    """The stream argument: the call waits for that stream's work, not the current one's."""
    import torch
    log("case: plan and rotation on a side stream")
    pk, g = PK(), _g(53)
    side = torch.cuda.Stream()
    n, P, most = 40, 8, 200
    args = []
    for _ in range(2):
        args.append((_i32([5 * i % 37 for i in range(n)]), _i32([i % 6 - (i % 11 == 3) * 7 for i in range(n)]),
                     torch.arange(n * 8, device="cuda").int().view(n, 8) % 300,
                     torch.arange(300, device="cuda").int().flip(0).contiguous(), _i32([50])))
    q = _randn(g, most, 4, D, dtype=torch.bfloat16)
    axes = pk.pair_axes((64,))
    a = pk.page_plan(*args[0], P, most)
    ra = pk.rotate(q, None, a.positions, axes, 1e4)[0]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        big = torch.randn(4000, 4000, device="cuda") @ torch.randn(4000, 4000, device="cuda")
        q2 = q * 1
    b = pk.page_plan(*args[1], P, most, stream=side)
    rb = pk.rotate(q2, None, b.positions, axes, 1e4, stream=side)[0]
    side.synchronize()
    assert bool(big.isfinite().all())
    for f in pk.PagePlan.__slots__:
        assert torch.equal(getattr(a, f), getattr(b, f)), f
    assert torch.equal(ra, rb) and all(torch.equal(x, y) for x, y in zip(args[0], args[1]))


def test_pages_few_rows_beside_many():
    """So many requests that those of few rows go to runs of tiles and the others to
    row blocks, which split their context."""
    log("case: few rows beside many")
    reqs = [(53 * i % 700, 1 + i % 2) for i in range(38)] + [(900, 50), (4000, 20)]
    _paged(reqs, 6, 2, 16, "bf16", 61, prior=True)


@pytest.mark.parametrize("reqs", [[(3000, 1), (10, 1)], [(1, 1), (700, 2), (0, 0), (64, 30)]])
def test_few_rows_where_there_might_have_been_many(reqs):
    """max_add above what any request has: row blocks with few rows in them."""
    log(f"case: few rows, many allowed {reqs}")
    _paged(reqs, 14, 2, 16, "bf16", 62, prior=True, max_add=300)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("add,n", [(1, 5), (3, 40), (70, 2)])
def test_pages_shared_by_requests_strided_queries_no_lse(add, n, dtype):
    """Requests over the same pages get the same rows, whichever of them asks; queries
    inside a projection's rows; lse not wanted; k and v one tensor."""
    import torch
    log(f"case: shared pages {n} x {add} {dtype}")
    pk, g = PK(), _g(71)
    dt, hq, hk, P, ctx = _dt(dtype), 6, 2, 16, 500
    kv = _randn(g, 40, hk, P, D, dtype=dt)
    row = torch.randperm(40, generator=g, device="cuda").int()[:(ctx + add + P - 1) // P]
    table = row.repeat(n, 1).contiguous()
    cu = _i32([add * i for i in range(n + 1)])
    lens = _i32([ctx + add] * n)
    one = _randn(g, add, (hq + 2 * hk) * D, dtype=dt)
    q = one.repeat(n, 1)[:, :hq * D].unflatten(1, (-1, D))   # rows at the projection's stride
    assert not q.is_contiguous()
    o, lse = pk.page_attend(q, (kv, kv), table, cu, lens, add)
    o2, none = pk.page_attend(q.contiguous(), (kv, kv), table, cu, lens, add, lse=False)
    torch.cuda.synchronize()
    assert none is False and torch.equal(o, o2)
    key = torch.arange(ctx + add, device="cuda")
    flat = kv[row.long()].permute(1, 0, 2, 3).flatten(1, 2)[:, :ctx + add]
    seen = key[None] <= (ctx + torch.arange(add, device="cuda"))[:, None]
    for i in range(n):
        sl = slice(i * add, (i + 1) * add)
        for h in range(hq):
            ref = attend64(q[sl, h], flat[h // 3], flat[h // 3], seen)
            check(o[sl, h], lse[sl, h], ref, ctx + add, dt, None, f"request {i}, head {h}")


# The last context split of these has two or three tiles, and the run of page ids that
# the second or the third is in begins inside it (tests/test_exact_splits.py replays
# the staging for all lengths).
SHORT_LAST = [
    ([(1024, 16)], 28, 4, 1, None), ([(1050, 128)], 28, 4, 1, None), ([(1072, 16), (1072, 16), (300, 16)], 28, 4, 1, None),
    ([(1024, 300)], 8, 8, 1, None), ([(2048, 16)], 28, 4, 2, None), ([(6144, 16)], 28, 4, 2, None),
    ([(8128, 128)], 28, 4, 8, None), ([(16320, 128)], 28, 4, 16, None), ([(16320, 128)], 28, 4, 16, 2048),
    ([(16320, 100)], 32, 8, 16, None)]


@pytest.mark.parametrize("reqs,hq,hk,P,width", SHORT_LAST)
def test_pages_whose_ids_begin_anew_in_a_short_last_split(reqs, hq, hk, P, width):
    log(f"case: short last split {reqs} heads {hq}/{hk} page {P} width {width}")
    _paged(reqs, hq, hk, P, "bf16", 31, width=width)


@pytest.mark.parametrize("reqs,hq,hk,P,width", SHORT_LAST)
def test_page_size_does_not_change_the_result(reqs, hq, hk, P, width):
    """The same tokens in small pages and in pages of 256, in tables of as many tokens:
    the same keys in the same order, so the same bits."""
    import torch
    log(f"case: small pages and large {reqs} heads {hq}/{hk} page {P} width {width}")
    pk, g = PK(), _g(32)
    kv, add = [c + a for c, a in reqs], [a for _, a in reqs]
    span = ((width * P if width else max(kv)) + 255) // 256 * 256
    q = _randn(g, sum(add), hq, D, dtype=torch.bfloat16, scale=2.0)
    k, v = (_randn(g, len(reqs), span, hk, D, dtype=torch.bfloat16) for _ in range(2))
    got = []
    for size in (P, 256):
        n = span // size
        order = torch.randperm(len(reqs) * n, generator=g, device="cuda")
        pages = []
        for x in (k, v):
            y = torch.empty(len(reqs) * n, hk, size, D, dtype=x.dtype, device="cuda")
            y[order] = x.view(len(reqs) * n, size, hk, D).transpose(1, 2)
            pages.append(y)
        table = order.view(len(reqs), n).int().contiguous()
        got.append(pk.page_attend(q, pages, table, _i32(np.cumsum([0] + add).tolist()), _i32(kv), max(add)))
    torch.cuda.synchronize()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
