"""GPU: the calls of a serving step around a paged dialogue against plain
implementations: head norms with the rotation, pages of 4 bits and their
attention (float64), forked and released pages (lists), and a run of them
together, eager and captured.  Each test prints its case before any GPU step.

Tolerances of the attention are tests/test_gpu_exact.py's: the values that a cache of
4 bits holds enter the products exactly.  Head norms: the mean is float64's to 2^-45;
its root's inverse, the product with x and that with the weight round once each, 3 u
of the value, before the rotation's own bound; a value below float32's normal range
is off by up to 2^-149 a step instead.
"""
import math

import numpy as np
import pytest

from tests.test_gpu_exact import D, HB, PK, U, _dt, _g, _gpu, _i32, _randn, attend64, check, log, rotate64  # noqa: F401

pytestmark = pytest.mark.gpu


# -- head norms and rotation ----------------------------------------------------------


def normed64(x, w, eps):
    x = x.double()
    y = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    return y if w is None else y * w.double()


def check_normed(got, x, w, eps, pos, axes, theta):
    """normed64, then the rotation's bound as in tests/test_gpu_exact.py, each value with 3 u more."""
    want, size = rotate64(normed64(x, w, eps), pos, axes, theta)
    import torch
    tol = (9 * U + 2e-6) * size + (HB if got.dtype == torch.bfloat16 else U) * want.abs() + 2.0 ** -147
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,hq,hk", [(1, 28, 4), (3, 1, 1), (65, 7, 1), (700, 6, 3), (5000, 2, 1)])
@pytest.mark.parametrize("store", [False, True])
def test_norm_rotate(n, hq, hk, dtype, store):
    import torch
    log(f"case: norm_rotate {n} tokens, heads {hq}/{hk} {dtype} store {store}")
    pk, g = PK(), _g(31)
    dt, eps, theta, P = _dt(dtype), 1e-6, 1e6, 16
    qkv = _randn(g, n, (hq + 2 * hk) * D, dtype=dt)
    # heads from far below eps to beyond float32's squares
    qkv *= (10.0 ** torch.randint(-25, 30, (n, hq + 2 * hk, 1), generator=g, device="cuda")).expand(-1, -1, D).flatten(1).to(dt)
    q, k, v = (x.unflatten(1, (-1, D)) for x in qkv.split([hq * D, hk * D, hk * D], dim=1))
    qw, kw = (1 + _randn(g, D, dtype=dt, scale=0.3) for _ in range(2))
    pos = torch.stack([torch.randint(0, m, (n,), generator=g, device="cuda") for m in (2 ** 31 - 1, 100, 5000)]).int()
    axes = pk.pair_axes((16, 24, 24), interleaved=n % 2 == 1)
    pages = (n + P - 1) // P + 2
    kp, vp = (torch.full((pages, hk, P, D), 3.0, dtype=dt, device="cuda") for _ in range(2))
    slots = torch.randperm(pages * P, generator=g, device="cuda")[:n].int()
    out = torch.arange(n, device="cuda") % 7 == 3   # not stored: below and beyond the pages
    slots[out] = torch.where(torch.arange(n, device="cuda") % 2 == 0, -1 - slots, pages * P + slots)[out].int()
    ko = torch.empty(n, hk, D, dtype=dt, device="cuda")
    kw_args = dict(v=v, pages=(kp, vp), slots=slots) if store else {}
    qo, _ = pk.norm_rotate(q, k, pos, axes, theta, qw, kw, eps, k_out=ko, **kw_args)
    torch.cuda.synchronize()
    check_normed(qo, q, qw, eps, pos, axes, theta)
    check_normed(ko, k, kw, eps, pos, axes, theta)
    if store:
        want_k, want_v = (torch.full((pages, hk, P, D), 3.0, dtype=dt, device="cuda") for _ in range(2))
        s = slots[~out].long()
        want_k[s // P, :, s % P] = ko[~out]
        want_v[s // P, :, s % P] = v[~out]
        assert torch.equal(kp, want_k) and torch.equal(vp, want_v)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_norm_rotate_in_place_alone_without_weights(dtype):
    """In place on strided rows; q or k alone; no weights; zeros, infinities and NaN in a head stay in it."""
    import torch
    log(f"case: norm_rotate in place {dtype}")
    pk, g = PK(), _g(32)
    dt, n, hq, hk = _dt(dtype), 37, 6, 2
    x = _randn(g, n, (hq + hk) * D + 64, dtype=dt)
    x[3, 2 * D + 5] = math.inf
    x[4, 7 * D + 9] = math.nan
    x[5, :D] = 0
    y = x.clone()
    q, k = (t[:, a * D:b * D].unflatten(1, (-1, D)) for t, a, b in ((x, 0, hq), (x, hq, hq + hk)))
    pos = torch.randint(0, 10 ** 6, (n,), generator=g, device="cuda").int()
    axes, w = pk.pair_axes((20, 44)), 1 + _randn(g, D, dtype=dt)
    a, b = pk.norm_rotate(q, None, pos, axes, 1e4, None, w, 1e-5)
    assert b is None
    a2, b2 = pk.norm_rotate(None, k, pos, axes, 1e4, w, w, 1e-5)
    assert a2 is None
    pk.norm_rotate(q, k, pos, axes, 1e4, None, w, 1e-5, q_out=q, k_out=k)
    torch.cuda.synchronize()

    def same(s, t):
        return torch.equal(s.isnan(), t.isnan()) and torch.equal(s.nan_to_num(), t.nan_to_num())

    assert same(q, a) and same(k, b2) and same(x[:, (hq + hk) * D:], y[:, (hq + hk) * D:])
    assert bool((a[5, 0] == 0).all()) and bool(b2[4, 1].isnan().all())
    heads = y[:, :hq * D].unflatten(1, (-1, D))
    good = torch.ones(n, hq, dtype=torch.bool, device="cuda")
    good[3, 2] = False
    assert torch.equal(a.isnan().any(-1), ~good)
    rows = [i for i in range(n) if i != 3]
    check_normed(a[rows], heads[rows], None, 1e-5, torch.stack([pos, pos])[:, rows], axes, 1e4)


def test_norm_rotate_eps_zero():
    import torch
    log("case: norm_rotate eps 0")
    pk, g = PK(), _g(33)
    q = _randn(g, 9, 4, D, dtype=torch.float32) * 1e-22
    # heads at the ends of float32: of its smallest numbers, and near its largest
    q[3] = torch.randint(-9, 10, (4, D), generator=g, device="cuda") * 2.0 ** -149
    q[4] = torch.rand(4, D, generator=g, device="cuda") * 3.4e38
    q[5, :, ::3] = 1e-30
    q[2, 1] = 0
    a, _ = pk.norm_rotate(q, None, _i32([0] * 9), pk.pair_axes((64,)), 1e4, None, None, 0.0)
    torch.cuda.synchronize()
    assert bool(a[2, 1].isnan().all())
    a[2, 1], q[2, 1] = 0, 1e-22
    want = normed64(q, None, 0.0)
    want[2, 1] = 0
    assert bool(((a.double() - want).abs() <= 3 * U * want.abs()).all())


# -- pages of 4 bits --------------------------------------------------------------------

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def codes_ref(x):
    """The definition: float64 rows [n][128] -> codes [n][128], scales [n][4]."""
    x = np.asarray(x, dtype=np.float64).reshape(len(x), 4, 32)
    codes, scales = np.zeros(x.shape, np.int64), np.zeros(x.shape[:2], np.int64)
    for i in np.ndindex(*scales.shape):
        b = x[i]
        if not np.isfinite(b).all():
            scales[i] = 255
            continue
        top = np.abs(b).max()
        e = -125
        while e < 125 and top > math.ldexp(7.0, e):
            e += 1
        scales[i] = e + 127
        a = np.abs(b) * math.ldexp(1.0, -e)
        off = np.abs(a[:, None] - GRID)
        best = off.argmin(1)
        for j in range(32):
            near = np.flatnonzero(off[j] == off[j].min())
            best[j] = near[near % 2 == 0][0] if len(near) > 1 else near[0]
        codes[i] = best + 8 * np.signbit(b)
    return codes.reshape(len(x), 128), scales


def values_ref(codes, scales):
    """float32 values [..., 128] of unpacked codes and scales."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    with np.errstate(over="ignore"):
        v = (v.reshape(*scales.shape, 32) * np.ldexp(1.0, scales - 127)[..., None]).astype(np.float32)
    v[scales == 255] = np.nan
    return v.reshape(codes.shape)


def unpack(codes):
    """Bytes [..., 64] -> codes [..., 128]"""
    c = codes.cpu().numpy().astype(np.int64)
    return np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], 128)


def pages4(n, hk, P, fill=255):
    """Pages whose every row reads as NaN."""
    import torch
    u8 = dict(dtype=torch.uint8, device="cuda")
    return tuple(torch.full((n, hk, P, w), f, **u8) for w, f in ((64, 0x77), (64, 0x77), (4, fill), (4, fill)))


def _blocks(dtype, g):
    """Rows whose blocks hold the format's borders, ends of the range, infinities and NaN."""
    import torch
    rows = [_randn(g, 200, D, dtype=torch.float32, scale=s) for s in (1.0, 1e-3, 1e4)]
    edge = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.5, 7.0, 7.03125, 7.5, 0.0, -0.0, 8.0, 1e-9], device="cuda")
    both = torch.cat([edge, -edge])
    around = torch.stack([both * (1 + 2 * d * U) for d in (-2, -1, 0, 1, 2)])   # next to the borders in float32
    for e in (-149, -130, -126, -125, -124, -100, -2, 0, 1, 100, 122, 123, 124, 125):
        rows.append((around.double() * 2.0 ** e).float().repeat(1, 4))
    odd = _randn(g, 40, D, dtype=torch.float32)
    for i, x in enumerate((math.inf, -math.inf, math.nan)):
        odd[i::4, 32 * i + 7] = x
    top = torch.finfo(_dt(dtype)).max
    odd[3::4, 50] = top
    odd[7::8, 90] = -top
    rows += [odd, torch.zeros(2, D, device="cuda")]
    bits = torch.arange(1 << 16, device="cuda").to(torch.int32).to(torch.int16).view(torch.bfloat16).float()
    rows.append(bits[torch.randperm(1 << 16, generator=g, device="cuda")].view(-1, D))   # every bfloat16
    rows.append(bits.view(-1, D))
    x = torch.cat(rows).to(_dt(dtype))
    return x[:x.shape[0] // 2 * 2].contiguous()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_page4_codes(dtype):
    """Codes and scales bit for bit, and the values read back."""
    import torch
    log(f"case: page4 codes {dtype}")
    pk, g = PK(), _g(41)
    dt = _dt(dtype)
    x = _blocks(dtype, g).unflatten(0, (-1, 2))
    n, hk, P = x.shape[0], 2, 8
    k, v = x, x.flip(0).contiguous()
    pages = pages4(n // P + 2, hk, P)
    slots = torch.randperm((n // P + 2) * P, generator=g, device="cuda")[:n].int()
    pk.page4_store(k, v, pages, slots)
    kr, vr = pk.page4_read(pages, slots, dt)
    torch.cuda.synchronize()
    s = slots.cpu().numpy().astype(np.int64)
    for rows, codes, scales, back in ((k, pages[0], pages[2], kr), (v, pages[1], pages[3], vr)):
        flat = rows.double().cpu().numpy().reshape(-1, D)
        wc, ws = codes_ref(flat)
        wc, ws = wc.reshape(n, hk, D), ws.reshape(n, hk, 4)
        got_c = unpack(codes).transpose(0, 2, 1, 3).reshape(-1, hk, D)
        got_s = scales.cpu().numpy().astype(np.int64).transpose(0, 2, 1, 3).reshape(-1, hk, 4)
        assert (got_s[s] == ws).all()
        assert (got_c[s] == wc).all()
        rest = np.ones(len(got_s), bool)
        rest[s] = False
        assert (got_s[rest] == 255).all() and (got_c[rest] == 7).all()
        want = values_ref(wc, ws)
        got = back.float().cpu().numpy()
        assert ((got == want) | (np.isnan(got) & np.isnan(want))).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_page4_reads_every_scale_and_code(dtype):
    """Also those that store does not write."""
    import torch
    log(f"case: page4 read {dtype}")
    pk = PK()
    byte, scale = np.meshgrid(np.arange(256), np.arange(256))
    n = 256 * 4   # a row: one scale, 64 of the bytes
    codes = byte.reshape(n, 64).astype(np.uint8)
    scales = np.repeat(scale.reshape(n, 64)[:, :1], 4, 1).astype(np.uint8)
    kp, ks = torch.from_numpy(codes).cuda().view(n // 8, 1, 8, 64), torch.from_numpy(scales).cuda().view(n // 8, 1, 8, 4)
    pages = (kp, kp.flip(0).contiguous(), ks, ks.flip(0).contiguous())
    k, v = pk.page4_read(pages, torch.arange(n, device="cuda").int(), _dt(dtype))
    torch.cuda.synchronize()
    for got, c, s in ((k, pages[0], pages[2]), (v, pages[1], pages[3])):
        want = values_ref(unpack(c).reshape(n, 1, D), s.cpu().numpy().astype(np.int64).reshape(n, 1, 4))
        want = torch.from_numpy(want).to(_dt(dtype)).float().numpy()
        got = got.float().cpu().numpy()
        assert ((got == want) | (np.isnan(got) & np.isnan(want))).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,hk,P", [(1, 1, 1), (5, 3, 16), (1000, 8, 64), (77, 1, 1024), (10007, 8, 32)])
def test_page4_rows_strided_repeated_and_of_no_slot(n, hk, P, dtype):
    import torch
    log(f"case: page4 rows {n} x {hk} page {P} {dtype}")
    pk, g = PK(), _g(42)
    dt = _dt(dtype)
    qkv = _randn(g, n, (2 * hk + 3) * D, dtype=dt)
    k, v = qkv[:, D:(hk + 1) * D].unflatten(1, (-1, D)), qkv[:, (hk + 2) * D:(2 * hk + 2) * D].unflatten(1, (-1, D))
    count = (n + P - 1) // P + 1
    pages = pages4(count, hk, P)
    slots = torch.randperm(count * P, generator=g, device="cuda")[:n].int()
    if n > 3:
        slots[1], slots[3] = -1, count * P
    pk.page4_store(k, v, pages, slots)
    ask = torch.cat([slots, slots[:1], _i32([-5, 2 ** 31 - 1])])
    wide = torch.full((n + 3, (2 * hk + 1) * D), 5.0, dtype=dt, device="cuda")
    ko, vo = wide[:, :hk * D].unflatten(1, (-1, D)), wide[:, (hk + 1) * D:].unflatten(1, (-1, D))
    pk.page4_read(pages, ask, dt, k_out=ko, v_out=vo)
    torch.cuda.synchronize()
    assert bool((wide[:, hk * D:(hk + 1) * D] == 5.0).all())
    some = list(range(n)) if n <= 1000 else list(range(200)) + list(range(n - 200, n))   # (the reference is slow)
    for x, got in ((k, ko), (v, vo)):
        c, s = codes_ref(x[some].double().cpu().numpy().reshape(-1, D))
        want = torch.from_numpy(values_ref(c, s)).view(len(some), hk, D).to(dt).cuda()
        if n > 3:
            want[1], want[3] = 0, 0
        assert torch.equal(got[some], want) and torch.equal(got[n], want[0]) and bool((got[n + 1:] == 0).all())
        if n > 1000:   # the rest in parts, which one piece to a thread takes
            parts = pages4(count, hk, P)
            for i in range(0, n, 1000):
                pk.page4_store(k[i:i + 1000], v[i:i + 1000], parts, slots[i:i + 1000].contiguous())
            assert all(torch.equal(a, b) for a, b in zip(parts, pages))


def held(g, pages, own, m, hk, P, dtype, scale=1.2):
    """Rows of normal values put into the first m places of the pages `own`; -> the values held, [hk][m][D] each."""
    import torch
    k, v = (_randn(g, m, hk, D, dtype=_dt(dtype), scale=scale) for _ in range(2))
    at = torch.arange(m, device="cuda")
    slots = (own[at // P] * P + at % P).int()
    pk = PK()
    if m:
        pk.page4_store(k, v, pages, slots)
    k, v = pk.page4_read(pages, slots, _dt(dtype))
    return k.transpose(0, 1), v.transpose(0, 1)


def _paged4(reqs, hq, hk, P, dtype, seed, prior=False, tail=2, bad=(), width=None, lens=None, max_add=None, workspace=None):
    """reqs: (context, new); everything that no token fills is NaN; bad: (request, page)
    entries set outside the pages.  lens: kv_len where it is not context + new."""
    import torch
    pk, g = PK(), _g(seed)
    dt = _dt(dtype)
    kv = [c + a for c, a in reqs] if lens is None else lens
    need = [(max(x, 0) + P - 1) // P for x in kv]
    width = width or max(max(need), 1)
    need = [min(x, width) for x in need]
    count = sum(need) + 2
    order = torch.randperm(count, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(reqs), width), -7, dtype=torch.int32, device="cuda")
    pages = pages4(count, hk, P)
    at, ks, vs = 0, [], []
    for i, n in enumerate(need):
        own = order[at:at + n].long()
        at += n
        table[i, :n] = own.int()
        k, v = held(g, pages, own, min(max(kv[i], 0), width * P), hk, P, dtype)
        ks.append(k)
        vs.append(v)
    gone = [set() for _ in reqs]
    for i, p in bad:
        table[i, p] = [-1, count, 2 ** 31 - 1, -2 ** 31][(i + p) % 4]
        gone[i].add(p)
    add = [a for _, a in reqs]
    total = sum(add) + tail
    q = _randn(g, total, hq, D, dtype=dt, scale=2.0)
    o = torch.full((total, hq, D), 7.5, dtype=dt, device="cuda")
    lse = torch.full((total, hq), 8.5, device="cuda")
    pr = (_randn(g, total, hq, D, dtype=dt), torch.randn(total, hq, generator=g, device="cuda") + 3) if prior else None
    pk.page4_attend(q, pages, table, _i32(np.cumsum([0] + add).tolist()), _i32(kv), max_add or max(max(add), 1), out=o,
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
def test_page4_attend(reqs, hq, hk, P, dtype):
    log(f"case: page4 attend {reqs[:6]} heads {hq}/{hk} page {P} {dtype}")
    _paged4(reqs, hq, hk, P, dtype, 11)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("reqs", [[(400, 1), (77, 1)], [(400, 30), (77, 9)]])
def test_page4_attend_with_prior(reqs, dtype):
    log(f"case: page4 attend with prior {reqs} {dtype}")
    _paged4(reqs, 14, 2, 16, dtype, 12, prior=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("add", [1, 25])
def test_page4_attend_pages_that_are_none_hold_no_tokens(dtype, add):
    log(f"case: page4 bad pages {dtype} add {add}")
    bad = [(0, 0), (0, 5), (0, 6), (0, 7), (0, 8), (0, 9), (0, 10), (1, 0), (1, 1), (1, 2), (1, 3), (2, 20)]
    _paged4([(300, add), (64 - add, add), (320, add)], 6, 2, 16, dtype, 13, bad=bad)
    _paged4([(300, add), (64 - add, add), (320, add)], 6, 2, 16, dtype, 13, bad=bad, prior=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("prior", [False, True])
def test_page4_attend_rows_before_the_first_token_see_nothing(dtype, prior):
    log(f"case: page4 short kv_len {dtype} prior {prior}")
    _paged4([(0, 10), (0, 3), (0, 40), (0, 2), (0, 1)], 6, 2, 16, dtype, 14, prior=prior, lens=[4, 0, -9, 300, 0], width=19)


@pytest.mark.parametrize("reqs", [[(5000, 1)], [(2000, 1), (9000, 1), (10, 1)], [(6000, 50)], [(4000, 1), (4500, 200)],
                                  [(20000, 2), (300, 1)]])
def test_page4_attend_split_over_the_context(reqs):
    log(f"case: page4 split context {reqs}")
    _paged4(reqs, 7, 1, 16, "bf16", 17, prior=True)
    _paged4(reqs, 4, 2, 32, "fp32", 17)


def test_page4_attend_of_many_requests():
    log("case: page4 attend of many requests")
    rng = np.random.default_rng(21)
    reqs = [(int(rng.integers(0, 90)), int(rng.choice([0, 1, 1, 1, 1, 2]))) for _ in range(700)]
    reqs[300], reqs[690] = (300, 40), (10, 70)
    _paged4(reqs, 2, 1, 8, "bf16", 21)


@pytest.mark.parametrize("reqs", [[(255, 1), (0, 1), (200, 0)], [(256, 1), (3, 1)], [(250, 6)] * 3, [(100, 156), (17, 1)], [(255, 1)] * 100])
def test_page4_attend_of_short_tables(reqs):
    """Contexts that one wave goes through, so that nothing is left to join, and the first that it does not."""
    log(f"case: page4 short tables {reqs[:3]}")
    _paged4(reqs, 7, 1, 16, "bf16", 24, prior=True)
    _paged4(reqs, 6, 2, 8, "bf16", 24)


def test_page4_attend_of_many_single_tokens():
    """Hundreds of requests of one token or none: short items, and long ones that several waves share."""
    log("case: page4 attend of many single tokens")
    rng = np.random.default_rng(22)
    reqs = [(int(rng.integers(0, 700)), int(rng.random() < 0.9)) for _ in range(300)]
    reqs[5], reqs[200], reqs[299] = (9000, 1), (6000, 1), (3000, 1)
    _paged4(reqs, 5, 1, 16, "bf16", 22, prior=True)


@pytest.mark.parametrize("hq,hk,P,prior", [(14, 2, 16, True), (28, 4, 16, False)])
def test_page4_attend_of_some_rows_to_many_requests(hq, hk, P, prior):
    """So many requests of some rows that they go in groups of 32, whole items and shared ones."""
    log(f"case: page4 attend of some rows heads {hq}/{hk} prior {prior}")
    _paged4([(97 * i % 1500, i % 17) for i in range(64)], hq, hk, P, "bf16", 23, prior=prior)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq,most", [(2, 4), (2, 1), (40, 4)])
def test_page4_attend_rows_beyond_max_add_are_left(hq, most, dtype):
    import torch
    log(f"case: page4 max_add {most} {dtype}")
    pk, g = PK(), _g(16)
    dt = _dt(dtype)
    pages = pages4(4, 1, 16)
    held(g, pages, torch.arange(4, device="cuda"), 64, 1, 16, dtype)
    q = _randn(g, 12, hq, D, dtype=dt)
    args = (pages, _i32([[0, 1], [2, 3]]), _i32([0, 8, 12]), _i32([20, 30]))
    full, _ = pk.page4_attend(q, *args, 8)
    o = torch.full_like(full, 7.5)
    pk.page4_attend(q, *args, most, out=o)
    torch.cuda.synchronize()
    keep = torch.zeros(12, dtype=torch.bool, device="cuda")
    keep[:most] = keep[8:8 + most] = True
    assert bool((o[~keep] == 7.5).all())
    got, want = o[keep].double(), full[keep].double()
    assert bool(((got - want).abs() <= 2 * HB * (want.abs() + 0.05)).all())


@pytest.mark.parametrize("P", [1, 2])
def test_page4_attend_ids_staged_in_runs(P):
    log(f"case: page4 {P} tokens to a page")
    _paged4([(4500, 1), (4300, 70)], 2, 1, P, "bf16", 18)


@pytest.mark.parametrize("reqs,hq,hk,P,width", [
    ([(1024, 16)], 28, 4, 1, None), ([(1072, 16), (1072, 16), (300, 16)], 28, 4, 1, None), ([(6144, 16)], 28, 4, 2, None),
    ([(16320, 128)], 28, 4, 16, 2048), ([(4000, 1), (10, 40), (1, 1)], 28, 4, 16, 2048)])
def test_page4_attend_tables_wider_than_the_contexts(reqs, hq, hk, P, width):
    log(f"case: page4 attend {reqs} heads {hq}/{hk} page {P} width {width}")
    _paged4(reqs, hq, hk, P, "bf16", 31, width=width)


@pytest.mark.parametrize("add,n,ctx", [(40, 3, 700), (300, 1, 100), (512, 2, 3000)])
def test_page4_attend_is_page_attend_of_the_values(add, n, ctx):
    """Many rows: the same products in the same order over the values in bfloat16 pages, so the same
    bits.  Requests of some rows go to another kernel than there: each within its bound of float64."""
    import torch
    log(f"case: page4 attend against exact pages {n} x {add} over {ctx}")
    pk, g = PK(), _g(51)
    hq, hk, P = 14, 2, 16
    width = (ctx + add + P - 1) // P
    pages = pages4(n * width, hk, P)
    order = torch.randperm(n * width, generator=g, device="cuda")
    table = order.int().view(n, width)
    exact = tuple(torch.full((n * width, hk, P, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    at = torch.arange(ctx + add, device="cuda")
    for i in range(n):
        own = table[i].long()
        for x, y in zip(exact, held(g, pages, own, ctx + add, hk, P, "bf16")):
            x[own[at // P], :, at % P] = y.transpose(0, 1)
    q = _randn(g, n * add, hq, D, dtype=torch.bfloat16, scale=2.0)
    cu, lens = _i32([add * i for i in range(n + 1)]), _i32([ctx + add] * n)
    a = pk.page4_attend(q, pages, table, cu, lens, add)
    b = pk.page_attend(q, exact, table, cu, lens, add)
    torch.cuda.synchronize()
    if add >= 300:
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        return
    seen = at[None] <= (ctx + torch.arange(add, device="cuda"))[:, None]
    for i in range(n):
        K, V = (x[table[i].long()].transpose(0, 1).flatten(1, 2)[:, :ctx + add] for x in exact)
        sl = slice(i * add, (i + 1) * add)
        for h in range(hq):
            ref = attend64(q[sl, h], K[h // 7], V[h // 7], seen)
            for o, lse in (a, b):
                check(o[sl, h], lse[sl, h], ref, ctx + add, torch.bfloat16, None, f"request {i}, head {h}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("add,hq,hk", [(20, 2, 2), (4, 6, 2), (100, 6, 2)])
def test_page4_attend_nan_blocks_stay_where_they_are_seen(add, hq, hk, dtype):
    """A block that reads as NaN reaches the rows that see it and, of a value, its own 32 dims only."""
    import torch
    log(f"case: page4 attend NaN blocks add {add} {dtype}")
    pk, g = PK(), _g(4)
    dt, P, ctx = _dt(dtype), 16, 300
    n = ctx + add
    pages = pages4((n + P - 1) // P, hk, P)
    own = torch.randperm(pages[0].shape[0], generator=g, device="cuda")
    held(g, pages, own, n, hk, P, dtype)
    q = _randn(g, add, hq, D, dtype=dt)
    args = (own.int()[None], _i32([0, add]), _i32([n]), add)
    clean = pk.page4_attend(q, pages, *args)
    a, b = ctx + add // 2, ctx + add - 1   # a value's block, the last key's block
    pages[3][own[a // P], 0, a % P, 2] = 255
    pages[2][own[b // P], hk - 1, b % P, 1] = 255
    o, lse = pk.page4_attend(q, pages, *args)
    torch.cuda.synchronize()
    grp = hq // hk
    same = torch.ones(add, hq, D, dtype=torch.bool, device="cuda")
    same[a - ctx:, :grp, 64:96] = False
    same[b - ctx:, -grp:] = False
    assert bool(o[a - ctx:, :grp, 64:96].isnan().all()) and bool(o[b - ctx:, -grp:].isnan().all())
    tol = 2 * HB if dt == torch.bfloat16 else 1e-5
    d = (o.double() - clean[0].double()).abs()
    assert bool((d[same] <= tol * (clean[0].double().abs()[same] + 0.05)).all())
    keep = torch.ones(add, hq, dtype=torch.bool, device="cuda")
    keep[b - ctx:, -grp:] = False
    assert torch.equal(lse[keep], clean[1][keep])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_page4_attend_one_key_returns_its_value(dtype):
    """A row with one key: the value held.  In float32 its weight w = 2^(s c - m) is 1 but for the
    rounding of the reference m, and w v, 1 / w and their product round once each: 3 u of the
    value (3.01 with the products of the errors); in bfloat16 the rounding of the result takes
    that away, as a value has three bits: bit for bit."""
    import torch
    log(f"case: page4 attend of one key {dtype}")
    pk, g = PK(), _g(5)
    n, hq, hk, P = 50, 4, 2, 1
    pages = pages4(n, hk, P)
    own = torch.randperm(n, generator=g, device="cuda")
    k, v = held(g, pages, own, n, hk, P, dtype, scale=3.0)
    q = _randn(g, n, hq, D, dtype=_dt(dtype), scale=3.0)
    o, _ = pk.page4_attend(q, pages, own.int()[:, None].contiguous(), _i32(list(range(n + 1))), _i32([1] * n), 1)
    torch.cuda.synchronize()
    want = v.transpose(0, 1).repeat_interleave(2, dim=1)
    tol = 3.01 * U if dtype == "fp32" else 0.0
    assert bool(((o.double() - want.double()).abs() <= tol * want.double().abs()).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_page4_cache_beyond_4_gib(dtype):
    """Pages whose byte offsets pass 32 bits, unsigned too."""
    import torch
    log(f"case: large cache of 4 bits {dtype}")
    pk, g = PK(), _g(19)
    dt, P, hk = _dt(dtype), 64, 8
    count = (5 << 30) // (hk * P * 64)
    u8 = dict(dtype=torch.uint8, device="cuda")
    pages = tuple(torch.empty(count, hk, P, w, **u8) for w in (64, 64, 4, 4))
    top = [count - 1, count - 2, count // 2 + 3, 0]
    small = pages4(4, hk, P)
    held(g, small, torch.arange(4, device="cuda"), 4 * P, hk, P, dtype)
    for x, s in zip(pages, small):
        x[torch.tensor(top, device="cuda")] = s
    for add in (1, 20):
        q = _randn(g, add, 16, D, dtype=dt)
        args = (_i32([0, add]), _i32([230]), add)
        o, lse = pk.page4_attend(q, pages, _i32([top]), *args)
        o2, lse2 = pk.page4_attend(q, small, _i32([[0, 1, 2, 3]]), *args)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    # written and read there
    k, v = (_randn(g, 3, hk, D, dtype=dt) for _ in range(2))
    near = pages4(1, hk, 4)
    slots = _i32([(count - 1) * P + 63, (count // 2 + 3) * P, 5])
    pk.page4_store(k, v, pages, slots)
    pk.page4_store(k, v, near, _i32([0, 1, 2]))
    got, want = pk.page4_read(pages, slots, dt), pk.page4_read(near, _i32([0, 1, 2]), dt)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # and copied there
    pk.page_copy(pages, _i32([count - 1]), _i32([count - 3]))
    for x in pages:
        assert torch.equal(x[count - 3], x[count - 1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [3, 70])
def test_page4_attend_senseless_rows_stay_inside(dtype, n):
    """cu that falls, is negative or passes the rows, tables and lengths of any value."""
    import torch
    log(f"case: page4 senseless cu {dtype} {n}")
    pk, g = PK(), _g(8)
    dt = _dt(dtype)
    total, hq, hk, P = 200, 4, 2, 16
    wild = [0, 60, 20, 900, -5, 2 ** 31 - 1, -2 ** 31, 130]
    cu = _i32([wild[i % 8] for i in range(n + 1)])
    q = _randn(g, total, hq, D, dtype=dt)
    big = torch.full((total + 400, hq, D), 7.5, dtype=dt, device="cuda")
    bl = torch.full((total + 400, hq), 8.5, device="cuda")
    o, lse = big[200:200 + total], bl[200:200 + total]
    pages = tuple(torch.randint(0, 256, (20, hk, P, w), generator=g, device="cuda").to(torch.uint8) for w in (64, 64, 4, 4))
    table = torch.randint(-3, 25, (n, 9), generator=g, device="cuda").int()
    lens = torch.randint(-50, 400, (n,), generator=g, device="cuda").int()
    for add in (1, 200):
        pk.page4_attend(q, pages, table, cu, lens, add, out=o, lse=lse)
    torch.cuda.synchronize()
    for x, s in ((big, 7.5), (bl, 8.5)):
        assert bool((x[:200] == s).all()) and bool((x[200 + total:] == s).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("reqs,hq,hk", [([(40, 1)], 4, 2), ([(9000, 1), (5, 2)], 7, 1), ([(700, 150)], 6, 2), ([(12000, 40)], 4, 1)])
def test_page4_attend_in_the_prior_s_own_arrays_strided_without_lse(reqs, hq, hk, dtype):
    import torch
    log(f"case: page4 in place {reqs[:2]} heads {hq}/{hk} {dtype}")
    pk, g = PK(), _g(52)
    dt, P = _dt(dtype), 16
    need = [(c + a + P - 1) // P for c, a in reqs]
    width, count = max(need), sum(need)
    table = torch.full((len(reqs), width), -1, dtype=torch.int32, device="cuda")
    order = torch.randperm(count, generator=g, device="cuda")
    pages = pages4(count, hk, P)
    for i, n in enumerate(need):
        own = order[sum(need[:i]):sum(need[:i]) + n]
        table[i, :n] = own.int()
        held(g, pages, own, sum(reqs[i]), hk, P, dtype)
    add = [a for _, a in reqs]
    total = sum(add)
    cu, lens = _i32(np.cumsum([0] + add).tolist()), _i32([c + a for c, a in reqs])
    q, po = (_randn(g, total, hq, D, dtype=dt) for _ in range(2))
    pl = torch.randn(total, hq, generator=g, device="cuda") + 4
    want_o, want_l = pk.page4_attend(q, pages, table, cu, lens, max(add), prior=(po, pl))
    o, lse = po.clone(), pl.clone()
    pk.page4_attend(q, pages, table, cu, lens, max(add), prior=(o, lse), out=o, lse=lse)
    wide = torch.cat([q, q], dim=1)[:, :hq]   # rows at another stride
    o2, none = pk.page4_attend(wide, pages, table, cu, lens, max(add), prior=(po, pl), lse=False)
    torch.cuda.synchronize()
    assert torch.equal(o, want_o) and torch.equal(lse, want_l)
    assert none is False and torch.equal(o2, want_o)


# -- shared pages ---------------------------------------------------------------------


def fork_ref(ctx, src, dst, at, table, shares, stack, count, P):
    table, shares = [list(r) for r in table], list(shares)
    R, width, pages = len(ctx), len(table[0]), len(stack)
    count = min(max(count, 0), pages)
    cl = [min(max(c, 0), width * P) for c in ctx]
    fit = [0 <= s < R and 0 <= d < R and s != d for s, d in zip(src, dst)]
    sources = {s for s, f in zip(src, fit) if f}
    out, seen, asked, used, ctx_out = [], set(), 0, 0, list(ctx)
    before = [list(r) for r in table]
    for i, (s, d) in enumerate(zip(src, dst)):
        ok = fit[i] and d not in sources and d not in seen and ctx[d] <= 0
        if fit[i]:
            seen.add(d)
        n = (cl[s] if at is None else min(max(at[i], 0), cl[s])) if ok else 0
        need = n % P > 0
        asked += need
        if need and asked > count:
            ok = False
        if not ok:
            out.append((-1, -1, -1, 0))
            continue
        for j in range(n // P):
            table[d][j] = before[s][j]
            if 0 <= before[s][j] < pages:
                shares[before[s][j]] += 1
        a = b = -1
        if need:
            a, b = before[s][n // P], stack[count - asked]
            table[d][n // P] = b
            used += 1
        ctx_out[d] = n
        out.append((n, a, b, n % P))
    return table, shares, ctx_out, count - used, [list(x) for x in zip(*out)], sum(o[0] < 0 for o in out)


def release_ref(ctx, keep, table, shares, stack, count, P):
    shares, stack = list(shares), list(stack)
    width, pages = len(table[0]), len(stack)
    count = min(max(count, 0), pages)
    up = lambda x: -(-x // P)  # noqa: E731
    drops, out, refused = [0] * pages, [], 0
    for i, c in enumerate(ctx):
        c = min(max(c, 0), width * P)
        n = min(max(keep[i], 0), c)
        if n < c and n % P and 0 <= table[i][n // P] < pages and shares[table[i][n // P]] > 0:
            n = c
            refused += 1
        out.append(n)
        for p in table[i][up(n):up(c)]:
            if 0 <= p < pages:
                drops[p] += 1
    for p in range(pages):
        if drops[p] > shares[p]:
            shares[p] = 0
            if count < pages:
                stack[count] = p
                count += 1
        else:
            shares[p] -= drops[p]
    return out, shares, stack, count, refused


def _world(rng, R, width, P, pages, holders, shared=0.0):
    """Requests 0 .. holders - 1 hold pages, some of them in common; -> ctx, table, shares, stack, count"""
    ids = [int(x) for x in rng.permutation(pages)]
    ctx, table = [0] * R, [[-1] * width for _ in range(R)]
    owners = [0] * pages
    for r in range(holders):
        c = int(rng.integers(0, width * P + 1))
        first = 0
        if r and rng.random() < shared:
            o = int(rng.integers(0, r))
            first = min(ctx[o], c) // P
            table[r][:first] = table[o][:first]
        need = -(-c // P) - first
        if need > len(ids) - 2:
            continue
        for j in range(first, first + need):
            table[r][j] = ids.pop()
        ctx[r] = c
        for j in range(-(-c // P)):
            owners[table[r][j]] += 1
    return ctx, table, [max(o - 1, 0) for o in owners], ids + [-1] * (pages - len(ids)), len(ids)


def _fork_case(ctx, src, dst, at, table, shares, stack, count, P):
    import torch
    pk = PK()
    want = fork_ref(ctx, src, dst, at, table, shares, stack, count, P)
    t, s, f = _i32(table), _i32(shares), _i32(stack)
    r = pk.page_fork(_i32(ctx), _i32(src), _i32(dst), t, s, f, _i32([count]), P, at=None if at is None else _i32(at))
    torch.cuda.synchronize()
    assert r.ctx.tolist() == want[2] and r.count.tolist() == [want[3]] and r.refused.tolist() == [want[5]]
    assert [r.lens.tolist(), r.copy_src.tolist(), r.copy_dst.tolist(), r.copy_rows.tolist()] == want[4]
    assert t.tolist() == want[0] and s.tolist() == want[1] and f.tolist() == list(stack)
    return r, t, s, f


@pytest.mark.parametrize("seed", range(6))
def test_page_fork(seed):
    """Forks of any requests: of the same one, to taken rows, of rows that are none, at any length, with too few pages."""
    rng = np.random.default_rng(seed)
    R, P, width = [(3, 16, 5), (40, 1, 9), (40, 8, 300), (300, 16, 20), (8192, 2, 3), (2500, 32, 7)][seed]
    n = [2, 60, 25, 300, 8192, 1025][seed]
    log(f"case: page_fork {n} of {R} requests, pages of {P}")
    ctx, table, shares, stack, count = _world(rng, R, width, P, R * width, R // 3 + 1)
    src = [int(x) for x in rng.integers(0, R // 3 + 1, n)]
    dst = [int(x) for x in rng.integers(0, R, n)]
    at = [int(x) for x in rng.integers(-5, width * P + 9, n)] if seed % 2 else None
    _fork_case(ctx, src, dst, at, table, shares, stack, count, P)
    _fork_case(ctx, src, dst, at, table, shares, stack, count // 50, P)
    for i in range(0, n, 5):
        src[i] = [-1, R, 2 ** 31 - 1, -2 ** 31, dst[i]][(i // 5) % 5]
    for i in range(3, n, 7):
        dst[i] = [-4, R + 3, 2 ** 31 - 1][(i // 7) % 3]
    _fork_case(ctx, src, dst, at, table, shares, stack, count, P)


def test_page_fork_senseless_state_stays_inside():
    """Contexts, counts, tables and stacks of any value."""
    import torch
    log("case: page_fork of senseless state")
    rng = np.random.default_rng(9)
    R, P, width, pages, n = 50, 4, 6, 40, 60
    wild = lambda *s: rng.choice([-2 ** 31, -7, -1, 0, 1, 3, 17, 39, 40, 1000, 2 ** 31 - 1], s).tolist()  # noqa: E731
    for count in (-3, 10, 2 ** 31 - 1):
        ctx, table, stack = wild(R), wild(R, width), wild(pages)
        src, dst, at = rng.integers(-2, R + 2, n).tolist(), rng.integers(-2, R + 2, n).tolist(), wild(n)
        r, *_ = _fork_case(ctx, src, dst, at, table, [0] * pages, stack, count, P)
        x = torch.randn(pages, 2, P, 8, device="cuda")
        y = x.clone()
        PK().page_copy((x,), r.copy_src, r.copy_dst, r.copy_rows)   # pages that are none are passed over
        torch.cuda.synchronize()
        touched = {d for d in r.copy_dst.tolist() if 0 <= d < pages}
        rest = [p for p in range(pages) if p not in touched]
        assert torch.equal(x[rest], y[rest])


@pytest.mark.parametrize("seed", range(7))
def test_page_release(seed):
    rng = np.random.default_rng(100 + seed)
    R, P, width, pages = [(1, 16, 3, 5), (30, 1, 20, 400), (60, 16, 300, 9000), (1500, 8, 9, 8192), (8192, 2, 3, 14000),
                          (40, 1024, 5, 4097), (200, 4, 70, 50000)][seed]
    log(f"case: page_release {R} requests, pages of {P}, {pages} pages")
    for shared in (0.0, 0.7):
        ctx, table, shares, stack, count = _world(rng, R, width, P, pages, R, shared)
        keep = [int(rng.choice([0, c, c + 5, -3, rng.integers(0, c + 1), rng.integers(0, c + 1) // P * P])) for c in ctx]
        _release_case(ctx, keep, table, shares, stack, count, P)
        _release_case(ctx, [0] * R, table, shares, stack, count, P)


def _release_case(ctx, keep, table, shares, stack, count, P):
    import torch
    want = release_ref(ctx, keep, table, shares, stack, count, P)
    t, s, f = _i32(table), _i32(shares), _i32(stack)
    r = PK().page_release(_i32(ctx), _i32(keep), t, s, f, _i32([count]), P)
    torch.cuda.synchronize()
    assert r.ctx.tolist() == want[0] and r.count.tolist() == [want[3]] and r.refused.tolist() == [want[4]]
    assert s.tolist() == want[1] and f.tolist() == want[2] and t.tolist() == [list(x) for x in table]


def test_page_release_senseless_state_stays_inside():
    """Contexts, tables and counts of any value, pages dropped more often than held: each goes onto the stack once."""
    log("case: page_release of senseless state")
    rng = np.random.default_rng(10)
    R, P, width, pages = 50, 4, 6, 40
    for count in (-3, 25, 2 ** 31 - 1):
        wild = lambda *s: rng.choice([-2 ** 31, -7, -1, 0, 1, 3, 17, 39, 40, 1000, 2 ** 31 - 1], s).tolist()  # noqa: E731
        _release_case(wild(R), wild(R), wild(R, width), rng.integers(0, 5, pages).tolist(), wild(pages), count, P)


@pytest.mark.parametrize("hk,P,what", [(1, 1, "bf16"), (2, 16, "fp32"), (4, 16, "4bit"), (8, 64, "bf16"), (3, 1024, "4bit")])
def test_page_copy(hk, P, what):
    """Rows of pages, in several layers and arrays at once; pages that are none, and a page to itself, are passed over."""
    import torch
    log(f"case: page_copy heads {hk} page {P} {what}")
    pk, g = PK(), _g(61)
    pages, L = 23, 3
    if what == "4bit":
        arrays = [torch.randint(0, 256, (L, pages, hk, P, w), generator=g, device="cuda").to(torch.uint8) for w in (64, 64, 4, 4)]
    else:
        arrays = [_randn(g, L, pages, hk, P, D, dtype=_dt(what)) for _ in range(2)]
    arrays.append(torch.randint(0, 99, (pages, hk, P, 3), generator=g, device="cuda").int())   # one layer, rows of 12 bytes
    src, dst = [0, 5, 5, 7, -1, 9, 23, 11, 12], [1, 2, 3, 7, 4, 23, 6, 2 ** 31 - 1, 13]
    rows = [P, max(P // 2, 1), P + 7, P, P, P, P, P, 0]
    for given in (rows, None):
        mine = [x.clone() for x in arrays]
        pk.page_copy(mine, _i32(src), _i32(dst), None if given is None else _i32(given))
        torch.cuda.synchronize()
        for x, y in zip(mine, arrays):
            want = y.clone()
            for i, (a, b) in enumerate(zip(src, dst)):
                if 0 <= a < pages and 0 <= b < pages and a != b:
                    m = P if given is None else min(max(given[i], 0), P)
                    want[..., b, :, :m, :] = y[..., a, :, :m, :]
            assert torch.equal(x, want)


def test_pages_calls_without_rows():
    import torch
    log("case: no rows")
    pk = PK()
    k = torch.empty(0, 2, D, dtype=torch.bfloat16, device="cuda")
    pages = pages4(3, 2, 16)
    none = _i32([])
    pk.page4_store(k, k, pages, none)
    ko, vo = pk.page4_read(pages, none, torch.float32)
    assert ko.shape == vo.shape == (0, 2, D)
    q = torch.empty(0, 4, D, dtype=torch.bfloat16, device="cuda")
    for cu in (_i32([0]), _i32([0, 0])):
        n = cu.shape[0] - 1
        o, lse = pk.page4_attend(q, pages, torch.zeros(n, 2, dtype=torch.int32, device="cuda"), cu, _i32([5] * n), 1)
        assert o.shape == q.shape and lse.shape == (0, 4)
    pk.page_copy(pages, none, none)
    a, b = pk.norm_rotate(q, k, none, pk.pair_axes((64,)), 1e4, None, None, 1e-6)
    torch.cuda.synchronize()
    assert a.shape == q.shape and b.shape == k.shape
    assert all(bool((x == f).all()) for x, f in zip(pages, (0x77, 0x77, 255, 255)))


# -- together ---------------------------------------------------------------------------


def test_answers_forked_from_one_dialogue():
    """A question's dialogue in a cache of 4 bits is forked to several answers, which grow token by
    token and are dropped; each answers as a dialogue of its own would, and every page comes back."""
    import torch
    log("case: forked answers")
    pk, g = PK(), _g(71)
    hq, hk, P, L, R, width, pages = 8, 2, 16, 2, 6, 12, 50
    caches = [pages4(pages, hk, P) for _ in range(L)]
    table = torch.full((R, width), -1, dtype=torch.int32, device="cuda")
    stack, count = torch.randperm(pages, generator=g, device="cuda").int(), _i32([pages])
    shares, ctx = torch.zeros(pages, dtype=torch.int32, device="cuda"), torch.zeros(R, dtype=torch.int32, device="cuda")
    axes, w = pk.pair_axes((64,)), 1 + _randn(g, D, dtype=torch.bfloat16, scale=0.2)
    said = [[[] for _ in range(L)] for _ in range(R)]   # (k, v) values of each request's tokens

    def step(add):
        nonlocal count, ctx
        n = sum(add)
        p = pk.page_plan(ctx, _i32(add), table, stack, count, P, n)
        count = p.count
        for l in range(L):
            q = _randn(g, n, hq, D, dtype=torch.bfloat16, scale=2.0)
            k, v = (_randn(g, n, hk, D, dtype=torch.bfloat16) for _ in range(2))
            qr, kr = pk.norm_rotate(q, k, p.positions, axes, 1e4, w, w, 1e-6)
            pk.page4_store(kr, v, caches[l], p.slots)
            o, lse = pk.page4_attend(qr, caches[l], table, p.cu, p.kv_len, max(add))
            kh, vh = pk.page4_read(caches[l], p.slots, torch.bfloat16)
            torch.cuda.synchronize()
            at = 0
            for r, a in enumerate(add):
                said[r][l] += [(kh[t], vh[t]) for t in range(at, at + a)]
                if a:
                    K, V = (torch.stack([x[j] for x in said[r][l]]) for j in (0, 1))
                    m = K.shape[0]
                    seen = torch.arange(m, device="cuda")[None] <= (m - a + torch.arange(a, device="cuda"))[:, None]
                    for h in range(hq):
                        ref = attend64(qr[at:at + a, h], K[:, h // 4], V[:, h // 4], seen)
                        check(o[at:at + a, h], lse[at:at + a, h], ref, m, torch.bfloat16, None, f"request {r}, layer {l}, head {h}")
                at += a
        ctx = ctx + _i32(add)

    step([37, 0, 20, 0, 0, 0])
    f = pk.page_fork(ctx, _i32([0, 0, 2, 0]), _i32([1, 3, 4, 5]), table, shares, stack, count, P, at=_i32([99, 99, 99, 18]))
    for cache in caches:
        pk.page_copy(cache, f.copy_src, f.copy_dst, f.copy_rows)
    assert f.lens.tolist() == [37, 37, 20, 18] and f.refused.tolist() == [0]
    ctx, count = f.ctx, f.count
    for s, d, n in ((0, 1, 37), (0, 3, 37), (2, 4, 20), (0, 5, 18)):
        said[d] = [list(said[s][l][:n]) for l in range(L)]
    assert int(shares.sum()) == 2 + 2 + 1 + 1
    for _ in range(3):
        step([0, 1, 1, 1, 1, 0])
    step([3, 20, 0, 1, 1, 40])
    # answer 3 goes back to its fork's end, in pages of its own; request 0 may not end inside a page it shares
    r = pk.page_release(ctx, _i32([18, 0, 99, 37, 0, 99]), table, shares, stack, count, P)
    assert r.refused.tolist() == [1] and r.ctx.tolist() == [40, 0, 23, 37, 0, 58]
    ctx, count = r.ctx, r.count
    said[1], said[4] = [[] for _ in range(L)], [[] for _ in range(L)]
    said[3] = [said[3][l][:37] for l in range(L)]
    step([1, 25, 1, 1, 0, 2])
    r = pk.page_release(ctx, _i32([0] * R), table, shares, stack, count, P)
    torch.cuda.synchronize()
    assert r.count.tolist() == [pages] and sorted(stack.tolist()) == list(range(pages))
    assert r.ctx.tolist() == [0] * R and not bool(shares.any())


def _serving(g, R, width, P, pages, most, hq, hk):
    import torch
    i32 = dict(dtype=torch.int32, device="cuda")
    st = {"ctx": torch.zeros(R, **i32), "add": torch.zeros(R, **i32), "keep": torch.zeros(R, **i32),
          "src": torch.full((4,), -1, **i32), "dst": torch.full((4,), -1, **i32),
          "table": torch.full((R, width), -1, **i32), "stack": torch.randperm(pages, generator=g, device="cuda").int(),
          "count": _i32([pages]), "shares": torch.zeros(pages, **i32),
          "qkv": torch.zeros(most, (hq + 2 * hk) * D, dtype=torch.bfloat16, device="cuda")}
    for name, x in zip("kvst", pages4(pages, hk, P)):
        st["p" + name] = x
    return st


def _serve(st, w, hq, hk, P, most, max_add):
    """Forks, a step of new tokens, releases: every length and number on the device."""
    pk = PK()
    cache = (st["pk"], st["pv"], st["ps"], st["pt"])
    f = pk.page_fork(st["ctx"], st["src"], st["dst"], st["table"], st["shares"], st["stack"], st["count"], P)
    pk.page_copy(cache, f.copy_src, f.copy_dst, f.copy_rows)
    q, k, v = (x.unflatten(1, (-1, D)) for x in st["qkv"].split([hq * D, hk * D, hk * D], dim=1))
    p = pk.page_plan(f.ctx, st["add"], st["table"], st["stack"], f.count, P, most)
    qr, kr = pk.norm_rotate(q, k, p.positions, pk.pair_axes((64,)), 1e4, w, w, 1e-6)
    pk.page4_store(kr, v, cache, p.slots)
    o, lse = pk.page4_attend(qr, cache, st["table"], p.cu, p.kv_len, max_add)
    r = pk.page_release(p.kv_len, st["keep"], st["table"], st["shares"], st["stack"], p.count, P)
    st["ctx"].copy_(r.ctx)
    st["count"].copy_(r.count)
    return o, lse, f.lens, p.slots, r.ctx


@pytest.mark.parametrize("max_add", [1, 40])
def test_serving_captured_and_eager(max_add):
    """The same rounds through a captured graph, replayed with eager work in between, and eagerly on
    a state of their own: the same bits in results, pages, tables and counts."""
    import torch
    log(f"case: serving, eager and captured, max_add {max_add}")
    R, width, P, pages, hq, hk = 6, 20, 8, 90, 6, 2
    most = R * max_add
    g = _g(81)
    w = 1 + _randn(g, D, dtype=torch.bfloat16, scale=0.2)
    a, b = (_serving(_g(82), R, width, P, pages, most, hq, hk) for _ in range(2))
    args = (w, hq, hk, P, most, max_add)
    warm = _serving(_g(82), R, width, P, pages, most, hq, hk)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _serve(warm, *args)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _serve(b, *args)
    for x in b:   # the capture ran nothing
        assert torch.equal(a[x], b[x]), x
    rng = np.random.default_rng(83)
    for turn in range(12):
        ctx = a["ctx"].tolist()
        empty = [r for r in range(R) if ctx[r] == 0]
        full = [r for r in range(R) if ctx[r] > 0]
        src, dst = [-1] * 4, [-1] * 4
        for i in range(min(len(empty) - 1, 4) if full else 0):
            src[i], dst[i] = int(rng.choice(full)), empty[i]
        add = [int(rng.integers(0, max_add + 1)) for _ in range(R)]
        now = [c + x for c, x in zip(ctx, add)]
        keep = [0 if rng.random() < 0.2 or now[r] > 100 else 10 ** 6 for r in range(R)]
        qkv = _randn(g, most, (hq + 2 * hk) * D, dtype=torch.bfloat16)
        for st in (a, b):
            st["qkv"].copy_(qkv)
            for name, x in (("add", add), ("keep", keep), ("src", src), ("dst", dst)):
                st[name].copy_(_i32(x))
        torch.cuda.synchronize()
        want = _serve(a, *args)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        n = sum(add)
        assert torch.equal(want[0][:n], got[0][:n]) and torch.equal(want[1][:n], got[1][:n]), f"turn {turn}"
        for x, y in zip(want[2:], got[2:]):
            assert torch.equal(x, y), f"turn {turn}"
        for x in a:
            assert torch.equal(a[x], b[x]), f"turn {turn}: {x}"


def test_pages_calls_on_streams_of_their_own():
    """Two streams at once, each call with its own results and workspace, against the same calls alone."""
    import torch
    log("case: two streams")
    pk, g = PK(), _g(91)
    hq, hk, P, n = 28, 4, 16, 6000
    made = []
    for add in (1, 60):
        pages = pages4(400, hk, P)
        own = torch.randperm(400, generator=g, device="cuda")
        held(g, pages, own, n, hk, P, "bf16")
        qkv = _randn(g, add, (hq + hk) * D, dtype=torch.bfloat16)
        made.append((qkv[:, :hq * D].unflatten(1, (-1, D)), qkv[:, hq * D:].unflatten(1, (-1, D)), pages, own.int()[:380].view(1, 380),
                     add, torch.arange(n, n + add, device="cuda").int(), own[375 + torch.arange(add, device="cuda") // P].int() * P
                     + torch.arange(add, device="cuda").int() % P))
    axes = pk.pair_axes((64,))

    def calls(q, k, pages, table, add, pos, slots, stream=None):
        qr, kr = pk.norm_rotate(q, k, pos, axes, 1e4, None, None, 1e-6, stream=stream)
        pk.page4_store(kr, kr, pages, slots, stream=stream)
        o, lse = pk.page4_attend(qr, pages, table, _i32_on(stream, [0, add]), _i32_on(stream, [n + add]), add, stream=stream)
        return (o, lse, *pk.page4_read(pages, slots, torch.float32, stream=stream))

    def _i32_on(stream, v):
        if stream is None:
            return _i32(v)
        with torch.cuda.stream(stream):
            return _i32(v)

    alone = [calls(*m) for m in made]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in made]
    for _ in range(5):
        both = [calls(*m, stream=s) for m, s in zip(made, streams)]
        torch.cuda.synchronize()
        for x, y in zip(both, alone):
            assert all(torch.equal(a, b) for a, b in zip(x, y))
