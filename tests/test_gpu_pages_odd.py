"""GPU: attention over pages of 4 bits that hold scale bytes which page4_store does not write.

With s = 253 the codes 4 and 6 are 2^128 and more, with s = 254 those from 2 on: infinities, as
protokv_page4_read returns them (tests/test_gpu_pages.py reads every byte).  What a row does not see must
reach nothing: later tokens, and page 0, which is read in the place of an entry outside the pages.  What it
sees is added: an infinity stays one, whether its key is the last, which a tile's end repeats, or not.
Tolerances of the finite outputs are tests/test_gpu_exact.py's, where float32 holds their sums: a weight
2^(s - m) is at most 2^8, as the reference m follows a row's largest score when that is 8 above it, so that n
products w v and all their partial sums stay below 2^8 n max|v|, below 2^127 for |v| <= 2^119 / n.  A
row that sees a larger finite value (2^125 to 1.5 * 2^127 here, beside the infinities) may have any value in that dim.
"""
import math

import numpy as np
import pytest

from tests.test_gpu_exact import D, PK, _dt, _g, _gpu, _i32, _randn, attend64, check, log  # noqa: F401
from tests.test_gpu_pages import held, pages4

pytestmark = pytest.mark.gpu

# at most 16 rows per kv head, one wave's and shared; 17 to 32; more, in groups of 32, whole and shared,
# and in row blocks, whole and split
SHAPES = [([(300, 1), (70, 1)], 4, 2), ([(300, 4)], 6, 2), ([(5000, 3), (200, 2)], 10, 2), ([(300, 20), (90, 3)], 2, 2),
          ([(4000, 8)], 4, 1), ([(130, 16)] * 64, 14, 2), ([(700, 150)], 6, 2), ([(300, 100)], 28, 4), ([(700, 700)], 28, 4)]


def _odd(reqs, hq, hk, scale, dtype, keys, bad, flip=0):
    """keys(ctx, add): the tokens of each request whose values get the scale byte, one in block 2 of kv head 0, the
    next in block 0 of the last.  bad: table entries of each request that are no page.  flip: the signs of every other one of a block."""
    import torch
    pk, g, P = PK(), _g(scale), 16
    dt = _dt(dtype)
    kv = [c + a for c, a in reqs]
    need = [(n + P - 1) // P for n in kv]
    pages = pages4(sum(need) + 1, hk, P, fill=scale)   # page 0 is nobody's
    pages[0][:, :, ::2] = 0xE5                          # of either sign
    order = 1 + torch.randperm(sum(need), generator=g, device="cuda")
    table = torch.full((len(reqs), max(need)), -1, dtype=torch.int32, device="cuda")
    at, rows = 0, []
    for i, n in enumerate(need):
        own = order[at:at + n]
        at += n
        table[i, :n] = own.int()
        held(g, pages, own, kv[i], hk, P, dtype)
        for j, x in enumerate(keys(*reqs[i])):
            h, b = (0, 2) if j % 2 == 0 else (hk - 1, 0)
            pages[3][own[x // P], h, x % P, b] = scale
            pages[1][own[x // P], h, x % P, 16 * b:16 * b + 16] = (torch.arange(16, device="cuda").to(torch.uint8) * 17) ^ (
                flip if j // 2 % 2 else 0)
        m = torch.arange(kv[i], device="cuda")
        rows.append(tuple(y.transpose(0, 1) for y in pk.page4_read(pages, (own[m // P] * P + m % P).int(), dt)))
    for i in range(len(reqs)):
        for j, p in enumerate(bad):
            table[i, p] = [-1, sum(need) + 1, 2 ** 31 - 1][(i + j) % 3]
    add = [a for _, a in reqs]
    q = _randn(g, sum(add), hq, D, dtype=dt, scale=2.0)
    o, lse = pk.page4_attend(q, pages, table, _i32(np.cumsum([0] + add).tolist()), _i32(kv), max(add))
    torch.cuda.synchronize()
    at, infinite = 0, 0
    for i, (ctx, a) in enumerate(reqs):
        k, v = rows[i]
        key = torch.arange(kv[i], device="cuda")
        here = torch.tensor([x // P not in bad for x in range(kv[i])], device="cuda")
        seen = (key[None] <= ctx + torch.arange(a, device="cuda")[:, None]) & here[None]
        for h in range(hq):
            kh, vh = k[h // (hq // hk)], v[h // (hq // hk)]
            k_seen = torch.where(here[:, None], kh, 0)
            up, down = (seen.double() @ ((vh == x) & here[:, None]).double() > 0 for x in (math.inf, -math.inf))
            got, what = o[at:at + a, h], f"request {i} {reqs[i]}, head {h}"
            want = torch.where(up & down, math.nan, torch.where(up, math.inf, -math.inf)).to(got.dtype)
            far = seen.double() @ (vh.isfinite() & (vh.double().abs() > 2.0 ** 119 / kv[i]) & here[:, None]).double() > 0
            hit = (up | down) & ~far
            assert torch.equal(got[~far].isnan(), (up & down)[~far]), what
            assert torch.equal(got[hit].nan_to_num(0.0), want[hit].nan_to_num(0.0)), what
            infinite += int(hit.sum())
            ref = attend64(q[at:at + a, h], k_seen, torch.where(vh.isfinite() & here[:, None], vh, 0), seen)
            wo, wl, A, e, s = ref
            clean = torch.where(hit | far, wo.to(got.dtype), got)
            check(clean, lse[at:at + a, h], ref, kv[i], dt, None, what)
        at += a
    return infinite


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [253, 254])
@pytest.mark.parametrize("reqs,hq,hk", SHAPES)
def test_page4_attend_infinite_values_reach_the_rows_that_see_them(reqs, hq, hk, scale, dtype):
    """Of a new token in the middle and of the last one, which stands at a tile's end once more."""
    log(f"case: page4 infinite values {reqs[:3]} heads {hq}/{hk} scale {scale} {dtype}")
    assert _odd(reqs, hq, hk, scale, dtype, lambda c, a: sorted({c + a // 2, c + a - 1}), ()) > 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [253, 254, 255])
@pytest.mark.parametrize("reqs,hq,hk", SHAPES)
def test_page4_attend_page_0_stands_for_no_page(reqs, hq, hk, scale, dtype):
    log(f"case: page4 page 0 odd {reqs[:3]} heads {hq}/{hk} scale {scale} {dtype}")
    assert _odd(reqs, hq, hk, scale, dtype, lambda c, a: (), (0, 1, 3)) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("reqs,hq,hk", SHAPES)
def test_page4_attend_infinite_values_and_pages_that_are_none(reqs, hq, hk, dtype):
    """A token on a page whose entry is none, one in the context that every row sees, and the last one."""
    log(f"case: page4 infinite values, entries outside {reqs[:3]} heads {hq}/{hk} {dtype}")
    assert _odd(reqs, hq, hk, 254, dtype, lambda c, a: (20, 40, c + a - 1), (1, 3)) > 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("reqs,hq,hk", SHAPES)
def test_page4_attend_infinite_values_of_both_signs_give_nan(reqs, hq, hk, dtype):
    """A row that sees +inf and -inf in a dim has NaN there, one that sees only the first keeps it."""
    log(f"case: page4 infinite values of both signs {reqs[:3]} heads {hq}/{hk} {dtype}")
    assert _odd(reqs, hq, hk, 253, dtype, lambda c, a: (8, 40, c + a // 2, c + a - 1), (), flip=0x88) > 0
