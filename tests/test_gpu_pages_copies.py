"""GPU: copies of pages in numbers that a fork can ask for, and arrays whose rows are no multiple of 16
bytes.  Each test prints its case before any GPU step."""
import pytest

from tests.test_gpu_exact import PK, _g, _gpu, _i32, log  # noqa: F401

pytestmark = pytest.mark.gpu


def _copied(x, src, dst, rows):
    want = x.clone()
    for a, b, m in zip(src, dst, rows):
        if 0 <= a < x.shape[-4]:
            want[..., b, :, :m, :] = x[..., a, :, :m, :]
    return want


@pytest.mark.parametrize("layers,pages,hk,P,row,real", [
    # 8192 x 160 pages of 256 KB: 16 workgroups to a page would be more than a launch has
    (160, 8, 8, 128, 256, (0, 5000, 8191)),
    # 8192 x 4000 pages of 64 bytes: two launches, of 4194 copies and the rest
    (4000, 12, 1, 4, 16, (0, 4192, 4193, 4194, 8191))])
def test_page_copy_of_a_fork_s_most(layers, pages, hk, P, row, real):
    """8192 copies, most of them none, as refused forks leave them."""
    import torch
    log(f"case: page_copy of 8192 in {layers} layers")
    pk, g = PK(), _g(71)
    x = torch.randint(0, 256, (layers, pages, hk, P, row), generator=g, device="cuda", dtype=torch.uint8)
    src, dst, rows = [-1] * 8192, [-1] * 8192, [0] * 8192
    for j, i in enumerate(real):
        src[i], dst[i], rows[i] = j, pages - 1 - j, P - j
    want = _copied(x, src, dst, rows)
    pk.page_copy([x], _i32(src), _i32(dst), _i32(rows))
    torch.cuda.synchronize()
    assert torch.equal(x, want)


def test_page_copy_of_more_than_a_fork_s_most():
    """As many copies as one launch takes with one workgroup to a page, and the first number that it does not."""
    import torch
    log("case: page_copy of 2^22 - 1")
    pk, n = PK(), (1 << 22) - 1
    x = torch.arange(4 * 6 * 16 * 64, device="cuda", dtype=torch.int32).view(4, 6, 1, 16, 64)
    src, dst = (torch.full((n + 1,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    src[0], dst[0], src[n - 1], dst[n - 1] = 0, 5, 1, 4
    want = _copied(x, [0, 1], [5, 4], [16, 16])
    with pytest.raises(pk.ProtoKVError, match="8192 copies"):
        pk.page_copy([x], src, dst)
    pk.page_copy([x], src[:n], dst[:n])
    torch.cuda.synchronize()
    assert torch.equal(x, want)


@pytest.mark.parametrize("layers,pages,hk,P,row", [(3, 7, 1, 1, 4), (5, 9, 1, 2, 4), (2, 5, 3, 1, 12), (4, 3, 1, 1, 20)])
def test_page_copy_of_rows_that_are_no_multiple_of_16(layers, pages, hk, P, row):
    """Scales of pages of one or two tokens: layers that do not begin at multiples of 16 bytes, in one array, each
    by itself, and beside an array of 64-byte rows."""
    import torch
    log(f"case: page_copy of {layers} layers of {pages} pages of {hk} x {P} rows of {row}")
    pk, g = PK(), _g(72)
    src, dst, rows = [0, 2, -1], [1, pages - 1, 0], [P, P, P]
    x = torch.randint(0, 256, (layers, pages, hk, P, row), generator=g, device="cuda", dtype=torch.uint8)
    y = torch.randint(0, 256, (layers, pages, hk, P, 64), generator=g, device="cuda", dtype=torch.uint8)
    want = [_copied(t, src, dst, rows) for t in (x, y)]
    a, b = x.clone(), x.clone()
    pk.page_copy([a, y], _i32(src), _i32(dst))
    for layer in b:
        pk.page_copy([layer], _i32(src), _i32(dst), _i32(rows))
    torch.cuda.synchronize()
    assert torch.equal(a, want[0]) and torch.equal(b, want[0]) and torch.equal(y, want[1])
