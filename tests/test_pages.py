"""CPU: the calls around a paged dialogue (head norms with the rotation, pages of 4
bits, shared pages) refuse what they cannot do before anything is launched, and say
why.  No GPU is touched: every call below is refused on the host."""
import ctypes

import pytest
import torch

from paper_2606_26762_amd import protokv as pk

GOOD = 1 << 20   # an aligned address; refused calls never read it


def _status(name, *args):
    return getattr(pk.lib(), "protokv_" + name)(*[ctypes.byref(a) for a in args], None)


def _set(a, **kw):
    for f, v in kw.items():
        head, _, rest = f.partition("__")
        setattr(getattr(a, head) if rest else a, rest or head, v)
    return a


def rotation(**kw):
    a = pk.RotateArgs(num_tokens=3, num_q_heads=8, num_kv_heads=2, head_dim=128, kv_dtype=pk.KV_BF16, num_axes=3,
                      positions=GOOD, position_stride=3, axes=pk.pair_axes((16, 24, 24)), theta=1e6, q=GOOD, k=GOOD,
                      q_stride=1024, k_stride=256, q_out=GOOD, k_out=GOOD, q_out_stride=1024, k_out_stride=256)
    return _set(a, **kw)


@pytest.mark.parametrize("kw,norm,status", [
    (dict(), dict(eps=-1e-6), 1), (dict(), dict(eps=float("nan")), 1), (dict(), dict(eps=float("inf")), 1),
    (dict(), dict(q_weight=GOOD + 8), 1), (dict(), dict(k_weight=GOOD + 2), 1), (dict(head_dim=64), {}, 2),
    (dict(num_q_heads=7), {}, 1), (dict(theta=1.0), {}, 1), (dict(q_stride=1020), {}, 1), (dict(q=None, q_out=None, k=None, k_out=None), {}, 1),
    (dict(num_tokens=1 << 27), {}, 2)])
def test_norm_rotate_refuses(kw, norm, status):
    assert _status("norm_rotate", rotation(**kw), _set(pk.HeadNorm(GOOD, GOOD, 1e-6), **norm)) == status
    assert b"norm_rotate: " in pk.lib().protokv_last_error(None)


def rows(**kw):
    a = pk.Page4RowsArgs(5, 2, 128, pk.KV_BF16, GOOD, GOOD + 65536, 256, 256, GOOD, pk.Pages4(*[GOOD + 4096 * i for i in range(4)], 10, 16))
    return _set(a, **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(num_tokens=-1), 1), (dict(num_kv_heads=0), 1), (dict(head_dim=64), 2), (dict(kv_dtype=2), 1), (dict(k=None), 1),
    (dict(v=GOOD + 8), 1), (dict(k_stride=255), 1), (dict(v_stride=260), 1), (dict(slots=None), 1), (dict(slots=GOOD + 2), 1),
    (dict(pages__num_pages=0), 1), (dict(pages__page_size=12), 2), (dict(pages__page_size=2048), 2),
    (dict(pages__num_pages=1 << 27), 2), (dict(pages__k=None), 1), (dict(pages__v=GOOD + 8), 1),
    (dict(pages__k_scale=None), 1), (dict(pages__v_scale=GOOD + 2), 1), (dict(num_tokens=1 << 27), 2),
    (dict(num_kv_heads=512, k_stride=65536, v_stride=65536, pages__num_pages=1 << 20), 2)])
def test_page4_rows_refuse(kw, status):
    for name in ("page4_store", "page4_read"):
        assert _status(name, rows(**kw)) == status
        assert name.encode() + b": " in pk.lib().protokv_last_error(None)


def test_page4_store_and_read_refuse_one_array_for_both():
    assert _status("page4_store", rows(pages__v=GOOD)) == 1
    assert _status("page4_store", rows(pages__v_scale=GOOD + 8192)) == 1
    assert _status("page4_read", rows(v=GOOD)) == 1


def attend(**kw):
    a = pk.Page4AttendArgs(8, 2, 128, pk.KV_BF16, 2, 40, 30, 64, GOOD, GOOD, GOOD, GOOD, 1024,
                           pk.Pages4(GOOD, GOOD, GOOD, GOOD, 100, 16), GOOD, GOOD, None, None, GOOD, 1 << 40)
    return _set(a, **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(num_q_heads=9), 1), (dict(head_dim=64), 2), (dict(kv_dtype=-1), 1), (dict(num_requests=-1), 1),
    (dict(total=-5), 1), (dict(total=1 << 28), 2), (dict(max_add=0), 1), (dict(table_stride=0), 1),
    (dict(table_stride=1 << 27), 1), (dict(cu=None), 1), (dict(kv_len=None), 1), (dict(kv_len=GOOD + 1), 1),
    (dict(table=None), 1), (dict(q=None), 1), (dict(q_stride=1000), 1), (dict(pages__page_size=0), 2),
    (dict(pages__page_size=48), 2), (dict(pages__num_pages=0), 1), (dict(pages__num_pages=1 << 27), 2),
    (dict(pages__k=None), 1), (dict(pages__v=GOOD + 2), 1), (dict(pages__k_scale=GOOD + 1), 1),
    (dict(pages__v_scale=None), 1), (dict(o=None), 1), (dict(prior_o=GOOD), 1), (dict(workspace=None), 3),
    (dict(workspace=GOOD + 16), 3), (dict(workspace_bytes=1000), 3), (dict(num_requests=1 << 23, max_add=100), 2)])
def test_page4_attend_refuses(kw, status):
    assert _status("page4_attend", attend(**kw)) == status
    assert b"page4_attend: " in pk.lib().protokv_last_error(None)


def test_page4_attend_workspace_goes_by_sizes_alone():
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    L = pk.lib()
    assert L.protokv_page4_attend_workspace(ctypes.byref(attend()), ctypes.byref(n)) == 0
    assert L.protokv_page4_attend_workspace(ctypes.byref(attend(cu=None, q=None, o=None, workspace=None, pages__k=None)),
                                            ctypes.byref(m)) == 0
    assert 0 < n.value == m.value < 1 << 28
    for kw, some in ((dict(max_add=1, table_stride=16), False), (dict(max_add=1, table_stride=17), True)):
        assert L.protokv_page4_attend_workspace(ctypes.byref(attend(**kw)), ctypes.byref(n)) == 0
        assert (n.value > 0) == some   # up to 256 tokens a wave needs no other
    assert L.protokv_page4_attend_workspace(ctypes.byref(attend(head_dim=64)), ctypes.byref(n)) == 2
    assert L.protokv_page4_attend_workspace(None, ctypes.byref(n)) == 1
    assert L.protokv_page4_attend_workspace(ctypes.byref(attend()), None) == 1


def fork(**kw):
    return _set(pk.PageForkArgs(4, 20, 100, 16, 8, *[GOOD + 4096 * i for i in range(15)]), **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(num_forks=0), 1), (dict(num_forks=8193), 2), (dict(num_requests=0), 1), (dict(num_requests=8193), 2),
    (dict(num_pages=0), 1), (dict(page_size=24), 2), (dict(num_pages=1 << 27), 2), (dict(page_size=1, num_pages=(1 << 29) + 1), 2),
    (dict(table_stride=0), 1), (dict(table_stride=1 << 27), 1), (dict(ctx=None), 1), (dict(src=None), 1), (dict(dst=GOOD + 1), 1),
    (dict(at=GOOD + 2), 1), (dict(table=None), 1), (dict(shares=None), 1), (dict(free_pages=None), 1), (dict(free_count=None), 1),
    (dict(free_count_out=None), 1), (dict(ctx_out=None), 1), (dict(lens=None), 1), (dict(copy_src=None), 1),
    (dict(copy_dst=None), 1), (dict(copy_rows=None), 1), (dict(refused=GOOD + 3), 1), (dict(ctx_out=GOOD), 1),
    (dict(free_count_out=GOOD + 4096 * 7), 1), (dict(lens=GOOD + 4096), 1), (dict(copy_src=GOOD + 4096 * 12), 1),
    (dict(shares=GOOD + 4096 * 4), 1), (dict(refused=GOOD + 4096 * 10), 1)])
def test_page_fork_refuses(kw, status):
    assert _status("page_fork", fork(**kw)) == status
    assert b"page_fork: " in pk.lib().protokv_last_error(None)


def release(**kw):
    return _set(pk.PageReleaseArgs(4, 100, 16, 8, *[GOOD + 4096 * i for i in range(10)]), **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(num_requests=0), 1), (dict(num_requests=8193), 2), (dict(num_pages=0), 1), (dict(page_size=24), 2),
    (dict(num_pages=1 << 27), 2), (dict(page_size=1, num_pages=(1 << 29) + 1), 2), (dict(table_stride=0), 1),
    (dict(table_stride=1 << 27), 1), (dict(ctx=None), 1), (dict(keep=None), 1), (dict(table=GOOD + 2), 1), (dict(shares=None), 1),
    (dict(free_pages=None), 1), (dict(free_count=None), 1), (dict(free_count_out=None), 1), (dict(ctx_out=None), 1),
    (dict(refused=None), 1), (dict(scratch=None), 1), (dict(ctx_out=GOOD), 1), (dict(free_count_out=GOOD + 4096 * 5), 1),
    (dict(scratch=GOOD + 4096 * 8), 1), (dict(ctx_out=GOOD + 4096), 1)])
def test_page_release_refuses(kw, status):
    assert _status("page_release", release(**kw)) == status
    assert b"page_release: " in pk.lib().protokv_last_error(None)


def copies(first=None, **kw):
    each = (pk.PageArray * 2)(pk.PageArray(GOOD, 256, 1, 0), pk.PageArray(GOOD, 4, 3, 1 << 20))
    _set(each[1], **(first or {}))
    a = _set(pk.PageCopyArgs(4, 2, 100, 16, 2, each, GOOD, GOOD, GOOD), **kw)
    a.keep = each
    return a


@pytest.mark.parametrize("first,kw,status", [
    ({}, dict(num_copies=-1), 1), ({}, dict(num_kv_heads=0), 1), ({}, dict(num_kv_heads=65537), 1), ({}, dict(num_pages=0), 1),
    ({}, dict(page_size=20), 2), ({}, dict(num_arrays=0), 1), ({}, dict(num_arrays=129), 1), ({}, dict(arrays=None), 1),
    ({}, dict(src=None), 1), ({}, dict(dst=GOOD + 2), 1), ({}, dict(rows=GOOD + 1), 1), (dict(base=None), {}, 1),
    (dict(base=GOOD + 8), {}, 1), (dict(row_bytes=6), {}, 1), (dict(row_bytes=0), {}, 1), (dict(row_bytes=4100), {}, 1),
    (dict(layers=0), {}, 1), (dict(layers=70000), {}, 2), (dict(layer_stride=12000), {}, 1), (dict(layer_stride=(1 << 20) + 8), {}, 1),
    ({}, dict(num_kv_heads=65536, page_size=1024), 2), ({}, dict(num_copies=1 << 23), 2)])
def test_page_copy_refuses(first, kw, status):
    assert _status("page_copy", copies(first, **kw)) == status
    assert b"page_copy: " in pk.lib().protokv_last_error(None)


def test_null_arguments_are_refused():
    L = pk.lib()
    for name in ("page4_store", "page4_read", "page4_attend", "page_fork", "page_copy", "page_release"):
        assert getattr(L, "protokv_" + name)(None, None) == 1
    assert L.protokv_norm_rotate(None, ctypes.byref(pk.HeadNorm(None, None, 0.0)), None) == 1
    assert L.protokv_norm_rotate(ctypes.byref(rotation()), None, None) == 1


def test_empty_calls_are_done_at_once():
    """Nothing to do is no error, and nothing is launched; empty tensors may have no address."""
    assert _status("norm_rotate", rotation(num_tokens=0, positions=None), pk.HeadNorm(None, None, 0.0)) == 0
    for name in ("page4_store", "page4_read"):
        assert _status(name, rows(num_tokens=0, k=None, v=None, slots=None)) == 0
    for kw in (dict(num_requests=0), dict(total=0)):
        assert _status("page4_attend", attend(**kw)) == 0
    assert _status("page_copy", copies(num_copies=0, src=None, dst=None)) == 0


# -- the binding, whose calls launch nothing here ------------------------------------


@pytest.fixture
def host(monkeypatch):
    """Host tensors pass as those of the current device; -> the statuses checked."""
    monkeypatch.setattr(pk, "_device", lambda t, stream: -1)
    monkeypatch.setattr(pk, "_raw_stream", lambda stream, dev: None)
    done = []
    monkeypatch.setattr(pk, "_check", lambda status: done.append(status))

    class Library:
        def __getattr__(self, call):
            return lambda *a: 0
    monkeypatch.setattr(pk, "lib", Library)
    return done


def _calls(**leaf):
    """Each call that takes floating-point tensors, with those named in `leaf` in place of its own."""
    t = dict(q=torch.zeros(4, 8, 128), k=torch.zeros(4, 2, 128), v=torch.zeros(4, 2, 128), q_norm=torch.ones(128),
             k_norm=torch.ones(128), out=torch.zeros(4, 8, 128), k_out=torch.zeros(4, 2, 128), v_out=torch.zeros(4, 2, 128),
             prior_o=torch.zeros(4, 8, 128), pages=torch.zeros(3, 2, 16, 128))
    t.update(leaf)
    i32 = dict(dtype=torch.int32)
    four = tuple(torch.zeros(3, 2, 16, n, dtype=torch.uint8) for n in (64, 64, 4, 4))
    slots, cu, one = torch.zeros(4, **i32), torch.tensor([0, 4], **i32), torch.tensor([20], **i32)
    uses = {
        "norm_rotate": ("q k q_norm k_norm out", lambda: pk.norm_rotate(
            t["q"], t["k"], slots, pk.pair_axes((64,)), 1e4, t["q_norm"], t["k_norm"], 1e-6, q_out=t["out"])),
        "page4_store": ("k v", lambda: pk.page4_store(t["k"], t["v"], four, slots)),
        "page4_read": ("k_out v_out", lambda: pk.page4_read(four, slots, torch.float32, k_out=t["k_out"], v_out=t["v_out"])),
        "page4_attend": ("q out prior_o", lambda: pk.page4_attend(
            t["q"], four, torch.zeros(1, 3, **i32), cu, one, 4, out=t["out"], prior=(t["prior_o"], torch.zeros(4, 8)))),
        "page_copy": ("pages", lambda: pk.page_copy((t["pages"],), one, one))}
    return [f for names, f in uses.values() if set(leaf) <= set(names.split())]


@pytest.mark.parametrize("name", ["q", "k", "v", "q_norm", "k_norm", "out", "k_out", "v_out", "prior_o", "pages"])
def test_binding_refuses_what_a_gradient_is_asked_of(name, host):
    """The results would carry none; with gradients off, the same tensors are only values."""
    shape = dict(q=(4, 8, 128), out=(4, 8, 128), prior_o=(4, 8, 128), q_norm=(128,), k_norm=(128,), pages=(3, 2, 16, 128)).get(
        name, (4, 2, 128))
    calls = _calls(**{name: torch.zeros(*shape, requires_grad=True)})
    assert calls
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
    assert not host
    with torch.no_grad():
        for call in calls:
            call()
    assert len(host) >= len(calls)


def test_binding_refuses_wrong_shapes_and_types(host):
    i32 = dict(dtype=torch.int32)
    k, slots = torch.zeros(4, 2, 128), torch.zeros(4, **i32)
    four = tuple(torch.zeros(3, 2, 16, n, dtype=torch.uint8) for n in (64, 64, 4, 4))
    bad = [
        lambda: pk.page4_store(k, k[:3], four, slots), lambda: pk.page4_store(k, k, four, slots[:3]),
        lambda: pk.page4_store(k, k, four, slots.long()), lambda: pk.page4_store(k.half(), k.half(), four, slots),
        lambda: pk.page4_store(k, k, (four[0], four[1], four[2], four[3].int()), slots),
        lambda: pk.page4_store(k, k, (four[0], four[1][:2], four[2], four[3]), slots),
        lambda: pk.page4_store(k, k, (four[0], four[1], four[2][:, :1], four[3]), slots),
        lambda: pk.page4_store(torch.zeros(4, 3, 128), torch.zeros(4, 3, 128), four, slots),
        lambda: pk.page4_read(four, slots, torch.float16), lambda: pk.page4_read(four, slots, torch.float32, k_out=k[:3]),
        lambda: pk.page4_read(four, slots, torch.bfloat16, v_out=k),
        lambda: pk.norm_rotate(k, None, slots, pk.pair_axes((64,)), 1e4, torch.ones(64), None, 1e-6),
        lambda: pk.norm_rotate(k, None, slots, pk.pair_axes((64,)), 1e4, torch.ones(128).bfloat16(), None, 1e-6),
        lambda: pk.norm_rotate(None, None, slots, pk.pair_axes((64,)), 1e4, None, None, 1e-6),
        lambda: pk.page_copy([], slots, slots), lambda: pk.page_copy([torch.zeros(3, 2)], slots, slots),
        lambda: pk.page_copy([torch.zeros(3, 2, 16, 8), torch.zeros(3, 2, 8, 8)], slots, slots),
        lambda: pk.page_copy([torch.zeros(3, 2, 16, 8)], slots, slots[:2]),
        lambda: pk.page_copy([torch.zeros(3, 2, 16, 8).transpose(1, 2)], slots, slots),
        lambda: pk.page_fork(slots, slots, slots, slots[None], slots, slots, slots[:1], 16),
        lambda: pk.page_fork(slots, slots, slots[:2], slots[:, None], slots, slots, slots[:1], 16),
        lambda: pk.page_fork(slots, slots, slots, slots[:, None], slots[:2], slots, slots[:1], 16),
        lambda: pk.page_release(slots, slots, slots[:, None], slots, slots, slots, 16),
        lambda: pk.page_release(slots, slots[:1], slots[:, None], slots, slots, slots[:1], 16),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    assert not host
