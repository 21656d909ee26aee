"""CPU: the handle-free calls (rotary positions, block tables, exact attention)
refuse what they cannot do before anything is launched, and say why.  No GPU is
touched: every call below is refused on the host."""
import ctypes

import pytest
import torch

from paper_2606_26762_amd import protokv as pk

GOOD = 1 << 20   # an aligned address; refused calls never read it


def _status(name, args):
    return getattr(pk.lib(), "protokv_" + name)(ctypes.byref(args), None)


def _set(a, **kw):
    for f, v in kw.items():
        head, _, rest = f.partition("__")
        setattr(getattr(a, head) if rest else a, rest or head, v)
    return a


def plan(**kw):
    a = pk.PagePlanArgs(4, 100, 16, 8, 64, *[GOOD + 4096 * i for i in range(12)])
    return _set(a, **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(num_requests=0), 1), (dict(num_requests=8193), 2), (dict(num_pages=0), 1), (dict(page_size=0), 2),
    (dict(page_size=24), 2), (dict(page_size=2048), 2), (dict(num_pages=1 << 27), 2), (dict(table_stride=0), 1),
    (dict(table_stride=1 << 27), 1), (dict(max_tokens=0), 1), (dict(max_tokens=(1 << 29) + 1), 1),
    (dict(page_size=1, num_pages=(1 << 29) + 1), 2),
    (dict(ctx=None), 1), (dict(add=None), 1), (dict(table=None), 1), (dict(free_pages=None), 1),
    (dict(free_count=None), 1), (dict(free_count_out=None), 1), (dict(cu=None), 1), (dict(kv_len=None), 1),
    (dict(slots=None), 1), (dict(slots=GOOD + 2), 1), (dict(base=GOOD + 1), 1), (dict(refused=GOOD + 3), 1),
    (dict(free_count_out=GOOD + 4096 * 5), 1), (dict(kv_len=GOOD), 1), (dict(cu=GOOD + 4096), 1),
    (dict(positions=GOOD + 4096 * 2), 1)])
def test_page_plan_refuses(kw, status):
    assert _status("page_plan", plan(**kw)) == status
    assert b"page_plan: " in pk.lib().protokv_last_error(None)


def rotate(**kw):
    a = pk.RotateArgs(num_tokens=3, num_q_heads=8, num_kv_heads=2, head_dim=128, kv_dtype=pk.KV_BF16, num_axes=3,
                      positions=GOOD, position_stride=3, axes=pk.pair_axes((16, 24, 24)), theta=1e6, q=GOOD, k=GOOD,
                      v=GOOD, q_stride=1024, k_stride=256, v_stride=256, q_out=GOOD, k_out=None, q_out_stride=1024,
                      k_out_stride=256, slots=GOOD)
    pages = pk.Pages(GOOD, GOOD, 10, 16)
    for f in [f for f in kw if f.startswith("pages__")]:
        setattr(pages, f[7:], kw.pop(f))
    a.pages = ctypes.pointer(pages)
    if kw.pop("no_pages", False):
        a.pages = None
    return _set(a, **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(num_tokens=-1), 1), (dict(num_q_heads=7), 1), (dict(num_kv_heads=0), 1), (dict(head_dim=64), 2),
    (dict(kv_dtype=2), 1), (dict(num_axes=0), 1), (dict(num_axes=9), 1), (dict(num_axes=2), 1), (dict(axes=None), 1),
    (dict(theta=1.0), 1), (dict(theta=float("nan")), 1), (dict(theta=float("inf")), 1), (dict(position_stride=-1), 1),
    (dict(positions=None), 1), (dict(positions=GOOD + 2), 1), (dict(q=None), 1), (dict(q_out=None), 1),
    (dict(k=None), 1), (dict(v=None), 1), (dict(no_pages=True), 1), (dict(no_pages=True, v=None), 1),
    (dict(slots=None), 1), (dict(q=GOOD + 8), 1), (dict(q_stride=1020), 1), (dict(q_stride=1025), 1),
    (dict(k_stride=255), 1), (dict(v_stride=260), 1), (dict(q_out_stride=2048), 1),
    (dict(k_out=GOOD + 16, k_out_stride=128), 1), (dict(pages__page_size=12), 2), (dict(pages__num_pages=0), 1),
    (dict(pages__num_pages=1 << 27), 2), (dict(pages__k=None), 1), (dict(pages__v=GOOD + 4), 1)])
def test_rotate_refuses(kw, status):
    assert _status("rotate", rotate(**dict(kw))) == status
    assert b"rotate: " in pk.lib().protokv_last_error(None)


def prompt(**kw):
    return _set(pk.PromptArgs(8, 2, 128, pk.KV_BF16, 2, 40, GOOD, GOOD, GOOD, GOOD, 1024, 256, 256, GOOD, GOOD, None,
                              None), **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(num_q_heads=9), 1), (dict(num_q_heads=0), 1), (dict(num_q_heads=1024, num_kv_heads=2, q_stride=1 << 17), 2),
    (dict(head_dim=96), 2), (dict(kv_dtype=7), 1), (dict(num_seqs=-1), 1), (dict(num_seqs=1 << 24), 2),
    (dict(total=-1), 1), (dict(total=1 << 28), 2), (dict(cu=None), 1), (dict(cu=GOOD + 2), 1), (dict(q=None), 1),
    (dict(k=GOOD + 4), 1), (dict(v=None), 1), (dict(q_stride=1016), 1), (dict(k_stride=257), 1),
    (dict(v_stride=(1 << 32) + 8), 1), (dict(o=None), 1), (dict(o=GOOD + 8), 1), (dict(lse=GOOD + 1), 1),
    (dict(prior_o=GOOD), 1), (dict(prior_lse=GOOD), 1), (dict(prior_o=GOOD + 8, prior_lse=GOOD), 1)])
def test_prompt_attend_refuses(kw, status):
    assert _status("prompt_attend", prompt(**kw)) == status
    assert b"prompt_attend: " in pk.lib().protokv_last_error(None)


def page(**kw):
    a = pk.PageAttendArgs(8, 2, 128, pk.KV_BF16, 2, 40, 30, 64, GOOD, GOOD, GOOD, GOOD, 1024,
                          pk.Pages(GOOD, GOOD, 100, 16), GOOD, GOOD, None, None, GOOD, 1 << 40)
    return _set(a, **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(num_q_heads=9), 1), (dict(head_dim=64), 2), (dict(kv_dtype=-1), 1), (dict(num_requests=-1), 1),
    (dict(total=-5), 1), (dict(total=1 << 28), 2), (dict(max_add=0), 1), (dict(table_stride=0), 1),
    (dict(table_stride=1 << 27), 1), (dict(cu=None), 1), (dict(kv_len=None), 1), (dict(kv_len=GOOD + 1), 1),
    (dict(table=None), 1), (dict(q=None), 1), (dict(q_stride=1000), 1), (dict(pages__page_size=0), 2),
    (dict(pages__page_size=48), 2), (dict(pages__num_pages=0), 1), (dict(pages__num_pages=1 << 27), 2),
    (dict(pages__k=None), 1), (dict(pages__v=GOOD + 2), 1), (dict(o=None), 1), (dict(prior_o=GOOD), 1),
    (dict(workspace=None), 3), (dict(workspace=GOOD + 16), 3), (dict(workspace_bytes=1000), 3)])
def test_page_attend_refuses(kw, status):
    assert _status("page_attend", page(**kw)) == status
    assert b"page_attend: " in pk.lib().protokv_last_error(None)


def test_null_arguments_are_refused():
    L = pk.lib()
    for name in ("page_plan", "rotate", "prompt_attend", "page_attend"):
        assert getattr(L, "protokv_" + name)(None, None) == 1
    n = ctypes.c_size_t()
    assert L.protokv_page_attend_workspace(None, ctypes.byref(n)) == 1
    assert L.protokv_page_attend_workspace(ctypes.byref(page()), None) == 1


def test_empty_calls_are_done_at_once():
    """Nothing to do is no error, and nothing is launched."""
    assert _status("rotate", rotate(num_tokens=0, positions=None, slots=None)) == 0
    for kw in (dict(num_seqs=0), dict(total=0)):
        assert _status("prompt_attend", prompt(**kw)) == 0
    for kw in (dict(num_requests=0), dict(total=0)):
        assert _status("page_attend", page(**kw)) == 0


def _workspace(**kw):
    n = ctypes.c_size_t(1 << 62)
    assert pk.lib().protokv_page_attend_workspace(ctypes.byref(page(**kw)), ctypes.byref(n)) == 0
    return n.value


def test_page_attend_workspace_goes_by_sizes_alone():
    base = _workspace()
    assert base == _workspace(cu=None, kv_len=None, table=None, q=None, o=None, workspace=None, pages__k=None)
    assert 0 < base < 1 << 28
    n = ctypes.c_size_t()
    assert pk.lib().protokv_page_attend_workspace(ctypes.byref(page(head_dim=64)), ctypes.byref(n)) == 2


def test_pair_axes():
    assert pk.pair_axes((16, 24, 24)) == bytes([0] * 16 + [1] * 24 + [2] * 24)
    inter = pk.pair_axes((16, 24, 24), interleaved=True)
    assert inter[:48] == bytes([0, 1, 2] * 16) and inter[48:] == bytes([1, 2] * 8)
    assert pk.pair_axes((64,)) == bytes(64) == pk.pair_axes([64], interleaved=True)
    for bad in ((16, 24), (65, -1), (), (8,) * 9, (0, 63)):
        with pytest.raises(ValueError):
            pk.pair_axes(bad)


def test_binding_refuses_host_tensors_and_wrong_shapes():
    q, k = torch.zeros(4, 8, 128, dtype=torch.bfloat16), torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError):
        pk.prompt_attend(q, k, k, cu)
    with pytest.raises(ValueError):
        pk.rotate(q, k, torch.zeros(4, dtype=torch.int32), pk.pair_axes((64,)), 1e4)
    with pytest.raises(ValueError):
        pk.rotate(None, None, cu, pk.pair_axes((64,)), 1e4)
    with pytest.raises(ValueError):
        pk.page_attend(q, (k, k), cu, cu, cu, 1)


def test_launches_that_would_be_too_large_are_refused():
    """A launch has fewer than 2^32 threads; counts that pass every other check."""
    for name, a in (("prompt_attend", prompt(num_seqs=(1 << 24) - 1, num_q_heads=8, num_kv_heads=8, k_stride=1024,
                                             v_stride=1024)),
                    ("page_attend", page(num_requests=1 << 23, max_add=100)),
                    ("rotate", rotate(num_tokens=1 << 27)), ("rotate", rotate(num_tokens=(1 << 25) + 1))):
        assert _status(name, a) == 2, name
        assert b"for one launch" in pk.lib().protokv_last_error(None) or b"2^29" in pk.lib().protokv_last_error(None)


def test_rotate_of_no_tokens_needs_no_addresses():
    """Empty tensors may have none."""
    assert _status("rotate", rotate(num_tokens=0, q=None, k=None, v=None, q_out=None, positions=None, slots=None)) == 0


def test_page_attend_refuses_places_that_would_pass_32_bits():
    for stride, size in (((1 << 27) - 1, 16), ((1 << 27) - 127, 16), ((1 << 21) - 1, 1024)):
        a = page(table_stride=stride)
        a.pages.page_size = size
        assert _status("page_attend", a) == 1
        assert b"2^31" in pk.lib().protokv_last_error(None)
    a = page(table_stride=(1 << 27) - 128, max_add=1, workspace=None)
    assert _status("page_attend", a) == 3   # its sizes are fine


@pytest.mark.parametrize("tokens", [(1 << 26) - 1, (1 << 26) - 3, 1 << 26])
def test_rotate_refuses_waves_that_make_2_to_32_threads_in_whole_workgroups(tokens):
    """A wave to a token; workgroups are of four."""
    a = rotate(num_tokens=tokens, k=None, v=None, slots=None, no_pages=True)
    assert _status("rotate", a) == 2
    assert b"2^29" in pk.lib().protokv_last_error(None)


def _calls_with(**leaf):
    """Each call that takes floating-point tensors, with those named in `leaf` in place of its own."""
    t = dict(q=torch.zeros(4, 8, 128), k=torch.zeros(4, 2, 128), v=torch.zeros(4, 2, 128), k_pages=torch.zeros(3, 2, 16, 128),
             v_pages=torch.zeros(3, 2, 16, 128), out=torch.zeros(4, 8, 128), prior_o=torch.zeros(4, 8, 128))
    t.update(leaf)
    i32 = dict(dtype=torch.int32)
    cu, one, pages = torch.tensor([0, 4], **i32), torch.tensor([20], **i32), (t["k_pages"], t["v_pages"])
    prior = (t["prior_o"], torch.zeros(4, 8))
    uses = {
        "rotate": ("q k v k_pages v_pages out", lambda: pk.rotate(
            t["q"], t["k"], torch.zeros(4, **i32), pk.pair_axes((64,)), 1e4, q_out=t["out"], v=t["v"], pages=pages,
            slots=torch.zeros(4, **i32))),
        "prompt_attend": ("q k v out prior_o", lambda: pk.prompt_attend(t["q"], t["k"], t["v"], cu, out=t["out"], prior=prior)),
        "page_attend": ("q k_pages v_pages out prior_o", lambda: pk.page_attend(
            t["q"], pages, torch.zeros(1, 3, **i32), cu, one, 4, out=t["out"], prior=prior))}
    return [f for names, f in uses.values() if set(leaf) <= set(names.split())]


@pytest.mark.parametrize("name", ["q", "k", "v", "k_pages", "v_pages", "out", "prior_o"])
def test_binding_refuses_what_a_gradient_is_asked_of(name, monkeypatch):
    """The results would carry none; with gradients off, the same tensors are only values."""
    monkeypatch.setattr(pk, "_device", lambda t, stream: -1)   # host tensors pass as those of the current device
    monkeypatch.setattr(pk, "_raw_stream", lambda stream, dev: None)
    done = []
    monkeypatch.setattr(pk, "_check", lambda status: done.append(status))
    class Library:   # launches nothing
        def __getattr__(self, call):
            return lambda *a: 0
    monkeypatch.setattr(pk, "lib", Library)
    shape = dict(q=(4, 8, 128), out=(4, 8, 128), prior_o=(4, 8, 128), k=(4, 2, 128), v=(4, 2, 128)).get(name, (3, 2, 16, 128))
    calls = _calls_with(**{name: torch.zeros(*shape, requires_grad=True)})
    assert calls
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
    assert not done
    with torch.no_grad():
        for call in calls:
            call()
    assert len(done) >= len(calls)
