"""Refusals of the 8-bit cache's calls: all of them come before anything is enqueued, so they run without a GPU."""
import ctypes as C

import numpy as np
import pytest

import cache_reference as ref


@pytest.fixture(scope="module")
def sb():
    import os
    from paper_2507_06517_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2507_06517_amd import build
        build.build_library(verbose=False)
    binding.lib()
    return binding


FAKE, NULL = 0x1000, None


def desc(sb, **kw):
    a = dict(n_pages=8, heads=2, page=64, dim=128, fmt=0, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, pos=None)
    a.update(kw)
    return C.byref(sb.CacheDesc(a["n_pages"], a["heads"], a["page"], a["dim"], a["fmt"], 0, a["k"], a["v"], a["ks"], a["vs"], a["pos"]))


BAD_CACHES = [(dict(n_pages=0), 1), (dict(heads=0), 1), (dict(heads=2000), 2), (dict(page=16), 2), (dict(page=96), 2), (dict(dim=64), 2),
              (dict(fmt=2), 1), (dict(k=None), 1), (dict(vs=None), 1), (dict(v=0x1008), 1), (dict(pos=0x1002), 1)]


def append(sb, cache=None, **kw):
    a = dict(table=FAKE, width=4, len=FAKE, batch=2, cu=FAKE, max_new=3, total=5, K=FAKE, V=FAKE, dtype=1, stride_b=0, sh=128, st=256, pos=None)
    a.update(kw)
    return sb.lib().spindle_cache_append(cache if cache is not None else desc(sb), a["table"], a["width"], a["len"], a["batch"], a["cu"], a["max_new"],
                                         a["total"], a["K"], a["V"], a["dtype"], a["stride_b"], a["sh"], a["st"], a["pos"], None)


def attend(sb, cache=None, **kw):
    a = dict(table=FAKE, width=64, len=FAKE, batch=2, cu=FAKE, max_q=3, total=5, Q=FAKE, dtype=1, group=4, st=1024, sh=128, scale=0.1, cap=0.0,
             out=FAKE, ws=FAKE, wsb=1 << 30)
    a.update(kw)
    return sb.lib().spindle_cache_attend(cache if cache is not None else desc(sb), a["table"], a["width"], a["len"], a["batch"], a["cu"], a["max_q"], a["total"],
                                         a["Q"], a["dtype"], a["group"], a["st"], a["sh"], a["scale"], a["cap"], None, None, None, a["out"], None,
                                         a["ws"], a["wsb"], None)


def compact(sb, cache=None, **kw):
    a = dict(table=FAKE, width=4, len=FAKE, batch=2, kept=FAKE, stride=10, n=FAKE, out=FAKE, out_width=1)
    a.update(kw)
    return sb.lib().spindle_cache_compact(cache if cache is not None else desc(sb), a["table"], a["width"], a["len"], a["batch"], a["kept"], a["stride"], a["n"],
                                          a["out"], a["out_width"], None)


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_bad_caches(sb, bad, code):
    c = desc(sb, **bad)
    n = C.c_size_t(0)
    assert append(sb, c) == code
    assert attend(sb, c) == code
    assert compact(sb, c) == code
    assert sb.lib().spindle_cache_copy(c, FAKE, 1, None) == code
    assert sb.lib().spindle_attend_workspace_bytes(c, 1, 4, 1, 1, 4, 1, C.byref(n)) == code
    assert sb.lib().spindle_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(table=None), 1), (dict(len=None), 1), (dict(batch=0), 1), (dict(batch=40000), 2), (dict(width=0), 1), (dict(width=1 << 28), 2),
    (dict(K=None), 1), (dict(V=None), 1), (dict(K=0x1004), 1), (dict(dtype=3), 1), (dict(max_new=-1), 1), (dict(total=-1), 1),
    (dict(cu=None), 1), (dict(sh=64), 1), (dict(st=130), 1), (dict(stride_b=-8), 1), (dict(width=1 << 20, max_new=1 << 28, total=1 << 28), 2)])
def test_append_refuses(sb, bad, code):
    assert append(sb, **bad) == code


def test_nothing_to_do_is_no_error(sb):
    assert append(sb, max_new=0) == 0 and append(sb, total=0) == 0
    assert attend(sb, max_q=0) == 0 and attend(sb, total=0) == 0
    assert sb.lib().spindle_cache_copy(desc(sb), FAKE, 0, None) == 0


@pytest.mark.parametrize("bad,code", [
    (dict(table=None), 1), (dict(Q=None), 1), (dict(out=None), 1), (dict(Q=0x1008), 1), (dict(out=0x1004), 1), (dict(dtype=-1), 1),
    (dict(group=0), 1), (dict(group=300), 2), (dict(scale=0.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
    (dict(cap=-1.0), 1), (dict(cap=float("nan")), 1), (dict(st=64), 1), (dict(sh=132), 1), (dict(max_q=-2), 1), (dict(cu=None), 1),
    (dict(ws=None), 3), (dict(ws=0x1010), 3), (dict(wsb=16), 3), (dict(max_q=1 << 24), 2)])
def test_attend_refuses(sb, bad, code):
    assert attend(sb, **bad) == code


@pytest.mark.parametrize("bad,code", [(dict(kept=None), 1), (dict(stride=0), 1), (dict(n=None), 1), (dict(out=None), 1), (dict(out_width=0), 1),
                                      (dict(table=None), 1)])
def test_compact_refuses(sb, bad, code):
    assert compact(sb, **bad) == code


def test_pages_refuse(sb):
    L = sb.lib()

    def share(refs=FAKE, n_pages=8, table=FAKE, n=FAKE, rows=2, width=4, page=64, parent=FAKE, rows_out=2, out=0x2000, n_out=0x2000):
        return L.spindle_pages_share(refs, n_pages, table, n, rows, width, page, parent, rows_out, out, n_out, None)

    def reserve(refs=FAKE, n_pages=8, table=FAKE, n=FAKE, grow=FAKE, rows=2, width=4, page=64, n_out=0x2000, copies=FAKE, status=FAKE, ws=FAKE, wsb=256):
        return L.spindle_pages_reserve(refs, n_pages, table, n, grow, rows, width, page, n_out, copies, status, ws, wsb, None)

    def release(refs=FAKE, n_pages=8, table=FAKE, n=FAKE, rows=2, width=4, page=64):
        return L.spindle_pages_release(refs, n_pages, table, n, rows, width, page, None)

    for call in (share, reserve, release):
        for bad, code in ((dict(refs=None), 1), (dict(n_pages=0), 1), (dict(table=None), 1), (dict(n=None), 1), (dict(rows=0), 1),
                          (dict(width=0), 1), (dict(page=48), 2), (dict(width=1 << 27), 2)):
            assert call(**bad) == code, (call.__name__, bad)
    assert share(parent=None) == 1 and share(rows_out=0) == 1 and share(out=FAKE) == 1 and share(n_out=FAKE) == 1
    assert reserve(grow=None) == 1 and reserve(copies=None) == 1 and reserve(status=None) == 1 and reserve(n_out=FAKE) == 1
    assert reserve(rows=5000) == 2 and reserve(ws=None) == 3 and reserve(wsb=31) == 3 and reserve(ws=0x1010) == 3
    n = C.c_size_t(0)
    assert L.spindle_pages_workspace_bytes(0, C.byref(n)) == 1 and L.spindle_pages_workspace_bytes(8, None) == 1
    assert sb.spindle_pages_workspace_bytes(1000) >= 4000


def test_binding_refuses_what_does_not_fit(sb):
    import torch
    cache = sb.new_cache(4, 2, 64, "i8", positions=True, device="cpu")
    table, lens = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    x = torch.zeros((1, 2, 3, 128), dtype=torch.float16)
    with pytest.raises(ValueError, match="format"):
        sb.new_cache(4, 2, 64, "e5m2", device="cpu")
    with pytest.raises(ValueError, match="k must be"):
        sb.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale, None, 32, "i8")
    with pytest.raises(ValueError, match="lens"):
        sb.cache_append(cache, table, lens.long(), x, x)
    with pytest.raises(ValueError, match="table"):
        sb.cache_append(cache, table[0], lens, x, x)
    with pytest.raises(ValueError, match="same type"):
        sb.cache_append(cache, table, lens, x, x.float())
    with pytest.raises(ValueError, match=r"K and V must be \[1, 2"):
        sb.cache_append(cache, table, lens, x[:, :1], x[:, :1])
    with pytest.raises(ValueError, match="tokens are"):
        sb.cache_append(cache, table, lens, x.double(), x.double())
    with pytest.raises(ValueError, match="positions"):
        sb.cache_append(cache, table, lens, x, x, positions=lens)
    with pytest.raises(ValueError, match="Q is"):
        sb.cache_attend(cache, table, lens, x, 4)
    q = torch.zeros((1, 3, 8, 128), dtype=torch.float16)
    with pytest.raises(ValueError, match="slopes"):
        sb.cache_attend(cache, table, lens, q, 4, slopes=torch.zeros(4))
    with pytest.raises(ValueError, match="out must be"):
        sb.cache_attend(cache, table, lens, q, 4, out=q.float())
    with pytest.raises(ValueError, match="kept"):
        sb.cache_compact(cache, table, lens, torch.zeros((1, 3, 4), dtype=torch.int32), lens, table)
    with pytest.raises(ValueError, match="copies"):
        sb.cache_copy(cache, torch.zeros((2, 3), dtype=torch.int32))
    with pytest.raises(ValueError, match="parent"):
        sb.pages_share(lens, table, lens, torch.zeros(2), 64)
    with pytest.raises(ValueError, match="grow"):
        sb.pages_reserve(lens, table, lens, torch.zeros(2, dtype=torch.int32), 64)


# ------------------------------------------------------------------ the plain implementation itself

def test_codes_of_the_reference():
    import torch
    v = ref.E4M3[np.isfinite(ref.E4M3)]
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(ref.E4M3, want)
    np.testing.assert_array_equal(ref.nearest(v, "e4m3"), v)
    u = np.unique(v)
    mid = (u[1:] + u[:-1]) / 2                                       # halfway: the even neighbour, and just beside it the nearer one
    for x, lo, hi in zip(mid, u[:-1], u[1:]):
        assert ref.nearest(np.array([x]), "e4m3")[0] in (lo, hi)
        assert ref.nearest(np.array([x + 1e-12 * abs(x)]), "e4m3")[0] == hi
        assert ref.nearest(np.array([x - 1e-12 * abs(x)]), "e4m3")[0] == lo
    assert ref.nearest(np.array([17.0]), "e4m3")[0] == 16 and ref.nearest(np.array([19.0]), "e4m3")[0] == 20   # steps of 2: to even
    assert ref.nearest(np.array([0.5, 1.5, -2.5, 500.0, np.nan]), "i8").tolist() == [0, 2, -2, 127, 0]


def test_scales_of_the_reference():
    assert ref.scale_for(448.0, "e4m3") == 1 and ref.scale_for(448.01, "e4m3") == 2 and ref.scale_for(225.0, "e4m3") == 1 and ref.scale_for(224.0, "e4m3") == 0.5
    assert ref.scale_for(0.0, "e4m3") == ref.scale_for(0.0, "i8") == 2.0 ** -126
    assert ref.scale_for(127.0, "i8") == 1


def test_reservation_of_the_reference_by_hand():
    refs = np.int32([3, 0, 1, 0, 0, 0])
    table = np.int32([[0, -1, -1], [0, -1, -1], [0, -1, -1], [2, -1, -1]])
    n, copies, status = ref.reserve(refs, table, np.int32([40, 40, 40, 64]), np.int32([1, 30, 1, 1]), 64)
    assert status.tolist() == [0, 0] and n.tolist() == [41, 70, 41, 65]
    assert copies.tolist() == [[0, 1], [0, 3], [-1, -1], [-1, -1]]   # the third row is alone with the page by then
    assert table.tolist() == [[1, -1, -1], [3, 4, -1], [0, -1, -1], [2, 5, -1]]
    assert refs.tolist() == [1, 1, 1, 1, 1, 1]
    again = ref.reserve(refs, table, n, np.int32([0, 0, 0, 64]), 64)
    assert again[2].tolist() == [1, 0] and again[0].tolist() == n.tolist()


def test_grids_that_a_launch_cannot_hold_are_refused(sb):
    wide = desc(sb, heads=1024)
    assert attend(sb, wide, batch=32767, max_q=1, total=32767, group=1, width=4) == 2
    assert append(sb, wide, batch=32767, max_new=1, total=32767) == 2
    assert compact(sb, wide, batch=32767) == 2
    assert sb.lib().spindle_cache_copy(wide, FAKE, 1 << 20, None) == 2
    assert append(sb, desc(sb, n_pages=1 << 29, heads=2)) == 2


def test_calls_without_tokens_take_no_pointers(sb):
    """Tensors without elements have no address."""
    assert append(sb, max_new=0, K=None, V=None) == 0 and append(sb, total=0, K=None, V=None) == 0
    assert attend(sb, max_q=0, Q=None, out=None) == 0 and attend(sb, total=0, Q=None, out=None) == 0
    assert attend(sb, cu=None, batch=2, max_q=0, total=0, Q=None, out=None, ws=None, wsb=0) == 0
    assert sb.lib().spindle_cache_copy(desc(sb), None, 0, None) == 0
    assert append(sb, max_new=0, dtype=3) == 1 and attend(sb, max_q=0, scale=0.0) == 1     # everything else is looked at
    assert sb.lib().spindle_cache_copy(desc(sb), None, 1, None) == 1


def test_given_workspaces_are_looked_at(sb):
    """The library gets its address: it has to be on the cache's device and in one piece."""
    import torch
    cache = sb.new_cache(64, 1, 64, "i8", device="cpu")
    table, lens = torch.zeros((1, 60), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    q = torch.zeros((1, 1, 4, 128), dtype=torch.float16)
    n = sb.spindle_attend_workspace_bytes(cache.ref, 1, 60, 1, 1, 4, sb.F16)
    assert n > 0
    with pytest.raises(ValueError, match="workspace"):
        sb.cache_attend(cache, table, lens, q, 4, workspace=torch.empty(n, dtype=torch.uint8, device="meta"))
    with pytest.raises(ValueError, match="workspace"):
        sb.cache_attend(cache, table, lens, q, 4, workspace=torch.empty(2 * n, dtype=torch.uint8)[::2])


def test_tensors_that_are_not_on_the_current_gpu_are_refused(sb, monkeypatch):
    """Calls that fit in every other way: kernels must not get addresses of host memory, nor run beside the tensors' device."""
    import torch
    cache = sb.new_cache(4, 2, 64, "i8", device="cpu")
    table, lens = torch.zeros((1, 2), dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    kv, q, refs = torch.zeros((1, 2, 3, 128)), torch.zeros((1, 1, 8, 128)), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: sb.cache_append(cache, table, lens, kv, kv), lambda: sb.cache_attend(cache, table, lens, q, 4),
                 lambda: sb.cache_compact(cache, table, lens, torch.zeros((1, 2, 5), dtype=torch.int32), lens, table),
                 lambda: sb.cache_copy(cache, torch.zeros((1, 2), dtype=torch.int32)), lambda: sb.pages_share(refs, table, lens, lens, 64),
                 lambda: sb.pages_reserve(refs, table, lens, lens, 64), lambda: sb.pages_release(refs, table, lens, 64)):
        with pytest.raises(ValueError, match="not on a GPU"):
            call()
    monkeypatch.setattr(sb, "_raw_stream", lambda device: 7 + device)
    monkeypatch.setattr(sb, "_current_device", lambda: 0)
    assert sb._stream_on(torch.device("cuda", 0)) == 7
    with pytest.raises(ValueError, match="current device"):
        sb._stream_on(torch.device("cuda", 1))


def test_sizes_next_to_the_largest_integers(sb):
    """No sum of the sizes wraps around on the way to a grid: each of these asks for more than a launch holds."""
    wide = desc(sb, heads=1024)
    assert compact(sb, wide, batch=32767, stride=2 ** 31 - 1, out_width=4) == 2
    assert append(sb, wide, batch=32767, max_new=2 ** 31 - 1, total=2 ** 31 - 1, width=4) == 2


def test_counts_of_more_pages_than_a_pool_has_are_refused(sb):
    """The bookkeeping counts pages in steps of 16384, which must not pass the largest integer; a pool ends at 2^30."""
    L, n = sb.lib(), C.c_size_t(0)
    for n_pages in (2 ** 30, 2 ** 31 - 1):
        assert L.spindle_pages_share(FAKE, n_pages, FAKE, FAKE, 2, 4, 64, FAKE, 2, 0x2000, 0x2000, None) == 2
        assert L.spindle_pages_reserve(FAKE, n_pages, FAKE, FAKE, FAKE, 2, 4, 64, 0x2000, FAKE, FAKE, FAKE, 1 << 40, None) == 2
        assert L.spindle_pages_release(FAKE, n_pages, FAKE, FAKE, 2, 4, 64, None) == 2
        assert L.spindle_pages_workspace_bytes(n_pages, C.byref(n)) == 2
