"""The paged cache in 8 bits on the GPU against the plain implementation in 64 bits: stored codes and bookkeeping have to be
equal, attention within a bound made of its roundings."""
import numpy as np
import pytest

import cache_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FMTS = ["e4m3", "i8"]


@pytest.fixture(scope="module")
def sb():
    from paper_2507_06517_amd import binding
    binding.lib()
    return binding


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def pools_of(cache):
    h = [t.cpu().numpy() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    return ref.Pools(*h, None if cache.pos is None else cache.pos.cpu().numpy(), cache.page_tokens, cache.format)


def same_pools(cache, want):
    got = pools_of(cache)
    for w, name in enumerate("kv"):
        np.testing.assert_array_equal(got.s[w], want.s[w], err_msg=name + " scales")
        np.testing.assert_array_equal(got.x[w], want.x[w], err_msg=name + " codes")
    if want.pos is not None:
        np.testing.assert_array_equal(got.pos, want.pos)


def table_of(rng, counts, width, n_pages):
    order = rng.permutation(n_pages)
    t, at = np.full((len(counts), width), -1, np.int32), 0
    for b, n in enumerate(counts):
        t[b, :n] = order[at:at + n]
        at += n
    return t


def tokens(rng, n, heads):
    x = rng.standard_normal((n, heads, 128)) * np.exp(rng.uniform(-2, 2, (n, heads, 1)))
    return x.astype(np.float32)


def filled(sb, rng, lens, heads, page, fmt, positions=False, width=None, spare=2):
    """A cache that holds `lens` tokens of each sequence (scattered pages), and its table."""
    counts = [-(-max(n, 0) // page) for n in lens]
    n_pages = sum(counts) + spare
    cache = sb.new_cache(n_pages, heads, page, fmt, positions=positions)
    # what nobody wrote must not be seen: NaN codes (-128 as integers)
    cache.k.fill_(0x80 if fmt == "i8" else 0x7F)
    cache.v.fill_(0x80 if fmt == "i8" else 0xFF)
    cache.k_scale.fill_(float("nan"))
    cache.v_scale.fill_(float("nan"))
    table = table_of(rng, counts, width or max(max(counts), 1), n_pages)
    K, V = (dev(tokens(rng, sum(max(n, 0) for n in lens), heads)) for _ in range(2))
    cu = np.concatenate([[0], np.cumsum([max(n, 0) for n in lens])]).astype(np.int32)
    if K.shape[0]:
        sb.cache_append(cache, dev(table), dev(np.zeros(len(lens), np.int32)), K, V, cu_new=dev(cu), max_new=max(lens))
    return cache, table


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("page", [32, 64, 128, 256])
def test_append_in_pieces(sb, dtype, fmt, page):
    rng = np.random.default_rng(page)
    heads, steps = 3, [[0, 1, page, 2 * page + 5], [1, page - 1, 0, 7], [page, 1, 1, 1], [3, 2 * page, 70, 1]]
    total = np.sum(steps, 0)
    width = max(-(-int(n) // page) for n in total)
    table = table_of(rng, [-(-int(n) // page) for n in total], width, 24)
    cache = sb.new_cache(24, heads, page, fmt, positions=True)
    want, lens = pools_of(cache), np.zeros(4, np.int32)
    for k, new in enumerate(steps):
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        # magnitudes grow from step to step for one head and shrink for another
        xs = [torch.from_numpy(tokens(rng, int(cu[-1]), heads) * np.float32([[[1]], [[3.0 ** k]], [[0.2 ** k]]]).reshape(1, 3, 1)).to(DT[dtype]) for _ in range(2)]
        at = rng.integers(0, 1 << 20, int(cu[-1])).astype(np.int32) if k % 2 else None
        sb.cache_append(cache, dev(table), dev(lens), xs[0].cuda(), xs[1].cuda(), cu_new=dev(cu), max_new=max(new),
                        positions=None if at is None else dev(at))
        ref.append(want, table, lens, [x.double().numpy() for x in xs], cu, at)
        same_pools(cache, want)
        lens = lens + np.int32(new)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", list(DT))
def test_append_special_values(sb, dtype, fmt):
    """NaN, infinities, zeros, denormals, the largest numbers, and values halfway between two codes."""
    rng = np.random.default_rng(5)
    top = float(torch.finfo(DT[dtype]).max)
    x = tokens(rng, 96, 2)
    x[3, 0, 5], x[4, 0, 6], x[5, 0, 7], x[6, 0, 8] = np.nan, np.inf, -np.inf, -0.0
    x[32:64, 0] = 0
    x[32:64, 1] = 0
    x[40, 1, 9] = float(torch.finfo(DT[dtype]).tiny) * 0.75
    x[64:96, 0] = 448.0
    x[64:96, 1] = rng.integers(-254, 255, (32, 128)) / 2.0            # halves: ties of the integers at scale 1
    x[64, 1, 0] = 127.0
    if dtype != "f16":
        x[64:96, 0] *= top / 1000
    K = torch.from_numpy(x).to(DT[dtype])
    V = torch.from_numpy(x[::-1].copy()).to(DT[dtype])
    cache = sb.new_cache(4, 2, 32, fmt)
    want = pools_of(cache)
    table, cu = np.int32([[2, 0, 3]]), np.int32([0, 96])
    sb.cache_append(cache, dev(table), dev(np.int32([0])), K.cuda(), V.cuda(), cu_new=dev(cu), max_new=96)
    ref.append(want, table, [0], [K.double().numpy(), V.double().numpy()], cu, None)
    same_pools(cache, want)
    assert np.isfinite(pools_of(cache).x[0]).all()


def test_append_layouts_agree(sb):
    """[B, H, m, d], a cache stored token by token, and rows one behind the other."""
    rng = np.random.default_rng(6)
    B, H, m = 3, 4, 45
    x = [torch.from_numpy(rng.standard_normal((B, m, H, 128)).astype(np.float32)).half().cuda() for _ in range(2)]
    table, lens = dev(table_of(rng, [2, 2, 2], 2, 8)), dev(np.int32([0, 3, 19]))
    caches = [sb.new_cache(8, H, 32, "e4m3") for _ in range(3)]
    sb.cache_append(caches[0], table, lens, *(t.reshape(B * m, H, 128) for t in x), cu_new=dev(np.int32([0, m, 2 * m, 3 * m])), max_new=m)
    sb.cache_append(caches[1], table, lens, *(t.transpose(1, 2) for t in x))
    sb.cache_append(caches[2], table, lens, *(t.transpose(1, 2).contiguous() for t in x))
    for c in caches[1:]:
        for a, b in ((c.k, caches[0].k), (c.v, caches[0].v), (c.k_scale, caches[0].k_scale)):
            assert torch.equal(a, b)


def test_append_leaves_bad_pages_and_what_does_not_fit(sb):
    rng = np.random.default_rng(7)
    cache = sb.new_cache(4, 2, 32, "i8")
    want = pools_of(cache)
    table, lens = np.int32([[1, -1, 3], [99, 2, 0]]), np.int32([5, 40])
    cu = np.int32([0, 100, 164])                                     # both rows end behind the table's last page
    xs = [torch.from_numpy(tokens(rng, 164, 2)) for _ in range(2)]
    sb.cache_append(cache, dev(table), dev(lens), xs[0].cuda(), xs[1].cuda(), cu_new=dev(cu), max_new=100)
    # the pages that begin half full are empty here: scale 0, codes 0
    ref.append(want, table, lens, [x.double().numpy() for x in xs], cu, None)
    same_pools(cache, want)


# ------------------------------------------------------------------ attend

def check_attend(sb, rng, cache, table, lens, new, group, dtype, width=None, softcap=0.0, slopes=None, prefix=None, q_pos=None,
                 scale=None, q_scale=1.0):
    heads = cache.n_kv_heads
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    Q = torch.from_numpy((q_scale * rng.standard_normal((int(cu[-1]), heads * group, 128))).astype(np.float32)).to(DT[dtype])
    got, lse = sb.cache_attend(cache, dev(table), dev(np.int32(lens)), Q.cuda(), group, cu_q=dev(cu), max_q=max(new), scale=scale,
                               softcap=softcap, slopes=None if slopes is None else dev(slopes),
                               prefix=None if prefix is None else dev(np.int32(prefix)),
                               q_pos=None if q_pos is None else dev(np.int32(q_pos)), want_lse=True)
    want, want_lse, size, big = ref.attend(pools_of(cache), table, lens, Q.double().numpy(), cu, group, scale or 128 ** -0.5, softcap,
                                           slopes, prefix, q_pos)
    compare_attend(got, lse, want, want_lse, size, big, max(lens), dtype)
    return got, lse


def compare_attend(got, lse, want, want_lse, size, big, n, dtype):
    """A weight is off by its own rounding (f16: 2^-12, two f16: 2^-22), by twice its logit's error (products of a
    row of 128 and the steps to the exponent in f32: 2^-18 of the logits' size), sums of f32 by 2^-24 a step; then the output is rounded."""
    got, lse = got.double().cpu().numpy(), lse.double().cpu().numpy()
    weight = 2.0 ** (-21 if dtype == "f32" else -11) + 2 * 2.0 ** -18 * (1 + big[..., None]) + 2.0 ** -24 * (n / 64 + 64)
    tol = size * weight + np.abs(want) * float(torch.finfo(DT[dtype]).eps) / 2 + 1e-30
    if dtype == "f16":
        tol += 2.0 ** -25                                            # f16 numbers below 2^-14 are that far apart
    worst = np.abs(got - want) / tol
    assert (worst <= 1).all(), f"{worst.max()} times the bound at {np.unravel_index(worst.argmax(), worst.shape)}"
    seen = np.isfinite(want_lse)
    assert (np.isneginf(lse) == ~seen).all()
    assert (np.abs(lse[seen] - want_lse[seen]) <= 2.0 ** -18 * (1 + big[seen]) + 2.0 ** -20).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("page", [32, 64, 256])
def test_attend_single_tokens(sb, dtype, fmt, page):
    rng = np.random.default_rng(11)
    lens = [1, 31, 32, 33, 127, 128, 129, 500]
    cache, table = filled(sb, rng, lens, 2, page, fmt)
    check_attend(sb, rng, cache, table, lens, [1] * 8, 4, dtype, q_scale=3.0)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("group", [1, 3, 4, 8, 17])
def test_attend_pieces(sb, dtype, fmt, group):
    """Ragged numbers of new tokens: rows in tiles of 16, 32, 64 and several, a sequence without any, one of one token."""
    rng = np.random.default_rng(group)
    for new in ([1, 4, 0, 2], [9, 8, 1, 3], [70, 1, 33, 64]):
        lens = [n + e for n, e in zip(new, (0, 65, 10, 201))]
        cache, table = filled(sb, rng, lens, 2, 32, fmt)
        check_attend(sb, rng, cache, table, lens, new, group, dtype)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", list(DT))
def test_attend_options(sb, dtype, fmt):
    rng = np.random.default_rng(13)
    lens, new = [200, 77, 300], [40, 77, 5]
    cache, table = filled(sb, rng, lens, 2, 64, fmt)
    slopes = np.float32(2.0 ** -np.arange(1, 9))
    check_attend(sb, rng, cache, table, lens, new, 4, dtype, softcap=7.0, q_scale=4.0)
    check_attend(sb, rng, cache, table, lens, new, 4, dtype, slopes=slopes)
    check_attend(sb, rng, cache, table, lens, new, 4, dtype, prefix=[150, 40, 1000])
    check_attend(sb, rng, cache, table, lens, new, 4, dtype, prefix=[0, 77, 299], slopes=slopes, softcap=20.0, scale=0.3)
    check_attend(sb, rng, cache, table, lens, new, 4, dtype, q_pos=rng.integers(0, 5000, sum(new)), slopes=slopes)


@pytest.mark.parametrize("cap", [1e-42, 1e-3, 64.0, 65.0, 300.0, 1e4, 1e8, 1e20, 3e38])
@pytest.mark.parametrize("dtype", list(DT))
def test_attend_caps_of_any_size(sb, dtype, cap):
    """From caps that leave nothing of the logits to those that leave them as they are; few rows and many."""
    rng = np.random.default_rng(15)
    lens, new = [200, 40], [3, 40]
    cache, table = filled(sb, rng, lens, 2, 64, "e4m3")
    check_attend(sb, rng, cache, table, lens, new, 4, dtype, softcap=cap, q_scale=20.0)
    check_attend(sb, rng, cache, table, lens, [1, 2], 4, dtype, softcap=cap, q_scale=20.0)


@pytest.mark.parametrize("dtype", list(DT))
def test_attend_rows_that_see_nothing(sb, dtype):
    """Empty sequences, more queries than tokens, empty slots, absent pages."""
    rng = np.random.default_rng(17)
    lens = [0, 3, 100, 90]
    cache, table = filled(sb, rng, lens, 2, 32, "e4m3", positions=True)
    new = [2, 5, 3, 4]
    check_attend(sb, rng, cache, table, lens, new, 4, dtype)
    check_attend(sb, rng, cache, table, lens, new, 4, dtype, prefix=[5, 2, 0, 0])
    cache.pos[int(table[2, 0])] = -1                                 # slots without a token
    cache.pos[int(table[2, 2]), 1, ::3] = -1
    cache.pos[int(table[3, 0]):int(table[3, 0]) + 1, 1] = -7
    table[3, 1], table[3, 2] = -1, cache.n_pages
    got, lse = check_attend(sb, rng, cache, table, lens, new, 4, dtype, slopes=np.float32(0.01 * np.arange(8)))
    assert (got[:2] == 0).all() and torch.isneginf(lse[:2]).all()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", list(DT))
def test_attend_long_context_in_chunks(sb, dtype, fmt):
    """Few rows and many tokens: chunks are joined; a table that is wider than the sequences."""
    rng = np.random.default_rng(19)
    lens, new = [2500, 4, 1300], [1, 2, 3]
    cache, table = filled(sb, rng, lens, 1, 64, fmt, width=64)
    check_attend(sb, rng, cache, table, lens, new, 5, dtype, q_scale=2.0)
    check_attend(sb, rng, cache, table, lens, new, 5, dtype, softcap=9.0, prefix=[2500, 1, 1299])


@pytest.mark.parametrize("page", [32, 256])
@pytest.mark.parametrize("dtype", list(DT))
def test_attend_in_tables_far_wider_than_the_sequences(sb, dtype, page):
    """A server's tables have room for the longest context: lengths around the pieces of up to 1024 tokens that its chunks take
    in turn, one and a few new tokens (16 rows a workgroup), and enough of them for the kernel of many rows."""
    rng = np.random.default_rng(21)
    lens = [0, 1, 127, 128, 1023, 1024, 1025, 2048, 2500]
    cache, table = filled(sb, rng, lens, 1, page, "e4m3", width=131072 // page)
    check_attend(sb, rng, cache, table, lens, [1] * 9, 2, dtype)
    check_attend(sb, rng, cache, table, lens, [1, 2, 5, 3, 1, 9, 2, 4, 1], 2, dtype, slopes=np.float32([0.01, 0.002]))
    check_attend(sb, rng, cache, table, lens, [0, 1, 70, 3, 1, 40, 65, 0, 20], 2, dtype, softcap=20.0)


@pytest.mark.parametrize("dtype", list(DT))
def test_attend_pages_of_very_different_scales(sb, dtype):
    """Pages whose V differ by large factors, in rising and falling order, and a page of zeros."""
    rng = np.random.default_rng(23)
    for order in ([1, 1e-6, 1e4, 0, 1e-30], [1e4, 1, 1e-3, 1e-20, 0]):
        x = np.concatenate([tokens(rng, 64, 1) * np.float32(f) for f in order])
        k = np.concatenate([tokens(rng, 64, 1) * np.float32(min(f, 1.0)) for f in order])
        if dtype == "f16":
            x = np.clip(x, -6e4, 6e4)
        cache = sb.new_cache(8, 1, 64, "i8")
        table = np.int32([[3, 1, 4, 0, 6]])
        sb.cache_append(cache, dev(table), dev(np.int32([0])), dev(k), dev(x), cu_new=dev(np.int32([0, 320])), max_new=320)
        check_attend(sb, rng, cache, table, [320], [3], 4, dtype)


def test_attend_strides_and_given_buffers(sb):
    rng = np.random.default_rng(29)
    cache, table = filled(sb, rng, [300, 211], 2, 64, "e4m3")
    t, n = dev(table), dev(np.int32([300, 211]))
    wide = torch.from_numpy(rng.standard_normal((2, 3, 12, 256)).astype(np.float32)).half().cuda()
    Q = wide[:, :, 2:10, 128:]
    got = sb.cache_attend(cache, t, n, Q, 4)
    want = sb.cache_attend(cache, t, n, Q.contiguous(), 4)
    assert torch.equal(got, want)
    ragged = sb.cache_attend(cache, t, n, Q.contiguous().reshape(6, 8, 128), 4, cu_q=dev(np.int32([0, 3, 6])), max_q=3)
    assert torch.equal(ragged, want.reshape(6, 8, 128))
    out, lse = torch.empty_like(want), torch.empty(2, 3, 8, device="cuda")
    ws = torch.empty(sb.spindle_attend_workspace_bytes(cache.ref, 2, table.shape[1], 3, 6, 4, sb.F16), dtype=torch.uint8, device="cuda")
    back = sb.cache_attend(cache, t, n, Q, 4, out=out, lse=lse, workspace=ws)
    assert back[0] is out and back[1] is lse and torch.equal(out, want)


def test_attend_heavy_queries(sb):
    """One query's NaN or infinity stays in its own rows; large bf16 queries are no overflow."""
    rng = np.random.default_rng(31)
    cache, table = filled(sb, rng, [150], 1, 32, "e4m3")
    t, n = dev(table), dev(np.int32([150]))
    Q = torch.from_numpy(rng.standard_normal((1, 6, 4, 128)).astype(np.float32)).bfloat16().cuda()
    want = sb.cache_attend(cache, t, n, Q, 4)
    bad = Q.clone()
    bad[0, 2, 1, 7], bad[0, 3, 2, 9] = float("nan"), float("inf")
    got = sb.cache_attend(cache, t, n, bad, 4)
    spoiled = torch.zeros(6, 4, dtype=torch.bool, device="cuda")
    spoiled[2, 1] = spoiled[3, 2] = True
    assert torch.equal(got[0][~spoiled], want[0][~spoiled])
    assert torch.isnan(got[0, 2, 1]).all()
    huge = sb.cache_attend(cache, t, n, Q * 2.0 ** 100, 4, scale=2.0 ** -100 * 128 ** -0.5)
    assert torch.equal(huge, want)


def test_attend_on_another_stream_and_in_a_graph(sb):
    rng = np.random.default_rng(37)
    lens = [900, 40]
    cache, table = filled(sb, rng, lens, 2, 64, "i8")
    t, n = dev(table), dev(np.int32(lens))
    Q = torch.from_numpy(rng.standard_normal((2, 1, 8, 128)).astype(np.float32)).half().cuda()
    K, V = (torch.from_numpy(tokens(rng, 2, 2)).half().cuda().reshape(2, 2, 1, 128) for _ in range(2))
    before = n - 1
    sb.cache_append(cache, t, before, K, V)
    want = sb.cache_attend(cache, t, n, Q, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = sb.cache_attend(cache, t, n, Q, 4)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out = torch.empty_like(want)
    ws = torch.empty(sb.spindle_attend_workspace_bytes(cache.ref, 2, table.shape[1], 1, 2, 4, sb.F16), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sb.cache_append(cache, t, before, K, V)
        sb.cache_attend(cache, t, n, Q, 4, out=out, workspace=ws)
    for k in range(4):
        V.mul_(1.5)
        Q.mul_(0.9)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        graphed = out.clone()
        sb.cache_append(cache, t, before, K, V)
        assert torch.equal(graphed, sb.cache_attend(cache, t, n, Q, 4)), k


def test_calls_give_the_same_bits_again(sb):
    rng = np.random.default_rng(41)
    cache, table = filled(sb, rng, [5000], 2, 64, "e4m3")
    t, n = dev(table), dev(np.int32([5000]))
    Q = torch.from_numpy(rng.standard_normal((1, 3, 8, 128)).astype(np.float32)).cuda()
    first = sb.cache_attend(cache, t, n, Q, 4)
    for _ in range(5):
        assert torch.equal(sb.cache_attend(cache, t, n, Q, 4), first)


# ------------------------------------------------------------------ compact

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("page", [32, 128])
@pytest.mark.parametrize("positions", [False, True])
def test_compact(sb, fmt, page, positions):
    rng = np.random.default_rng(43)
    lens, n_kept, heads = [700, 45, 33, 5], [130, 45, 0, 1], 3
    cache, table = filled(sb, rng, lens, heads, page, fmt, positions=positions, spare=12)
    kept = np.full((4, heads, 140), -1, np.int32)
    for b, (n, k) in enumerate(zip(lens, n_kept)):
        for h in range(heads):
            kept[b, h, :k] = np.sort(rng.permutation(n)[:k])
    if positions:                                                    # heads that keep fewer tokens; entries that are none
        kept[0, 1, 100:] = -1
        kept[0, 2, 7], kept[1, 0, 3] = 700, 1 << 30
    free = np.setdiff1d(np.arange(cache.n_pages), table[table >= 0])
    need = [-(-k // page) for k in n_kept]
    out = np.full((4, max(need) + 1), -1, np.int32)
    at = 0
    for b, k in enumerate(need):
        out[b, :k] = free[at:at + k]
        at += k
    want = pools_of(cache)
    sb.cache_compact(cache, dev(table), dev(np.int32(lens)), dev(kept), dev(np.int32(n_kept)), dev(out))
    ref.compact(want, table, lens, kept, n_kept, out)
    same_pools(cache, want)
    check_attend(sb, rng, cache, out, n_kept, [1, 1, 0, 1], 2, "f16", slopes=np.float32([0.1, 0, 0.2, 0.01, 0.5, 0.3]) if positions else None)


def test_compact_keeps_equal_pages_as_they_are(sb):
    rng = np.random.default_rng(47)
    for fmt in FMTS:
        cache, table = filled(sb, rng, [64], 2, 64, fmt, spare=1)
        to = 1 - int(table[0, 0])
        kept = dev(np.tile(np.arange(64, dtype=np.int32), (1, 2, 1)))
        sb.cache_compact(cache, dev(table), dev(np.int32([64])), kept, dev(np.int32([64])), dev(np.int32([[to]])))
        assert torch.equal(cache.k[to], cache.k[1 - to])


# ------------------------------------------------------------------ pages

@pytest.mark.parametrize("page", [32, 256])
def test_pages_through_many_steps(sb, page):
    """Forks, growth, copies and releases in turn, against the plain bookkeeping; pages run out now and then."""
    rng = np.random.default_rng(page)
    n_pages, width, rows = 22, 9, 12
    refs = np.zeros(n_pages, np.int32)
    table, lens = np.full((rows, width), -1, np.int32), np.zeros(rows, np.int32)
    d_refs = dev(refs)
    lacked = 0
    for step in range(40):
        grow = np.where(rng.random(rows) < 0.6, rng.integers(0, 2 * page, rows), rng.integers(-1, 2, rows)).astype(np.int32)
        d_table, d_lens = dev(table), dev(lens)
        n, copies, status = sb.pages_reserve(d_refs, d_table, d_lens, dev(grow), page)
        want_n, want_copies, want_status = ref.reserve(refs, table, lens, grow, page)
        np.testing.assert_array_equal(status.cpu().numpy(), want_status, err_msg=f"step {step}")
        np.testing.assert_array_equal(n.cpu().numpy(), want_n)
        np.testing.assert_array_equal(copies.cpu().numpy(), want_copies)
        np.testing.assert_array_equal(d_table.cpu().numpy(), table)
        np.testing.assert_array_equal(d_refs.cpu().numpy(), refs)
        lens = want_n
        lacked += want_status.any()
        parent = rng.integers(0, rows, rows).astype(np.int32)
        parent[rng.random(rows) < 0.3] = -1
        parent[0] = rows + 3
        new_table, new_lens = sb.pages_share(d_refs, d_table, dev(lens), dev(parent), page)
        w_table, w_lens = ref.share(refs, table, lens, parent, page)
        sb.pages_release(d_refs, d_table, dev(lens), page)
        ref.release(refs, table, lens, page)
        np.testing.assert_array_equal(new_table.cpu().numpy(), w_table)
        np.testing.assert_array_equal(new_lens.cpu().numpy(), w_lens)
        np.testing.assert_array_equal(d_refs.cpu().numpy(), refs)
        table, lens = w_table, w_lens
    assert 0 < lacked < 40


def test_pages_of_many_rows_and_a_large_pool(sb):
    """More rows than threads, more pages than one pass looks at; every row shares one last page."""
    rng = np.random.default_rng(53)
    rows, n_pages, width, page = 1500, 50000, 4, 32
    refs = (rng.random(n_pages) < 0.5).astype(np.int32)
    lens = np.full(rows, 70, np.int32)
    own = rng.permutation(np.flatnonzero(refs))[:3]
    table = np.tile(np.int32([own[0], own[1], own[2], -1]), (rows, 1))
    refs[own] = rows
    grow = rng.integers(0, 50, rows).astype(np.int32)
    d_refs, d_table = dev(refs), dev(table)
    n, copies, status = sb.pages_reserve(d_refs, d_table, dev(lens), dev(grow), page)
    # the same, without looking for each free page anew
    free = iter(np.flatnonzero(refs == 0))
    left = rows
    for r in range(rows):
        if grow[r] > 0 and left > 1:
            table[r, 2] = next(free)
            refs[table[r, 2]] = 1
            left -= 1
        for j in range(3, -(-(70 + int(grow[r])) // page)):
            table[r, j] = next(free)
            refs[table[r, j]] = 1
    refs[own[2]] = left
    assert status.tolist() == [0, 0]
    np.testing.assert_array_equal(d_table.cpu().numpy(), table)
    np.testing.assert_array_equal(d_refs.cpu().numpy(), refs)
    np.testing.assert_array_equal(n.cpu().numpy(), lens + grow)
    moved = copies.cpu().numpy()[:, 0] >= 0
    np.testing.assert_array_equal(moved, table[:, 2] != own[2])
    assert (copies.cpu().numpy()[moved] == np.stack([np.full(moved.sum(), own[2]), table[moved, 2]], 1)).all()


@pytest.mark.parametrize("positions", [False, True])
def test_copy(sb, positions):
    rng = np.random.default_rng(59)
    cache, table = filled(sb, rng, [200, 100], 3, 64, "e4m3", positions=positions, spare=6)
    free = np.setdiff1d(np.arange(cache.n_pages), table[table >= 0])
    pairs = np.int32([[table[0, 1], free[0]], [-1, -1], [table[1, 0], free[1]], [table[0, 0], cache.n_pages], [cache.n_pages, free[2]]])
    pools = [p for p in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.pos) if p is not None]
    want = [p.clone() for p in pools]
    for p in want:
        p[free[0]], p[free[1]] = p[int(table[0, 1])], p[int(table[1, 0])]
    sb.cache_copy(cache, dev(pairs))
    for p, w in zip(pools, want):
        assert torch.equal(p.view(torch.uint8) if p.dtype == torch.uint8 else p.view(torch.int32), w.view(torch.uint8) if w.dtype == torch.uint8 else w.view(torch.int32))


# ------------------------------------------------------------------ with the eviction

def test_evicted_prompt_is_stored_and_attended(sb):
    """compress_deep's kept rows stored directly, and its kept indices compacted in the cache, are the same tokens."""
    rng = np.random.default_rng(61)
    B, H, G, l, budget = 2, 2, 4, 600, 96
    K, V = (torch.from_numpy(tokens(rng, B * H * l, 1).reshape(B, H, l, 128)).half().cuda() for _ in range(2))
    Qw = torch.from_numpy(rng.standard_normal((B, H * G, 32, 128)).astype(np.float32)).half().cuda()
    kept, K_out, V_out, _ = sb.compress_deep(K, V, Qw, G, "f16", 32, 7, budget)
    pages, page = -(-l // 32), 32
    cache = sb.new_cache(2 * pages + 2 * 3, H, page, "i8", positions=True)
    table = dev(np.arange(2 * pages, dtype=np.int32).reshape(2, pages))
    out = dev(np.arange(2 * pages, 2 * pages + 6, dtype=np.int32).reshape(2, 3))
    zero, lens, n_kept = (dev(np.int32([x, x])) for x in (0, l, budget))
    sb.cache_append(cache, table, zero, K, V)
    sb.cache_compact(cache, table, lens, kept, n_kept, out)
    where = cache.pos[out.long()].transpose(1, 2).reshape(B, H, 96)
    assert torch.equal(where, kept)
    q = torch.from_numpy(rng.standard_normal((B, 1, H * G, 128)).astype(np.float32)).half().cuda()
    got = sb.cache_attend(cache, out, n_kept, q, G).float()
    direct = sb.new_cache(6, H, page, "i8")
    t2 = dev(np.arange(6, dtype=np.int32).reshape(2, 3))
    sb.cache_append(direct, t2, zero, K_out, V_out)
    once = sb.cache_attend(direct, t2, n_kept, q, G).float()
    # two roundings of the codes against one: a step of the integers is 1/127 of a page's largest value
    step = (direct.v_scale.max() * 1.5).item()
    assert (got - once).abs().max().item() < 3 * step


# ------------------------------------------------------------------ larger pools, and all of it together

def test_pools_beyond_32_bits(sb):
    """Pages whose bytes lie behind the first 4 GiB of a pool."""
    rng = np.random.default_rng(67)
    n_pages, H, page = 17000, 8, 256                                  # 4.5e9 bytes of K, as many of V
    k, v = (torch.empty((n_pages, H, page, 128), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((n_pages, H), dtype=torch.float32, device="cuda") for _ in range(2))
    cache = sb.Cache(k, v, ks, vs, None, page, "i8")
    last = np.int32([[n_pages - 1, n_pages - 3, 16500]])
    x = [torch.from_numpy(tokens(rng, 700, H)).half() for _ in range(2)]
    sb.cache_append(cache, dev(last), dev(np.int32([0])), x[0].cuda(), x[1].cuda(), cu_new=dev(np.int32([0, 700])), max_new=700)
    near = sb.new_cache(6, H, page, "i8")
    low = np.int32([[0, 1, 2]])
    sb.cache_append(near, dev(low), dev(np.int32([0])), x[0].cuda(), x[1].cuda(), cu_new=dev(np.int32([0, 700])), max_new=700)
    for a, b in ((cache.k, near.k), (cache.v, near.v), (cache.k_scale, near.k_scale), (cache.v_scale, near.v_scale)):
        assert torch.equal(a[dev(last[0]).long()], b[:3])
    n = dev(np.int32([700]))
    for m in (1, 5, 200):
        q = torch.from_numpy(rng.standard_normal((1, m, H * 4, 128)).astype(np.float32)).half().cuda()
        assert torch.equal(sb.cache_attend(cache, dev(last), n, q, 4), sb.cache_attend(near, dev(low), n, q, 4))
    kept = dev(np.sort(rng.permuted(np.tile(np.arange(700, dtype=np.int32), (1, H, 1)), axis=2)[:, :, :300], axis=2))
    sb.cache_compact(cache, dev(last), n, kept, dev(np.int32([300])), dev(np.int32([[16999 - 1, 16400]])))
    sb.cache_compact(near, dev(low), n, kept, dev(np.int32([300])), dev(np.int32([[3, 4]])))
    assert torch.equal(cache.k[16998], near.k[3]) and torch.equal(cache.v[16400], near.v[4])
    sb.cache_copy(cache, dev(np.int32([[16998, 16450]])))
    assert torch.equal(cache.v[16450], near.v[3])


@pytest.mark.parametrize("fmt", FMTS)
def test_many_rows_of_a_long_context(sb, fmt):
    """A piece of a prompt over what is stored (the kernel for many rows, tokens in chunks) against single tokens, each with its
    own length, which the plain implementation holds above."""
    rng = np.random.default_rng(71)
    n, m, G = 3000, 150, 4
    cache, table = filled(sb, rng, [n], 2, 64, fmt)
    t = dev(table)
    for dtype in ("f16", "bf16"):
        Q = torch.from_numpy(rng.standard_normal((1, m, 8, 128)).astype(np.float32)).to(DT[dtype]).cuda()
        got, lse = sb.cache_attend(cache, t, dev(np.int32([n])), Q, G, want_lse=True)
        for i in (0, 1, 70, m - 2, m - 1):
            one, one_lse = sb.cache_attend(cache, t, dev(np.int32([n - m + i + 1])), Q[:, i:i + 1].contiguous(), G, want_lse=True)
            # both are within their own bounds of the truth: twice the weights' and logits' share, and a step of the output
            size = float(one.abs().max())
            np.testing.assert_allclose(got[0, i].float().cpu(), one[0, 0].float().cpu(), rtol=2 * float(torch.finfo(DT[dtype]).eps), atol=size * 2.0 ** -8)
            np.testing.assert_allclose(lse[0, i].cpu(), one_lse[0, 0].cpu(), rtol=0, atol=2.0 ** -11)


def test_example_serves_from_the_cache(sb):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_from_cache.py")
    spec = importlib.util.spec_from_file_location("serve_from_cache", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    out, pages, _ = ex.serve(prompt=700, budget=200, branches=3, steps=70)
    assert out.shape == (70, 3, 128) and torch.isfinite(out.float()).all()
    # 11 pages of the prompt, 4 of the budget (200 tokens), then each branch its copy of the last one and one more
    assert pages == [11, 4, 3 + 3 * 2]
    again = ex.serve(prompt=700, budget=200, branches=3, steps=70)[0]
    assert torch.equal(out, again)
    # the same text through integers: the codes' steps are all that differs
    other = ex.serve(prompt=700, budget=200, branches=3, steps=4, fmt="i8")[0].float()
    assert (other[0] - out[0].float()).abs().max() < 0.25


# ------------------------------------------------------------------ compaction at the ends of the numbers

@pytest.mark.parametrize("fmt", FMTS)
def test_compact_of_zeros_from_pages_of_large_values(sb, fmt):
    """A new page whose kept tokens are zeros (zero vectors, NaN stored as zeros) has the smallest scale, and its pages' scales
    over that one are no number."""
    rng = np.random.default_rng(73)
    x = tokens(rng, 128, 2) * np.float32(1e4)
    x[40:50], x[100:110] = 0, np.nan
    cache = sb.new_cache(4, 2, 64, fmt)
    table, out = np.int32([[1, 3]]), np.int32([[2]])
    sb.cache_append(cache, dev(table), dev(np.int32([0])), dev(x), dev(x[::-1]), cu_new=dev(np.int32([0, 128])), max_new=128)
    zeros = np.r_[40:50, 100:110]                                     # of K; mirrored ones of V
    kept = np.int32([[zeros, np.r_[0:20]]])
    want = pools_of(cache)
    sb.cache_compact(cache, dev(table), dev(np.int32([128])), dev(kept), dev(np.int32([20])), dev(out))
    ref.compact(want, table, [128], kept, [20], out)
    same_pools(cache, want)
    assert (cache.k[2, 0] == 0).all() and cache.k_scale[2, 0].item() == ref.TINY and cache.v_scale[2, 0].item() > 1


@pytest.mark.parametrize("fmt", FMTS)
def test_compact_of_the_largest_numbers(sb, fmt):
    """127 times a scale made of the largest number is none any more; the scale of the new page has to stay one."""
    rng = np.random.default_rng(79)
    x = tokens(rng, 64, 1)
    x[5, 0, 7], x[6, 0, 8] = np.finfo(np.float32).max, -np.finfo(np.float32).max
    cache = sb.new_cache(2, 1, 64, fmt)
    sb.cache_append(cache, dev(np.int32([[1]])), dev(np.int32([0])), dev(x), dev(-x), cu_new=dev(np.int32([0, 64])), max_new=64)
    sb.cache_compact(cache, dev(np.int32([[1]])), dev(np.int32([64])), dev(np.arange(64, dtype=np.int32).reshape(1, 1, 64)), dev(np.int32([64])),
                     dev(np.int32([[0]])))
    for codes, scale in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        assert torch.equal(codes[0], codes[1]) and torch.equal(scale[0], scale[1])
        assert torch.isfinite(scale).all() and (codes[0, 0, 5:7, 7:9] != 0).any()


# ------------------------------------------------------------------ attention: layouts, scales of any kind, far pages, precision

def test_attend_queries_whose_dimensions_of_one_entry_have_any_stride(sb):
    """One token a sequence, out of [B, Hq, 1, d] (a decode step's usual order) or out of a longer piece; one head; one sequence."""
    rng = np.random.default_rng(83)
    cache, table = filled(sb, rng, [300, 211, 70], 2, 64, "e4m3")
    t, n = dev(table), dev(np.int32([300, 211, 70]))
    Q = torch.from_numpy(rng.standard_normal((3, 1, 8, 128)).astype(np.float32)).half().cuda()
    want, want_lse = sb.cache_attend(cache, t, n, Q, 4, want_lse=True)
    turned = torch.empty((3, 8, 1, 128), dtype=torch.float16, device="cuda").copy_(Q.transpose(1, 2)).transpose(1, 2)
    assert turned.stride() == (1024, 128, 128, 1)
    piece = torch.zeros((3, 5, 8, 128), dtype=torch.float16, device="cuda")
    piece[:, 4:] = Q
    for q in (turned, piece[:, 4:], Q.as_strided((3, 1, 8, 128), (1024, 3, 128, 1))):
        got, lse = sb.cache_attend(cache, t, n, q, 4, want_lse=True)
        assert torch.equal(got, want) and torch.equal(lse, want_lse)
    one = sb.cache_attend(cache, t[:1], n[:1], Q[:1].as_strided((1, 1, 8, 128), (7, 5, 128, 1)), 4)
    assert torch.equal(one, want[:1])
    ragged = sb.cache_attend(cache, t[:1], n[:1], Q[:1, 0].as_strided((1, 8, 128), (3, 128, 1)), 4, cu_q=dev(np.int32([0, 1])), max_q=1)
    assert torch.equal(ragged, want[:1, 0])
    single, rows = filled(sb, rng, [40, 90], 1, 64, "i8")
    t, n = dev(rows), dev(np.int32([40, 90]))
    q = torch.from_numpy(rng.standard_normal((2, 3, 1, 128)).astype(np.float32)).half().cuda()
    want = sb.cache_attend(single, t, n, q, 1)
    assert torch.equal(sb.cache_attend(single, t, n, q.as_strided((2, 3, 1, 128), (384, 128, 5, 1)), 1), want)


def test_append_of_k_and_v_in_layouts_of_their_own(sb):
    """K as a rotation leaves it and V as a part of a wider projection; dimensions of one entry, whose strides mean nothing."""
    rng = np.random.default_rng(89)
    B, H, m = 3, 4, 21
    wide = torch.from_numpy(rng.standard_normal((B, m, 3 * H, 128)).astype(np.float32)).half().cuda()
    K, V = wide[:, :, H:2 * H].transpose(1, 2).contiguous(), wide[:, :, 2 * H:].transpose(1, 2)
    table, lens = dev(table_of(rng, [2, 2, 2], 2, 8)), dev(np.int32([0, 3, 19]))

    def stored(k, v, at=lens, **kw):
        cache = sb.new_cache(8, H, 32, "i8")
        sb.cache_append(cache, table, at, k, v, **kw)
        return [cache.k, cache.v, cache.k_scale, cache.v_scale]

    def same(a, b):
        assert all(torch.equal(x, y) for x, y in zip(a, b))

    want = stored(K, V.contiguous())
    same(stored(K, V), want)
    same(stored(V.contiguous(), K.transpose(1, 2).contiguous().transpose(1, 2)), [want[1], want[0], want[3], want[2]])
    cu = dev(np.int32([0, m, 2 * m, 3 * m]))
    rows = [x.transpose(1, 2).reshape(B * m, H, 128) for x in (K, V)]
    same(stored(rows[0], wide.view(B * m, 3 * H, 128)[:, 2 * H:], cu_new=cu, max_new=m), want)
    # one token a sequence: one and the same memory has many strides
    k, v = K[:, :, :1].contiguous(), V[:, :, :1].contiguous()
    want = stored(k, v)
    turned = torch.empty((B, 1, H, 128), dtype=torch.float16, device="cuda").copy_(v.transpose(1, 2)).transpose(1, 2)
    assert turned.stride() != k.stride()
    same(stored(k, turned), want)
    same(stored(k.as_strided((B, H, 1, 128), (H * 128, 128, 3, 1)), v), want)
    # one token in all
    same(stored(k[:1, :, 0].as_strided((1, H, 128), (5, 128, 1)), v[:1, :, 0], at=lens, cu_new=dev(np.int32([0, 1, 1, 1])), max_new=1),
         stored(k[:1, :, 0].clone(), v[:1, :, 0].clone(), at=lens, cu_new=dev(np.int32([0, 1, 1, 1])), max_new=1))


def test_calls_without_tokens(sb):
    rng = np.random.default_rng(131)
    cache, table = filled(sb, rng, [40, 90], 2, 64, "i8")
    t, n, before = dev(table), dev(np.int32([40, 90])), pools_of(cache)
    q, kv = torch.empty((2, 0, 8, 128), dtype=torch.float16, device="cuda"), torch.empty((2, 2, 0, 128), device="cuda")
    assert sb.cache_attend(cache, t, n, q, 4).shape == (2, 0, 8, 128)
    out, lse = sb.cache_attend(cache, t, n, q.view(0, 8, 128), 4, cu_q=dev(np.int32([0, 0, 0])), want_lse=True)
    assert out.shape == (0, 8, 128) and lse.shape == (0, 8)
    sb.cache_append(cache, t, n, kv, kv)
    sb.cache_append(cache, t, n, kv.view(0, 2, 128), kv.view(0, 2, 128), cu_new=dev(np.int32([0, 0, 0])))
    sb.cache_copy(cache, torch.empty((0, 2), dtype=torch.int32, device="cuda"))
    same_pools(cache, before)


@pytest.mark.parametrize("dtype,m", [("f16", 3), ("bf16", 40), ("f32", 3)])
def test_attend_leaves_sequences_whose_queries_lie_outside(sb, dtype, m):
    """Starts that are negative, behind the queries, or so large that the sum with a count wraps around: nothing is read or written
    for them (sequences in chunks and whole ones)."""
    rng = np.random.default_rng(137)
    lens, top = [1200, 70, 1200], 2 ** 31 - 1
    for width in (64, 20):
        cache, table = filled(sb, rng, lens, 1, 64, "e4m3", width=width)
        Q = torch.from_numpy(rng.standard_normal((m, 4, 128)).astype(np.float32)).to(DT[dtype]).cuda()
        want = sb.cache_attend(cache, dev(table[1:2]), dev(np.int32(lens[1:2])), Q, 4, cu_q=dev(np.int32([0, m])), max_q=m)
        for cu in ([-5, 0, m, m + 2], [m + 1, 0, m, top], [-2 ** 31, 0, m, m + 1], [top, -2 ** 31 + 5, top]):
            out, lse, B = torch.full_like(Q, 9.0), torch.full((m, 4), 9.0, device="cuda"), len(cu) - 1
            sb.cache_attend(cache, dev(table[:B]), dev(np.int32(lens[:B])), Q, 4, cu_q=dev(np.int32(cu)), max_q=m, out=out, lse=lse)
            if B == 2:
                assert (out == 9).all() and (lse == 9).all()
            else:                                                    # (another number of chunks: two results within their bounds)
                assert (out - want).abs().max().item() <= max(2 * float(torch.finfo(DT[dtype]).eps), 2.0 ** -16) * want.abs().max().item(), cu


@pytest.mark.parametrize("dtype", list(DT))
def test_attend_scales_that_are_no_powers_of_two(sb, dtype):
    """A code stands for code times scale, whatever the scale of a pool that somebody else filled; few rows and many."""
    rng = np.random.default_rng(97)
    lens = [130, 300]
    cache, table = filled(sb, rng, lens, 2, 64, "e4m3")
    for scale in (cache.k_scale, cache.v_scale):
        scale.mul_(dev(rng.uniform(1, 2, scale.shape).astype(np.float32)))
    check_attend(sb, rng, cache, table, lens, [1, 2], 4, dtype)
    check_attend(sb, rng, cache, table, lens, [40, 25], 4, dtype)
    cache.v_scale.fill_(2.0 ** -126 * 0.75)                           # below the smallest normal number
    cache.k_scale.fill_(1.5)
    got, _ = check_attend(sb, rng, cache, table, lens, [40, 25], 4, dtype)
    assert torch.isfinite(got.float()).all()


@pytest.mark.parametrize("new", [3, 40])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", list(DT))
def test_attend_beside_a_page_of_far_larger_values_that_gets_no_weight(sb, dtype, fmt, new):
    """The first page's V is some 10^9 times the others', and a bias by distance leaves it nothing: what the others give keeps its
    bits."""
    rng = np.random.default_rng(103)
    n = 320
    K, V = tokens(rng, n, 2), tokens(rng, n, 2)
    V[:64] *= np.float32(2e9)
    cache = sb.new_cache(6, 2, 64, fmt)
    table = np.int32([[3, 0, 4, 1, 5]])
    sb.cache_append(cache, dev(table), dev(np.int32([0])), dev(K), dev(V), cu_new=dev(np.int32([0, n])), max_new=n)
    check_attend(sb, rng, cache, table, [n], [new], 4, dtype, slopes=np.full(8, 0.5, np.float32))
    # the same within one step of 64 tokens: the second page of 32 gets nearly all the weight
    V = tokens(rng, n, 2)
    V[:32] *= np.float32(2e9)
    cache = sb.new_cache(12, 2, 32, fmt)
    table = table_of(rng, [10], 10, 12)
    sb.cache_append(cache, dev(table), dev(np.int32([0])), dev(K), dev(V), cu_new=dev(np.int32([0, n])), max_new=n)
    check_attend(sb, rng, cache, table, [n], [new], 4, dtype, slopes=np.full(8, 2, np.float32), q_pos=np.full(new, 63))


@pytest.mark.parametrize("new", [2, 40])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", list(DT))
def test_attend_weights_hold_their_bits(sb, dtype, fmt, new):
    """Two tokens of opposite V and nearly equal weights: the output is the difference of the weights, where their own rounding
    is not hidden by the output's.  16-bit queries: two bf16, half a step of the second is 2^-16 of a weight; f32: three, whose
    rounding is behind that of the sums.  In f32 and relative to the weights: 3 x 128 products of a logit (2^-23 of their size
    each, matrix instructions may cut off), two logits; exponential, factors, sums and quotient some 2^-23 each, 2^-20 in all."""
    rng = np.random.default_rng(107)
    K, V = tokens(rng, 2, 2), tokens(rng, 2, 2)
    V[1] = -V[0]
    cache = sb.new_cache(2, 2, 32, fmt)
    table, lens, cu = np.int32([[1]]), np.int32([2]), np.int32([0, new])
    sb.cache_append(cache, dev(table), dev(np.int32([0])), dev(K), dev(V), cu_new=dev(np.int32([0, 2])), max_new=2)
    Q = torch.from_numpy((1e-3 * rng.standard_normal((new, 8, 128))).astype(np.float32)).to(DT[dtype])
    got = sb.cache_attend(cache, dev(table), dev(lens), Q.cuda(), 4, cu_q=dev(cu), max_q=new, prefix=dev(np.int32([2])))
    want, _, size, big = ref.attend(pools_of(cache), table, lens, Q.double().numpy(), cu, 4, 128 ** -0.5, prefix=[2])

    def bound(bits):
        rounding = np.abs(want) * float(torch.finfo(DT[dtype]).eps) / 2 + (2.0 ** -25 if dtype == "f16" else 1e-30)
        return size * (bits + 2 * 384 * 2.0 ** -23 * big[..., None] + 2.0 ** -20) + rounding

    tol = bound(0.0 if dtype == "f32" else 2.0 ** -16)
    worst = (np.abs(got.double().cpu().numpy() - want) / tol).max()
    assert worst <= 1, f"{worst} times the bound"
    # the bound tells one operand less apart: weights p and 1 - p of V and -V, the larger one counted as 1
    x = pools_of(cache)
    v = np.repeat(x.x[1][1, :, 0] * x.s[1][1, :, None], 4, axis=0)
    less = np.zeros_like(want)
    for i in range(new):
        for h in range(8):
            p = np.clip((1 + want[i, h, np.abs(v[h]).argmax()] / v[h][np.abs(v[h]).argmax()]) / 2, 0, 1)
            w = np.array([p, 1 - p]) / max(p, 1 - p)
            step = 2.0 ** np.floor(np.log2(w)) * (2.0 ** -7 if dtype != "f32" else 2.0 ** -15)
            w = np.rint(w / step) * step
            less[i, h] = v[h] * (w[0] - w[1]) * max(p, 1 - p)
    assert (np.abs(less - want) > tol).any()


@pytest.mark.parametrize("new", [3, 40])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", list(DT))
def test_attend_largest_numbers_in_masked_places(sb, dtype, fmt, new):
    """The last token's V holds the largest numbers; the rows before do not see it, whether they share a step with it or a wave
    only."""
    rng = np.random.default_rng(101)
    n = 516
    K, V = (dev(tokens(rng, n, 2)) for _ in range(2))
    V[n - 1] = torch.finfo(torch.float32).max
    cache = sb.new_cache(18, 2, 32, fmt)
    table = table_of(rng, [17], 17, 18)
    sb.cache_append(cache, dev(table), dev(np.int32([0])), K, V, cu_new=dev(np.int32([0, n])), max_new=n)
    Q = torch.from_numpy(rng.standard_normal((new, 8, 128)).astype(np.float32)).to(DT[dtype])
    cu = np.int32([0, new])
    got, lse = sb.cache_attend(cache, dev(table), dev(np.int32([n])), Q.cuda(), 4, cu_q=dev(cu), max_q=new, want_lse=True)
    want = ref.attend(pools_of(cache), table, [n], Q.double().numpy(), cu, 4, 128 ** -0.5)
    compare_attend(got[:-1], lse[:-1], *(x[:-1] for x in want), n, dtype)


# ------------------------------------------------------------------ the kernel for many rows: what the tests above show with few

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_many_rows_with_positions_empty_slots_and_absent_pages(sb, dtype, fmt):
    rng = np.random.default_rng(109)
    lens, new = [0, 3, 170, 90, 300], [40, 45, 44, 50, 41]
    cache, table = filled(sb, rng, lens, 2, 32, fmt, positions=True)
    where = np.cumsum(rng.integers(1, 5, (cache.n_pages, 2, 32)), axis=2).astype(np.int32)   # gaps, other ones for each head
    for b, n in enumerate(lens):
        for j in range(-(-n // 32)):
            cache.pos[int(table[b, j])] = dev(where[0] + 130 * j)
    slopes, q_pos = np.float32(0.003 * np.arange(8)), rng.integers(0, 1500, sum(new))
    check_attend(sb, rng, cache, table, lens, new, 4, dtype, slopes=slopes, q_pos=q_pos)
    check_attend(sb, rng, cache, table, lens, new, 4, dtype, prefix=[5, 2, 0, 0, 290])
    cache.pos[int(table[2, 0])] = -1                                 # slots without a token
    cache.pos[int(table[2, 2]), 1, ::3] = -1
    cache.pos[int(table[3, 0]), 1] = -7
    cache.pos[int(table[4, 3]), 0, 5:] = -1
    table[3, 1], table[3, 2], table[4, 8] = -1, cache.n_pages, -5
    got, lse = check_attend(sb, rng, cache, table, lens, new, 4, dtype, slopes=slopes, q_pos=q_pos)
    assert (got[:40] == 0).all() and torch.isneginf(lse[:40]).all()
    check_attend(sb, rng, cache, table, lens, new, 4, dtype, softcap=6.0, q_scale=4.0)
    # the same pages without positions
    plain = sb.Cache(cache.k, cache.v, cache.k_scale, cache.v_scale, None, 32, fmt)
    check_attend(sb, rng, plain, table, lens, new, 4, dtype)
    check_attend(sb, rng, plain, table, lens, new, 4, dtype, softcap=6.0, prefix=[0, 3, 100, 90, 7])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_many_rows_over_pages_of_very_different_scales(sb, dtype, fmt):
    rng = np.random.default_rng(113)
    for order in ([1, 1e-6, 1e4, 0, 1e-30], [1e4, 1, 1e-3, 1e-20, 0], [1e-30, 1e-20, 1e-3, 1, 30]):
        x = np.concatenate([tokens(rng, 64, 1) * np.float32(f) for f in order])
        k = np.concatenate([tokens(rng, 64, 1) * np.float32(min(f, 1.0)) for f in order])
        if dtype == "f16":
            x = np.clip(x, -6e4, 6e4)
        cache = sb.new_cache(8, 1, 64, fmt)
        table = np.int32([[3, 1, 4, 0, 6]])
        sb.cache_append(cache, dev(table), dev(np.int32([0])), dev(k), dev(x), cu_new=dev(np.int32([0, 320])), max_new=320)
        check_attend(sb, rng, cache, table, [320], [40], 4, dtype)
        check_attend(sb, rng, cache, table, [320], [320], 4, dtype)   # rows that see one page only, or two


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_many_rows_heavy_queries(sb, dtype, fmt):
    """One query's NaN or infinity stays in its own rows; large bf16 queries are no overflow."""
    rng = np.random.default_rng(127)
    cache, table = filled(sb, rng, [150], 1, 32, fmt)
    t, n = dev(table), dev(np.int32([150]))
    Q = torch.from_numpy(rng.standard_normal((1, 40, 4, 128)).astype(np.float32)).to(DT[dtype]).cuda()
    want = sb.cache_attend(cache, t, n, Q, 4)
    bad = Q.clone()
    bad[0, 2, 1, 7], bad[0, 33, 2, 9] = float("nan"), float("inf")
    got = sb.cache_attend(cache, t, n, bad, 4)
    spoiled = torch.zeros(40, 4, dtype=torch.bool, device="cuda")
    spoiled[2, 1] = spoiled[33, 2] = True
    assert torch.equal(got[0][~spoiled], want[0][~spoiled])
    assert torch.isnan(got[0, 2, 1]).all()
    if dtype == "bf16":
        assert torch.equal(sb.cache_attend(cache, t, n, Q * 2.0 ** 100, 4, scale=2.0 ** -100 * 128 ** -0.5), want)


@pytest.mark.parametrize("dtype", list(DT))
def test_attend_small_caps_over_large_keys(sb, dtype):
    """A product of zero stays zero, however large the quotient of K's scale and the cap is."""
    rng = np.random.default_rng(139)
    n = 70
    K, V = (dev(tokens(rng, n, 2)) for _ in range(2))
    cache = sb.new_cache(3, 2, 32, "i8")
    table = np.int32([[2, 0, 1]])
    sb.cache_append(cache, dev(table), dev(np.int32([0])), K * 1e15, V, cu_new=dev(np.int32([0, n])), max_new=n)
    for new in (3, 40):
        Q = torch.from_numpy(rng.standard_normal((new, 8, 128)).astype(np.float32)).to(DT[dtype])
        Q[::2] = 0
        cu = np.int32([0, new])
        got, lse = sb.cache_attend(cache, dev(table), dev(np.int32([n])), Q.cuda(), 4, cu_q=dev(cu), max_q=new, softcap=1e-30, want_lse=True)
        # logits of at most 1e-30 are none
        want = ref.attend(pools_of(cache), table, [n], Q.double().numpy() * 0, cu, 4, 128 ** -0.5)
        compare_attend(got, lse, *want, n, dtype)
