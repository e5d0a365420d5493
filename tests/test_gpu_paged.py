"""The paged-cache operators on the GPU against their plain 64-bit forms, within
the bounds of tests/paged_util.py."""
import numpy as np
import pytest
import torch

from paper_2606_00422_amd import upr
from tests.gpu_util import say
from tests.paged_util import EPS, Pages, attend, frequencies, normal, offsets, rotate

pytestmark = pytest.mark.gpu


def assert_close(got, want, bound, label):
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all(np.isfinite(want))
    over = ~(err <= bound)
    assert not over.any(), (f"{label}: {over.sum()} of {over.size} outside the bound, worst error {np.nanmax(err):.3e} "
                            f"at {np.argwhere(over)[0]}, bound {bound[tuple(np.argwhere(over)[0])]:.3e}")


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads,dim,rot", [(8, 64, 64), (3, 64, 32), (1, 32, 10), (5, 128, 128), (7, 128, 2), (4, 32, 16)])
def test_rope(kind, layout, heads, dim, rot):
    say(f"[gpu] rope {kind} {layout} {heads}x{dim} rot {rot}")
    rng = np.random.default_rng([heads, dim, rot])
    for rows, scaling in [(1, "none"), (77, "by_parts"), (1030, "linear")]:
        spec = dict(base=500000.0, scaling=scaling, factor=4.0, original_length=2048)
        r = upr.rope(rot, layout=layout, **spec)
        f, mag = frequencies(rot, **spec)
        x, xv = normal(rng, kind, rows, heads, dim)
        pos = rng.integers(-(1 << 20), 1 << 20, rows).astype(np.int32)
        pos[0] = (1 << 31) - 1 if rows > 1 else 0
        got = upr.rope_apply(x, torch.from_numpy(pos).cuda(), r)
        want, err = rotate(xv, pos, layout, f, mag)
        assert_close(got, want, err + EPS[kind] * (np.abs(want) + err), f"{rows} rows")
        assert torch.equal(got[..., rot:], x[..., rot:])
        same = upr.rope_apply(x, torch.from_numpy(pos).cuda(), r, out=x)
        assert same is x and torch.equal(x, got)


def test_rope_of_strided_rows_and_no_rows():
    rng = np.random.default_rng(5)
    big, bv = normal(rng, "bf16", 33, 6, 64)
    x = big[:, 2:4]                                     # heads 2 and 3 of wider rows
    pos = torch.arange(33, dtype=torch.int32, device="cuda")
    r = upr.rope(64)
    before = big.clone()
    got = upr.rope_apply(x, pos, r)
    want, err = rotate(bv[:, 2:4], np.arange(33), "half", *frequencies(64))
    assert_close(got, want, err + EPS["bf16"] * (np.abs(want) + err), "strided")
    upr.rope_apply(x, pos, r, out=x)
    assert torch.equal(x, got) and torch.equal(big[:, :2], before[:, :2]) and torch.equal(big[:, 4:], before[:, 4:])
    empty = upr.rope_apply(x[:0], pos[:0], r)
    assert tuple(empty.shape) == (0, 2, 64)


# ---------------------------------------------------------------------------
# Append
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dim,page,rot,layout,with_q", [
    (8, 8, 64, 64, 64, "half", True), (4, 1, 128, 16, 64, "interleaved", True), (6, 2, 32, 32, 6, "half", False),
    (2, 2, 32, 1024, 0, "half", True), (14, 2, 64, 16, 64, "interleaved", True),
])
def test_append(kind, heads, kv, dim, page, rot, layout, with_q):
    say(f"[gpu] append {kind} {heads}/{kv}x{dim} page {page} rot {rot}")
    rng = np.random.default_rng([heads, kv, dim, page])
    counts = [1, 0, 17, 130, 1, 16, 3]
    before = [0, 40, 15, 3, 1024, 16, 77]
    rows = np.asarray([b + c for b, c in zip(before, counts)], np.int32)
    pages = Pages(rng, kind, before, kv, dim, page, spare_rows=max(counts))
    off = offsets(counts, first=5)
    n = int(off[-1])
    k, kv_ = normal(rng, kind, n, kv, dim)
    v, _ = normal(rng, kind, n, kv, dim)
    q, qv = normal(rng, kind, n, heads, dim)
    r = upr.rope(rot, layout=layout) if rot else None
    f, mag = frequencies(rot) if rot else (np.zeros(0), 1.0)
    want_data = pages.data.clone()
    q_out = torch.full_like(q, 7.0)
    upr.paged_append(pages.cache(), off, rows, k, v, rope=r, q=q if with_q else None, q_out=q_out if with_q else None)
    torch.cuda.synchronize()
    pos = np.concatenate([np.arange(b, b + c) for b, c in zip(before, counts)])
    user = np.repeat(np.arange(len(counts)), counts)
    assert_rotated = lambda got, x: (lambda w: assert_close(got, w[0], w[1] + EPS[kind] * (np.abs(w[0]) + w[1]), "turned"))(
        rotate(x, pos, layout, f, mag))
    page_of, slot = pages.tables[user, pos // page], pos % page
    got_k = pages.data[page_of, 0, :, slot]
    if rot:
        assert_rotated(got_k, kv_[off[0]:])
    else:
        assert torch.equal(got_k, k[off[0]:])
    assert torch.equal(pages.data[page_of, 1, :, slot], v[off[0]:])
    # nothing else is written: other places of the pages, rows before the first
    want_data[page_of, :, :, slot] = pages.data[page_of, :, :, slot]
    assert torch.equal(pages.data.view(torch.uint8), want_data.view(torch.uint8))
    if with_q:
        if rot:
            assert_rotated(q_out[off[0]:], qv[off[0]:])
        else:
            assert torch.equal(q_out[off[0]:], q[off[0]:])
        assert bool((q_out[:off[0]] == 7.0).all())


def test_append_of_many_users_from_fused_rows():
    """More users than one launch takes, q | k | v side by side, queries in place."""
    rng = np.random.default_rng(8)
    U, H, D, page = 300, 2, 64, 16
    counts = rng.integers(0, 4, U)
    rows = (counts + rng.integers(0, 50, U)).astype(np.int32)
    pages = Pages(rng, "bf16", rows, H, D, page)
    off = offsets(counts)
    qkv, val = normal(rng, "bf16", int(off[-1]), 3 * H, D)
    before = qkv.clone()
    r = upr.rope(64)
    upr.paged_append(pages.cache(), off, rows, qkv[:, H:2 * H], qkv[:, 2 * H:], rope=r, q=qkv[:, :H], q_out=qkv[:, :H])
    user = np.repeat(np.arange(U), counts)
    pos = np.arange(off[-1]) - off[user] + rows[user] - counts[user]
    want, err = rotate(val[:, :2 * H], pos, "half", *frequencies(64))
    bound = err + EPS["bf16"] * (np.abs(want) + err)
    assert_close(qkv[:, :H], want[:, :H], bound[:, :H], "q")
    where = (pages.tables[user, pos // page], pos % page)
    assert_close(pages.data[where[0], 0, :, where[1]], want[:, H:], bound[:, H:], "k")
    assert torch.equal(pages.data[where[0], 1, :, where[1]], before[:, 2 * H:])
    assert torch.equal(qkv[:, H:], before[:, H:])


def test_pages_outside_the_pool():
    """Rows of a page number outside the pool: appended ones are dropped, cached
    ones read as zeros.  (Both kernels compare the number with the pool's page
    count before they form an address.)"""
    rng = np.random.default_rng(9)
    for kind in ("bf16", "f32"):
        pages = Pages(rng, kind, [40, 40], 2, 64, 16)
        for bad in (-1, pages.data.shape[0], 0x7fffffff):
            pages.tables[0, 1] = bad
            pages.tables_d.copy_(torch.from_numpy(pages.tables))
            k, _ = normal(rng, kind, 80, 2, 64)
            held = pages.data.clone()
            off = offsets([40, 40])
            upr.paged_append(pages.cache(), off, pages.rows, k, k)
            torch.cuda.synchronize()
            for u in range(2):
                for p in range(40):
                    if (u, p // 16) != (0, 1):
                        held[pages.tables[u, p // 16], :, :, p % 16] = k[40 * u + p]
            assert torch.equal(held.view(torch.uint8), pages.data.view(torch.uint8))
            kv = k.double().cpu().numpy().reshape(2, 40, 2, 64).transpose(0, 2, 1, 3).copy()
            kv[0, :, 16:32] = 0.0
            q, qv = normal(rng, kind, 6, 2, 64)
            got = upr.paged_attention(pages.cache(), offsets([3, 3]), pages.rows, q)
            for u in range(2):
                want, bound = attend(qv[3 * u:3 * u + 3], kv[u], kv[u], np.arange(37, 40), kind)
                assert_close(got[3 * u:3 * u + 3], want, bound, f"{kind} page {bad} user {u}")


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

def run_attend(rng, kind, counts, rows, H, kv, D, page, own=False, fill=None, first=0, label="", q_scale=1.0, **opt):
    pages = Pages(rng, kind, rows, kv, D, page, fill=fill)
    off = offsets(counts, first=first)
    q, qv = normal(rng, kind, int(off[-1]), H, D, scale=q_scale)
    slopes = None
    if opt.pop("bias", False):
        slopes = torch.tensor([2.0 ** -(h + 1) for h in range(H)], dtype=torch.float32, device="cuda")
    ks = vs = ksv = vsv = None
    if own:
        (ks, ksv), (vs, vsv) = normal(rng, kind, int(off[-1]), kv, D), normal(rng, kind, int(off[-1]), kv, D)
    out = torch.full_like(q, 5.0)
    call = dict(slopes=slopes, k_self=ks, v_self=vs, **opt)
    upr.paged_attention(pages.cache(), off, pages.rows, q, out=out, **call)
    torch.cuda.synchronize()
    for u, (c, n) in enumerate(zip(counts, rows)):
        if c == 0:
            continue
        a, b = int(off[u]), int(off[u + 1])
        pos = np.full(c, n) if own else np.arange(n - c, n)
        want, bound = attend(qv[a:b], *pages.hist[u], pos, kind, own=(ksv[a:b], vsv[a:b]) if own else None,
                             slopes=None if slopes is None else slopes.double().cpu().numpy(), **opt)
        assert_close(out[a:b], want, bound, f"{label} user {u}: {c} rows over {n}")
    assert bool((out[:first] == 5.0).all())
    return pages, off, q, out, call


SHAPES = [  # heads, kv heads, head_dim, page
    (8, 8, 64, 64), (4, 4, 32, 16), (8, 2, 128, 32), (7, 1, 64, 128), (3, 3, 128, 16), (32, 4, 32, 256)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("H,kv,D,page", SHAPES)
def test_single_rows(kind, H, kv, D, page):
    """One new row per user over histories from one row (itself) up, unused
    places holding NaN."""
    rng = np.random.default_rng([H, kv, D, 1])
    say(f"[gpu] attend {kind} {H}/{kv}x{D} single rows")
    run_attend(rng, kind, [1, 1, 0, 1, 1, 1, 1, 1], [1, 2, 9, 16, 31, 64, 65, 1000], H, kv, D, page)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("H,kv,D,page", SHAPES)
def test_chunks(kind, H, kv, D, page):
    rng = np.random.default_rng([H, kv, D, 2])
    say(f"[gpu] attend {kind} {H}/{kv}x{D} chunks")
    run_attend(rng, kind, [2, 33, 130, 5, 64, 17], [2, 33, 400, 300, 129, 18], H, kv, D, page, first=3)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("opt", [
    dict(softcap=3.0), dict(bias=True), dict(window=1), dict(window=20), dict(window=150),
    dict(softcap=5.0, bias=True, window=70, scale=0.3)], ids=str)
@pytest.mark.parametrize("own", [False, True], ids=["causal", "self"])
def test_options(kind, opt, own):
    rng = np.random.default_rng(3)
    say(f"[gpu] attend {kind} {opt} own {own}")
    run_attend(rng, kind, [1, 40, 200, 3], [300, 90, 333, 3], 4, 2, 64, 32, own=own, q_scale=3.0, **opt)
    run_attend(rng, kind, [1, 1], [700, 30], 8, 2, 128, 16, own=own, q_scale=3.0, **opt)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("H,kv,D,page", SHAPES)
def test_candidates(kind, H, kv, D, page):
    """Own keys: histories from none up; every row sees all of it and itself."""
    rng = np.random.default_rng([H, kv, D, 4])
    say(f"[gpu] attend {kind} {H}/{kv}x{D} candidates")
    run_attend(rng, kind, [3, 1, 150, 64, 0, 20], [0, 1, 77, 256, 9, 500], H, kv, D, page, own=True, first=2)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_long_histories_and_many_users(kind):
    """A few rows over a history long enough to be split, and more users than
    one launch takes."""
    rng = np.random.default_rng(6)
    say(f"[gpu] attend {kind} long, many users")
    run_attend(rng, kind, [1, 5, 18], [9001, 4100, 6000], 4, 2, 64, 64, q_scale=2.0)
    run_attend(rng, kind, [2, 1], [9001, 4100], 8, 8, 32, 64, own=True)
    counts = rng.integers(0, 3, 290)
    run_attend(rng, kind, counts, counts + rng.integers(0, 40, 290), 2, 1, 32, 16)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_large_scores(kind):
    """Scores of hundreds, rising and falling along the history: the running
    maximum moves."""
    rng = np.random.default_rng(12)
    run_attend(rng, kind, [1, 40, 64], [600, 500, 64], 2, 2, 64, 16, q_scale=60.0)
    run_attend(rng, kind, [40], [500], 2, 2, 64, 16, q_scale=60.0, own=True)


# Enough rows for the widest tiles (192 of 128 rows, counted with the heads).
WIDE = ([100, 97, 128, 111, 100, 100], [100, 300, 128, 333, 1000, 160])


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("opt", [
    dict(), dict(q_scale=60.0), dict(q_scale=600.0), dict(window=70), dict(window=1), dict(bias=True),
    dict(softcap=5.0, q_scale=4.0), dict(softcap=5.0, bias=True, window=90, scale=0.3)], ids=str)
@pytest.mark.parametrize("own", [False, True], ids=["causal", "self"])
def test_wide_tiles(D, opt, own):
    rng = np.random.default_rng([D, 19])
    say(f"[gpu] attend wide tiles, head_dim {D}, {opt}, own {own}")
    run_attend(rng, "bf16", *WIDE, 32, 8, D, 32, own=own, **opt)


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("step", [0.05, 0.9, 30.0, -30.0])
def test_scores_that_rise_along_the_history(D, step):
    """A row's reference is passed again and again: scores rise (or fall) by
    `step` bits a key on average."""
    rng = np.random.default_rng([D, 20])
    counts, rows = WIDE
    say(f"[gpu] attend head_dim {D}, scores rising by {step} bits a key")
    pages = Pages(rng, "bf16", rows, 8, D, 32)
    q, _ = normal(rng, "bf16", sum(counts), 32, D)
    q[..., 0] = float(D) ** 0.5
    for u, n in enumerate(rows):
        ramp = (torch.arange(n) * step * 0.6931).to(pages.dt)
        pages.hist[u][0, :, :, 0] = ramp.double().numpy()
        for p in range(n):
            pages.data[pages.tables[u, p // 32], 0, :, p % 32, 0] = ramp[p].item()
    off = offsets(counts)
    out = upr.paged_attention(pages.cache(), off, pages.rows, q)
    qv = q.double().cpu().numpy()
    for u, (c, n) in enumerate(zip(counts, rows)):
        a, b = int(off[u]), int(off[u + 1])
        want, bound = attend(qv[a:b], *pages.hist[u], np.arange(n - c, n), "bf16")
        assert_close(out[a:b], want, bound, f"user {u}")


def test_wide_tiles_unseen_rows_and_neighbours():
    """As the two tests below, in the widest tiles."""
    rng = np.random.default_rng(21)
    counts, rows = WIDE
    for D in (64, 128):
        pages, off, q, out, _ = run_attend(rng, "bf16", counts, rows, 32, 8, D, 32)
        u, n, c, a = 4, 1000, 100, int(off[4])
        want, bound = attend(q[a:a + c].double().cpu().numpy(), *pages.hist[u], np.arange(n - c, n), "bf16")
        for value in (float("nan"), float("inf"), torch.finfo(torch.bfloat16).max):
            for j in (n - 1, n - 30, 930):
                where = pages.tables[u, j // 32]
                held = pages.data[where, :, :, j % 32].clone()
                pages.data[where, :, :, j % 32] = value
                got = upr.paged_attention(pages.cache(), off, pages.rows, q)[a:a + c]
                pages.data[where, :, :, j % 32] = held
                blind = np.arange(n - c, n) < j
                assert_close(got[torch.from_numpy(blind).cuda()], want[blind], bound[blind], f"row {j} {value}")
                if value != value:
                    assert bool(torch.isnan(got[torch.from_numpy(~blind).cuda()]).all())
        pages, off, q, out, call = run_attend(rng, "bf16", counts, rows, 32, 8, D, 32, own=True, q_scale=20.0)
        order = np.concatenate([int(off[u]) + rng.permutation(c) for u, c in enumerate(counts)])
        perm = torch.from_numpy(order).cuda()
        call = dict(call, k_self=call["k_self"][perm], v_self=call["v_self"][perm])
        got = upr.paged_attention(pages.cache(), off, pages.rows, q[perm].contiguous(), **call)
        assert torch.equal(got, out[perm])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf"), None])
def test_unseen_rows_have_no_influence(kind, value):
    """Keys and values that a row does not see (later positions, behind the
    window) may be anything, the type's largest value (None) included."""
    rng = np.random.default_rng(13)
    H, D, n, c = 2, 64, 300, 140
    for window in (0, 50):
        pages, off, q, out, _ = run_attend(rng, kind, [c], [n], H, H, D, 16, window=window)
        # Not bit for bit: a row may be summed in another order.  Two orders of
        # n = 300 fp32 terms differ by up to 2 n roundings, 2 * 300 * 2^-24 of the
        # terms' size, so each result is held to the bound of the formula that
        # counts them (attend), which the unseen row is no part of.
        want, bound = attend(q.double().cpu().numpy(), *pages.hist[0], np.arange(n - c, n), kind, window=window)
        value = torch.finfo(pages.dt).max if value is None else value
        for j in (n - 1, n - 30, n - 77, 190, 130, 3):
            where = pages.tables[0, j // 16]
            held = pages.data[where, :, :, j % 16].clone()
            pages.data[where, :, :, j % 16] = value
            got = upr.paged_attention(pages.cache(), off, pages.rows, q, window=window)
            pages.data[where, :, :, j % 16] = held
            pos = np.arange(n - c, n)
            blind = torch.from_numpy((pos < j) | ((pos >= j + window) if window else np.zeros(c, bool))).cuda()
            mask = blind.cpu().numpy()
            assert_close(got[blind], want[mask], bound[mask], f"window {window}, row {j}")
            if value != value:
                assert bool(torch.isnan(got[~blind]).all()), (window, j)


def test_rows_do_not_depend_on_their_neighbours():
    """Permuted candidates give permuted outputs, bit for bit."""
    rng = np.random.default_rng(14)
    for kind in ("bf16", "f32"):
        pages, off, q, out, call = run_attend(rng, kind, [200], [700], 4, 4, 64, 64, own=True, q_scale=8.0)
        perm = torch.from_numpy(rng.permutation(200)).cuda()
        call = dict(call, k_self=call["k_self"][perm], v_self=call["v_self"][perm])
        got = upr.paged_attention(pages.cache(), off, pages.rows, q[perm].contiguous(), **call)
        assert torch.equal(got, out[perm])
        again = upr.paged_attention(pages.cache(), off, pages.rows, q[perm].contiguous(), **call)
        assert torch.equal(got, again)


def test_graphs_and_streams():
    """A captured append and attention replay to the eager result, two graphs
    with workspaces of their own; a call on another stream."""
    rng = np.random.default_rng(15)
    H, D = 4, 64
    rows = np.asarray([5000, 37, 800], np.int32)
    pages = Pages(rng, "bf16", rows, H, D, 64, fill=0.0)
    off = offsets([1, 1, 1])
    k, _ = normal(rng, "bf16", 3, H, D)
    r = upr.rope(64)
    cache = pages.cache()

    def make():
        q, _ = normal(rng, "bf16", 3, H, D)
        return dict(q=q, turned=torch.empty_like(q), out=torch.empty_like(q),
                    ws=upr.paged_attention_workspace(cache, off, rows, H))

    def step(s):
        upr.paged_append(cache, off, rows, k, k, rope=r, q=s["q"], q_out=s["turned"])
        upr.paged_attention(cache, off, rows, s["turned"], out=s["out"], ws=s["ws"])

    states = [make(), make()]
    want, graphs = [], []
    for s in states:
        step(s)
        torch.cuda.synchronize()
        want.append(s["out"].clone())
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(s)
        graphs.append(g)
    for _ in range(3):
        for s, g, w in zip(states, graphs, want):
            s["out"].fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(s["out"], w)
            step(states[0])
            torch.cuda.synchronize()
            assert torch.equal(states[0]["out"], want[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = torch.empty_like(states[1]["out"])
    upr.paged_attention(cache, off, rows, states[1]["turned"], out=got, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got, want[1])


def test_new_tensors_come_from_the_calls_stream():
    """What the current stream has freed may still be in use there: a call on
    another stream does not write to it."""
    rng = np.random.default_rng(18)
    rows = np.asarray([3000], np.int32)
    pages = Pages(rng, "bf16", rows, 4, 64, 64)
    q, _ = normal(rng, "bf16", 1, 4, 64)
    x = torch.zeros((8192, 4, 64), dtype=torch.bfloat16, device="cuda")
    at = torch.zeros(8192, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    size = upr.paged_attention_workspace(pages.cache(), offsets([1]), rows, 4).numel()
    assert size > 256
    torch.cuda.synchronize()
    freed = [torch.empty_like(x).data_ptr()]
    out = upr.rope_apply(x, at, upr.rope(64), stream=side.cuda_stream)
    assert out.data_ptr() not in freed
    freed = [torch.empty(size, dtype=torch.uint8, device="cuda").data_ptr()]
    ws = upr.paged_attention_workspace(pages.cache(), offsets([1]), rows, 4, stream=side.cuda_stream)
    assert ws.data_ptr() not in freed
    freed = [torch.empty_like(q).data_ptr()]
    got = upr.paged_attention(pages.cache(), offsets([1]), rows, q, ws=ws, stream=side.cuda_stream)
    assert got.data_ptr() not in freed
    torch.cuda.synchronize()
    assert torch.equal(got, upr.paged_attention(pages.cache(), offsets([1]), rows, q))


def test_wrappers_refuse():
    rng = np.random.default_rng(16)
    pages = Pages(rng, "bf16", [20], 2, 64, 16)
    cache, off = pages.cache(), offsets([4])
    q, _ = normal(rng, "bf16", 4, 4, 64)
    with pytest.raises(TypeError):
        upr.paged_attention(cache, off, pages.rows, q.float())
    with pytest.raises(TypeError):
        upr.paged_attention(cache, off, pages.rows, q.cpu())
    with pytest.raises(ValueError):
        upr.paged_attention(cache, off, pages.rows, q[:3])
    with pytest.raises(ValueError):
        upr.paged_attention(cache, off, pages.rows, q.transpose(0, 1).contiguous().transpose(0, 1))
    with pytest.raises(TypeError):
        upr.paged_attention(cache, off, pages.rows.astype(np.int64), q)
    with pytest.raises(ValueError):
        upr.paged_attention(cache, offsets([4, 0]), np.asarray([20, 3], np.int32), q)     # one table
    with pytest.raises(ValueError):
        upr.paged_attention(cache, off, pages.rows, q, slopes=torch.zeros(2, dtype=torch.float32, device="cuda"))
    with pytest.raises(ValueError):
        upr.PagedCache(pages.data.transpose(2, 3), pages.tables_d)
    with pytest.raises(upr.UprError):
        upr.paged_append(cache, off, pages.rows, q[:, :2], q[:, :2], q=q)
    with pytest.raises(ValueError):
        upr.rope_apply(q, torch.zeros(3, dtype=torch.int32, device="cuda"), upr.rope(64))


# ---------------------------------------------------------------------------
# Sizes past 32 bits
# ---------------------------------------------------------------------------

def test_offsets_past_32_bits():
    """Pages, queries and outputs beyond 2^32 bytes from their base."""
    D, H, page = 128, 1, 1024
    n_pages = 17000                                     # 17000 * 2 * 1024 * 128 * 2 B = 8.9 GB
    data = torch.zeros((n_pages, 2, H, page, D), dtype=torch.bfloat16, device="cuda")
    tables = torch.tensor([[n_pages - 1, 3], [n_pages - 2, n_pages - 3]], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(17)
    wide = torch.zeros((3, 1 << 30), dtype=torch.bfloat16, device="cuda")       # rows 2 GiB apart
    x = wide[:, :D].unflatten(1, (H, D))
    val, vv = normal(rng, "bf16", 3, H, D)
    x.copy_(val)
    off, rows = offsets([1, 2]), np.asarray([1500, 1026], np.int32)
    cache = upr.PagedCache(data, tables)
    upr.paged_append(cache, off, rows, x, x)
    assert torch.equal(data[3, 0, :, 475], val[0]) and torch.equal(data[n_pages - 3, 1, :, 0:2].transpose(0, 1), val[1:])
    got = upr.paged_attention(cache, off, rows, x)
    for u, (a, b) in enumerate([(0, 1), (1, 3)]):
        n = int(rows[u])
        K = np.zeros((H, n, D))
        K[:, n - (b - a):] = vv[a:b].transpose(1, 0, 2)
        want, bound = attend(vv[a:b], K, K, np.arange(n - (b - a), n), "bf16")
        assert_close(got[a:b], want, bound, f"user {u}")
    del wide, data


def test_rows_of_the_largest_call():
    """The most rows that a call takes of one user, 2^27 with their heads, where
    each head's last tile is part empty: without history a row gives its value."""
    H, D = 33, 32
    rows = (1 << 27) // H
    x = torch.empty((rows, H, D), dtype=torch.float32, device="cuda")
    x.view(-1).copy_(torch.arange(D * 1009, dtype=torch.float32, device="cuda").repeat(x.numel() // (D * 1009) + 1)[:x.numel()])
    x.mul_(2.0 ** -15)
    cache = upr.PagedCache(torch.zeros((1, 2, H, 16, D), dtype=torch.float32, device="cuda"),
                           torch.zeros((1, 1), dtype=torch.int32, device="cuda"))
    out = torch.full_like(x, float("nan"))
    upr.paged_attention(cache, offsets([rows]), np.zeros(1, np.int32), x, out=out, k_self=x, v_self=x)
    for i in range(0, rows, 1 << 18):
        assert torch.equal(out[i:i + (1 << 18)], x[i:i + (1 << 18)]), i
    del x, out
