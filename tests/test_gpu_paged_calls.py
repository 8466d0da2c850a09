"""Calls of the paged cache that its documentation allows, away from the ordinary ones: gates
that are not finite in an earlier call, rows whose own page is not in the cache, rows that no
sequence brings, scales that do not bound the logits, call arrays of any content."""
import math

import pytest
import torch

from paper_2504_06949_amd import acp, ops
from tests._helpers import ensure_built
from tests.test_gpu_paged import BF, E, EPS, F32, World

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---- gates ---------------------------------------------------------------------------------

@pytest.mark.parametrize("n", [1, 16, 17, 64, 65, 3000])
@pytest.mark.parametrize("gate", [-math.inf, math.nan, math.inf])
def test_a_sum_of_gates_that_is_not_finite_stays_reported(n, gate):
    """Every later sum of the head inherits it, whatever its own gates."""
    H = 5                                       # (more heads than a workgroup sums, and not a multiple)
    cache = ops.PagedCache(60, H, 64, 1)
    table = torch.arange(60, dtype=torch.int32, device="cuda")[None]
    flags = torch.full((1, H), -1, dtype=torch.int32, device="cuda")
    at = 0
    for call, rows in enumerate((n, min(n, 400), min(n, 400))):
        kv = torch.zeros((rows, 1, 64), dtype=BF, device="cuda")
        f = torch.full((rows, H), -0.25, device="cuda")
        if call == 0:
            f[n // 2, 1] = f[n - 1, 4] = gate
        cache.append(kv, kv, f, ints(0, rows), ints(at), table, flags=flags)
        assert flags.tolist() == [[0, 2, 0, 0, 2]], call
        at += rows


# ---- rows whose own page is bad -----------------------------------------------------------

def check_with_bad_pages(w, o, lse, bad, eps, rows, L_max=4096):
    """O and lse of the given rows of sequence 0 where the pages `bad` are not in the cache: their keys
    are left out, and c_i is 0 for a row on one.  Tolerances as in World.reference."""
    p0, L = w.past[0], w.past[0] + w.new[0]
    j = torch.arange(L, device="cuda")
    i = j[p0:, None]
    here = torch.ones(L // 64 + 1, dtype=torch.bool, device="cuda")
    here[list(bad)] = False
    here = here[j // 64]
    wt = 2.0 ** -8 if w.dtype == BF else 0.0
    half = torch.finfo(w.dtype).eps / 2
    for h in range(w.H):
        hk = h // (w.H // w.Hk)
        q, k, v = w.q[0][p0:, h].double(), w.k[0][:, hk].double(), w.v[0][:, hk].double()
        c = w.c[0][:, h]
        decay = torch.where(here[p0:], c[p0:], 0.0)[:, None] - c[None]
        seen = (j[None] <= i) & here[None]
        if eps > 0:
            u = float(w.gq[h].double() * w.gk[hk].double()) * math.sqrt(w.d)
            delta = -(2 * u + math.log(L_max) - math.log(eps))
            last = (j // 64 * 64 + 63).clamp(max=L - 1)
            seen &= (j // 64)[None] == i // 64
            kept = decay.gather(1, last[None].expand_as(decay)) >= delta
            seen |= (j[None] // 64 < i // 64) & here[None] & kept
        x = torch.where(seen, q @ k.t() / math.sqrt(w.d) + decay, -math.inf)
        top = x.amax(1, keepdim=True)
        p = torch.exp(x - top)
        tot = p.sum(1, keepdim=True)
        p = p / tot
        t = E * ((w.d / 4 + 8) * (q.abs() @ k.abs().t() / math.sqrt(w.d) + decay.abs()) + 8 + 2 * (top - x))
        pt = torch.where(seen, p * (t + wt + 200 * E), 0.0)
        fin = torch.isfinite(v)
        v0 = torch.where(fin, v, 0.0)
        ro = p @ v0
        to = pt @ v0.abs() + pt.sum(1)[:, None] * ro.abs() + 4 * E * ro.abs() + half * ro.abs()
        reached = (seen.double() @ (~fin).double()) > 0          # a value that is not finite is seen
        rl = (top + tot.log())[:, 0]
        tl = torch.where(seen, p * (t + 200 * E), 0.0).sum(1) + 8 * E * (rl.abs() + 1)
        go, gl = o[rows, h].double(), lse[rows, h].double()
        ro, to, reached, rl, tl = (x[rows] for x in (ro, to, reached, rl, tl))
        assert torch.equal(torch.isfinite(go), ~reached), (h, "which are finite")
        off = ((go - ro).abs() / to)[~reached].max()
        assert off <= 1, (h, "O", float(off))
        assert ((gl - rl).abs() / tl).max() <= 1, (h, "lse", float(((gl - rl).abs() / tl).max()))


def bad_page_world(new, past, bad, G, d, dtype, strong):
    """Gates behind one that makes |c| 1e5.  Strong: they leave out all but a page or two, and there is a NaN
    and an infinity in pages that rows with their own gate leave out, and c_i = 0 does not.  Weak: every
    page counts for every row."""
    w = World([new], [past], 2 * G, 2, d, dtype, seed=30, mu=(0.3, 0.6) if strong else (6.0, 9.0))
    w.f[0][5] = -1e5
    w.c = [torch.cumsum(f.double(), 0) for f in w.f]
    if strong:
        w.v[0][20, :, 7] = float("nan")
        w.v[0][70, :, 9] = float("inf")
    w.fill_past()
    w.append()
    for n in bad:
        w.table[0, n] = (-1, w.P)[n % 2]
    return w


BAD_TILES = [(128, 300, [4]), (128, 300, [5]), (128, 300, [6]), (128, 300, [4, 6]),     # tiles of 128 rows
             (60, 300, [4]), (60, 300, [5]), (200, 290, [6]),                           # of 64, two tiles
             (16, 310, [4]), (16, 310, [5]), (3, 318, [5])]                             # few rows


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new,past,bad", BAD_TILES)
def test_good_rows_beside_rows_whose_own_page_is_bad(new, past, bad, dtype):
    for G, d, strong in ((1, 64, True), (2, 128, True), (1, 64, False), (2, 128, False)):
        print(f"case: own page bad new={new} past={past} bad={bad} G={G} d={d} strong={strong} {dtype}", flush=True)
        w = bad_page_world(new, past, bad, G, d, dtype, strong)
        good = torch.tensor([(past + r) // 64 not in bad for r in range(new)], device="cuda")
        flags = torch.zeros((1, w.H), dtype=torch.int32, device="cuda")
        for eps in (EPS, 0.0):
            o, lse = w.attend(eps, flags=flags)
            assert (flags == ops.FLAG_BAD_PAGE).all()
            if good.any():
                assert torch.isfinite(o[good]).all() or (eps == 0.0 and strong)
                check_with_bad_pages(w, o, lse, bad, eps, good)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new,past,bad", BAD_TILES)
def test_rows_whose_own_page_is_bad_whatever_their_neighbours_keep(new, past, bad, dtype):
    """With c_i = 0 they leave out no page, also where the rows before them in the tile do: a value that is
    not finite reaches them from any page."""
    for G, d in ((1, 64), (2, 128)):
        print(f"case: own page bad, rows new={new} past={past} bad={bad} G={G} d={d} {dtype}", flush=True)
        w = bad_page_world(new, past, bad, G, d, dtype, True)
        rows = torch.tensor([(past + r) // 64 in bad for r in range(new)], device="cuda")
        for eps in (EPS, 0.0):
            o, lse = w.attend(eps)
            assert not torch.isfinite(o[rows][:, :, [7, 9]]).any()
            check_with_bad_pages(w, o, lse, bad, eps, rows)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new,past", [(128, 12300), (9, 12345)])
def test_dropped_pages_in_front_of_rows_whose_own_page_is_bad(new, past, dtype):
    """Pages that nobody keeps may be gone, hundreds of them: a row on a bad page starts behind them."""
    w = World([new], [past], 2, 2, 64, dtype, seed=38, mu=(0.0, 1.0))
    w.fill_past()
    w.append()
    bad = [past // 64 + 1]
    gone = list(range(130))
    w.table[0, gone + bad] = -1
    o, lse = w.attend()
    on_bad = torch.tensor([(past + r) // 64 in bad for r in range(new)], device="cuda")
    for rows in (on_bad, ~on_bad):
        check_with_bad_pages(w, o, lse, bad + gone, EPS, rows)


# ---- rows that nothing writes --------------------------------------------------------------

def poisoned(*shapes):
    """Memory of these shapes given back to the allocator full of 7."""
    for shape, t in shapes:
        torch.full(shape, 7.0, dtype=t, device="cuda")
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new,past,extra,max_new", [
    ([40, 1, 7], [100, 64, 3], 9, 40), ([1, 1], [100, 64], 5, 1), ([3, 80, 1, 17], [100, 10, 200, 0], 0, 3),
    ([3, 80, 1, 17], [100, 10, 200, 0], 300, 3), ([0, 5], [64, 1], 2, 5), ([0, 0], [64, 0], 70, 1)])
def test_rows_that_nothing_attends_for_are_empty(new, past, extra, max_new, dtype):
    """Rows behind the last sequence, and those of a sequence with more than max_new of them where only
    single tokens are expected: O = 0 and lse = -inf in outputs that the call makes itself."""
    w = World(new, past, 4, 2, 64, dtype, seed=31, extra_rows=extra)
    w.fill_past()
    w.append()
    T, n = w.T, sum(new)
    assert T == n + extra
    flags = torch.zeros((len(new), 4), dtype=torch.int32, device="cuda")
    for kw in ({}, {"flags": flags}):
        poisoned(((T, 4, 64), dtype), ((T, 4), torch.float32))
        o, lse = w.attend(max_new=max_new, **kw)
        on = torch.zeros(T, dtype=torch.bool, device="cuda")
        at = 0
        for s, m in enumerate(new):
            if m <= 8 or max_new > 8:            # (few rows: 16 with those of two heads per key head)
                on[at:at + m] = True
                w.check(o, lse, seqs=[s])
            at += m
        assert not o[~on].any() and (lse[~on] == -math.inf).all()
    assert [bool(f & ops.FLAG_MAX_NEW) for f in flags[:, 0].tolist()] == [m > 8 and max_new <= 8 for m in new]


def test_no_sequence_at_all():
    w = World([4], [10], 2, 2, 64, BF, seed=32)
    q = w.packed("q")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    poisoned(((4, 2, 64), BF), ((4, 2), torch.float32))
    o, lse = w.cache.attend(q, ints(0), none, w.table[:0], 1)
    assert not o.any() and (lse == -math.inf).all()


def test_a_table_as_wide_as_positions_go():
    """The default max_len of a table of more than 2^31 positions is within its range."""
    w = World([2, 20], [70, 3], 2, 2, 64, BF, seed=34)
    w.fill_past()
    w.append()
    wide = torch.full((2, (1 << 25) + 3), -1, dtype=torch.int32, device="cuda")
    wide[:, :w.table.shape[1]] = w.table
    w.table = wide
    w.check(*w.attend(max_new=20))


# ---- scales --------------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [100, 40, 8])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_logits_outside_what_the_scales_allow_are_reported(new, sign, d):
    """Keys that are the queries or their negatives, and gates of e^-70: a row's logit is all but its own
    key's, +-U.  At both ends of the bound nothing is reported.  Where the scales allow 1 in place of 110,
    the weights of a chunk in bfloat16 leave float32's range, which is reported; few rows do without
    the bound."""
    U = [8.0, 31.0, 45.0, 51.0]                          # (the reference is U up to 32, 64 - U up to 52)
    for u in U + [110.0]:
        scale = math.sqrt(u / math.sqrt(d))
        w = World([new], [30], 4, 4, d, BF, seed=33, scale=scale, mu=(-70.0, -70.0))
        w.k = [(sign * t).contiguous() for t in w.q]
        w.fill_past()
        w.append()
        flags = torch.full((1, 4), -1, dtype=torch.int32, device="cuda")
        o, lse = w.attend(flags=flags)
        assert not flags.any(), u
        w.check(o, lse)
    w.gq[1] = w.gq[3] = 1.0 / (scale * math.sqrt(d))
    o, lse = w.attend(flags=flags)
    chunk = 0 if new <= 16 else ops.FLAG_SCALES
    assert flags.tolist() == [[0, chunk, 0, chunk]]
    if not chunk:
        w.check(o, lse)
    w.attend()                                           # (the same without flags)


# ---- call arrays and scratch -----------------------------------------------------------------

class Guarded:
    """Buffers with a pattern on both sides."""

    def __init__(self):
        self.all = []

    def __call__(self, nbytes, fill=0x5a):
        side = 1 << 16
        whole = torch.full((nbytes + 2 * side,), 0xa5, dtype=torch.uint8, device="cuda")
        inner = whole[side:side + nbytes]
        inner.fill_(fill)
        self.all.append((whole, side, nbytes))
        return inner

    def check(self):
        for whole, side, n in self.all:
            assert (whole[:side] == 0xa5).all() and (whole[side + n:] == 0xa5).all()


@pytest.mark.parametrize("max_new", [1, 75])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_call_arrays_of_any_content_touch_nothing_else(dtype, max_new):
    """cu, past and table of any content: what lies around the cache, the outputs, the flags and the
    workspace stays, and so do the pages that the table does not name."""
    H, Hk, d, T, N, W, P = 4, 2, 64, 75, 2, 3, 9
    dt = acp.ACP_F32 if dtype == F32 else acp.ACP_BF16
    L = ops.lib()
    n = ops._sz(0)
    guard = Guarded()
    acp._check(L.acp_paged_cache_size(P, H, Hk, d, dt, ops.ctypes.byref(n)))
    cache = guard(n.value, 0)
    y = ops.PagedLayout()
    acp._check(L.acp_paged_offsets(P, H, Hk, d, dt, ops.ctypes.byref(y)))
    pages = {k: cache[a:b].view(P, -1) for k, a, b in (("k", y.k, y.v), ("v", y.v, y.c), ("c", y.c, y.total))}
    acp._check(L.acp_paged_workspace_size(T, N, H, Hk, d, dt, max_new, 64 * W, ops.ctypes.byref(n)))
    ws = guard(n.value)
    o, lse, flags = guard(T * H * d * (4 if dtype == F32 else 2)), guard(T * H * 4), guard(N * H * 4)
    g = torch.Generator(device="cuda").manual_seed(35)
    q = torch.randn((T, H, d), generator=g, device="cuda").to(dtype)
    kv = torch.randn((T, Hk, d), generator=g, device="cuda").to(dtype)
    f = torch.full((T, H), -0.5, device="cuda")
    gq, gk = torch.ones(H, device="cuda"), torch.ones(Hk, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    tables = [[[0, 2, 4], [6, 7, 8]], [[-1, P, 4], [-(1 << 31), 7, (1 << 31) - 1]],
              [[P + 1, -5, 1 << 30], [3, -1, -1]], [[-2, -2, -2], [P, P, P]]]
    for cu in ([0, 5, 75], [0, 1000, 75], [5, 0, -3], [-7, 200, 100], [80, 90, 95], [0, 0, 0], [0, 1, 2]):
        for past in ([64, 10], [-5, 1 << 30], [0x7fffffff, 0x7fffffff], [-(1 << 31), 190]):
            for table in tables:
                print(f"case: call arrays cu={cu} past={past} table={table} {dtype} {max_new}", flush=True)
                cu_t, past_t, table_t = ints(*cu), ints(*past), torch.tensor(table, dtype=torch.int32, device="cuda")
                before = {m: t.clone() for m, t in pages.items()}
                acp._check(L.acp_paged_append(
                    kv.data_ptr(), None, kv.data_ptr(), None, f.data_ptr(), None, dt, T, N, W, P, H, Hk, d,
                    cu_t.data_ptr(), past_t.data_ptr(), table_t.data_ptr(), cache.data_ptr(), cache.numel(),
                    flags.data_ptr(), stream))
                named = {p for r in table for p in r}
                rest = [p for p in range(P) if p not in named]
                for m, t in pages.items():
                    assert torch.equal(t[rest], before[m][rest]), m
                kept = cache.clone()
                for eps, attend in ((EPS, L.fox_attn_paged), (0.0, L.fox_attn_paged), (EPS, L.fox_attn_paged_filled)):
                    acp._check(attend(
                        q.data_ptr(), None, dt, T, N, W, P, H, Hk, d, cu_t.data_ptr(), past_t.data_ptr(),
                        table_t.data_ptr(), cache.data_ptr(), cache.numel(), gq.data_ptr(), gk.data_ptr(), eps, 4096,
                        max_new, 64 * W, o.data_ptr(), lse.data_ptr(), flags.data_ptr(), ws.data_ptr(), ws.numel(),
                        stream))
                assert torch.equal(cache, kept)
        guard.check()


def test_pages_past_32_bit_offsets():
    """Every page of the call starts past 2^32 elements of its tensor, and past 2^32 bytes of the gates'."""
    P = (1 << 32) // (4 * 64 * 128) + 20
    w = World([1, 40], [200, 70], 4, 4, 128, BF, seed=36, spare=0)
    first = P - w.P
    w.table = torch.where(w.table >= 0, first + w.table, w.table)
    w.cache = ops.PagedCache(P, 4, 128, 4, BF)
    assert w.P <= 20 and int(w.table[w.table >= 0].min()) * 4 * 64 * 128 >= 1 << 32
    w.fill_past()
    w.append()
    w.check_pages()
    for eps in (EPS, 0.0):
        w.check(*w.attend(eps), eps)


def test_a_captured_step_stores_and_attends():
    """Replays with the new rows' slots and the outputs overwritten before each: what the graph leaves is
    what an eager step of the same contents leaves, pages and outputs."""
    w = World([1, 1, 30], [500, 63, 100], 4, 2, 64, BF, seed=37)
    w.fill_past()
    q, k, v, f = (w.packed(n) for n in "qkvf")
    pos = torch.cat([torch.arange(p, p + n, device="cuda") for p, n in zip(w.past, w.new)])
    seq = torch.cat([torch.full((n,), s, device="cuda") for s, n in enumerate(w.new)])
    page, slot = w.table[seq, pos // 64].long(), pos % 64
    views = w.cache.views()

    def step():
        w.cache.append(k, v, f, w.cu, w.past_t, w.table)
        return w.cache.attend(q, w.cu, w.past_t, w.table, 30, gamma_q=w.gq, gamma_k=w.gk, eps=EPS, L_max=4096)

    def wipe(*outs):
        for t in views.values():
            t[page, :, slot] = float("nan")
        for t in outs:
            t.fill_(float("nan"))

    wipe()
    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    for r in range(4):
        for x in (q, k, v, f):
            x.copy_(x.roll(1, 0))
        wipe()
        want = [t.clone() for t in step()]
        held = {n: t[page, :, slot].clone() for n, t in views.items()}
        assert all(torch.isfinite(t).all() for t in held.values()) and torch.isfinite(want[0]).all()
        for g, out in graphs if r % 2 else graphs[::-1]:
            wipe(*out)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for n, t in views.items():
                assert torch.equal(t[page, :, slot], held[n]), (r, n)
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), r


@pytest.mark.parametrize("long", [False, True])
def test_the_most_sequences_of_a_call(long):
    """65535 sequences without a past, one token each (one has 40, some none), 16 query heads on one key head:
    the single tokens return their values, with their logit as log-sum-exp."""
    N, H, d = 65535, 16, 64
    n = torch.ones(N, dtype=torch.int32, device="cuda")
    n[5::1000] = 0
    if long:
        n[40000] = 40
    cu = torch.zeros(N + 1, dtype=torch.int32, device="cuda")
    cu[1:] = torch.cumsum(n, 0)
    T = int(cu[-1])
    g = torch.Generator(device="cuda").manual_seed(39)
    q, k, v = (torch.randn((T, heads, d), generator=g, device="cuda").to(BF) for heads in (H, 1, 1))
    f = -torch.rand((T, H), generator=g, device="cuda")
    cache = ops.PagedCache(N, H, d, 1)
    table = torch.randperm(N, generator=g, device="cuda").to(torch.int32)[:, None]
    flags = torch.full((N, H), -1, dtype=torch.int32, device="cuda")
    past = torch.zeros(N, dtype=torch.int32, device="cuda")
    cache.append(k, v, f, cu, past, table, flags=flags)
    assert not flags.any()
    o, lse = cache.attend(q, cu, past, table, 40 if long else 1, flags=flags)
    assert not flags.any()
    one = torch.ones(T, dtype=torch.bool, device="cuda")
    if long:
        at = int(cu[40000])
        one[at:at + 40] = False
        c = f[at:at + 40, 3].double().cumsum(0)
        x = q[at:at + 40, 3].double() @ k[at:at + 40, 0].double().t() / 8 + c[:, None] - c[None]
        x = torch.where(torch.ones_like(x).tril() > 0, x, -math.inf)
        # (a logit of at most 10: 24 e of it; 40 keys: 40 e more)
        assert (lse[at:at + 40, 3].double() - torch.logsumexp(x, 1)).abs().max() <= 300 * E
    assert torch.equal(o[one], v[one].expand(-1, H, -1))
    want = (q.float() * k.float()).sum(-1) / 8
    # (64 products of float32 size |q k|, in any order)
    assert ((lse - want)[one].abs() <= 64 * E * ((q.float() * k.float()).abs().sum(-1)[one] / 8 + 1)).all()
