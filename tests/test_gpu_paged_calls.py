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
    H = 5                                                # (more heads than a workgroup sums, and not a multiple)
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
    """O and lse of the given rows of sequence 0 where the pages `bad` are not in the cache: their keys are left out, and
    c_i is 0 for a row on one.  Tolerances as in World.reference."""
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
            delta = -(2 * float(w.gq[h].double() * w.gk[hk].double()) * math.sqrt(w.d) + math.log(L_max) - math.log(eps))
            last = (j // 64 * 64 + 63).clamp(max=L - 1)
            seen &= (j // 64)[None] == i // 64
            seen |= (j[None] // 64 < i // 64) & here[None] & (decay.gather(1, last[None].expand_as(decay)) >= delta)
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
        assert ((go - ro).abs() / to)[~reached].max() <= 1, (h, "O", float(((go - ro).abs() / to)[~reached].max()))
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
    for rows in ([r for r in range(new) if (past + r) // 64 not in bad], [r for r in range(new) if (past + r) // 64 in bad]):
        check_with_bad_pages(w, o, lse, bad + gone, EPS, torch.tensor(rows, device="cuda"))


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
            if m <= 16 // 2 or max_new > 16 // 2:         # (few rows: 16 with those of two heads per key head)
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
    w.check(*w.cache.attend(w.packed("q"), w.cu, w.past_t, wide, 20, gamma_q=w.gq, gamma_k=w.gk, eps=EPS, L_max=4096))


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
