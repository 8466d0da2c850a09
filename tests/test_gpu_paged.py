"""The paged cache and the attention of new tokens over it, against float64.

Tolerances.  With e = 2^-24, logit x_ij = s_ij + c_i - c_j is formed with an error of at most
    t_ij = e ((d / 4 + 8) (sum_k |q_ik k_jk| / sqrt(d) + |c_i - c_j|) + 8 + 2 (max_j x_ij - x_ij)),
a weight p_ij with t_ij relative, and sums over keys add 200 e; bfloat16 weights are off by
2^-8 more.  O moves by at most sum_j p_ij t_ij (|v_j| + |O_i|), plus the sums' and the output
type's rounding; lse by sum_j p_ij t_ij and its own rounding."""
import math

import numpy as np
import pytest
import torch

from paper_2504_06949_amd import acp, ops
from tests._helpers import ensure_built

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
EPS = math.exp(-10.0)
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_built()


class World:
    """Sequences with all their tokens, and a cache with pages in random order."""

    def __init__(self, new, past, H, Hk, d, dtype, seed=0, mu=(1.0, 8.0), spare=5, extra_rows=0, scale=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.new, self.past, self.H, self.Hk, self.d, self.dtype = new, past, H, Hk, d, dtype
        N = len(new)
        tot = [a + b for a, b in zip(new, past)]

        def rows(L, heads):
            x = torch.randn((L, heads, d), generator=g, device="cuda")
            return x * torch.rsqrt((x * x).mean(-1, keepdim=True)) * (1 - 2.0 ** -7) * scale

        self.q = [rows(L, H).to(dtype) for L in tot]
        self.k = [rows(L, Hk).to(dtype) for L in tot]
        self.v = [torch.randn((L, Hk, d), generator=g, device="cuda").to(dtype) for L in tot]
        m = torch.linspace(mu[0], mu[1], H, device="cuda", dtype=torch.float64)
        self.f = [(-torch.nn.functional.softplus(
            -(torch.randn((L, H), generator=g, device="cuda", dtype=torch.float64) * 0.5 + m))).float() for L in tot]
        self.c = [torch.cumsum(f.double(), 0) for f in self.f]
        self.gq = torch.full((H,), scale, device="cuda")
        self.gk = torch.full((Hk,), scale, device="cuda")
        need = [(L + 63) // 64 for L in tot]
        self.P, W = sum(need) + spare, max(need + [1]) + 1
        order = torch.randperm(self.P, generator=g, device="cuda")
        self.table = torch.full((N, W), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n].int()
            at += n
        self.T = sum(new) + extra_rows
        self.past_t = torch.tensor(past, dtype=torch.int32, device="cuda").reshape(N)
        self.cu = torch.tensor([0] + np.cumsum(new).tolist(), dtype=torch.int32, device="cuda")
        self.cache = ops.PagedCache(self.P, H, d, Hk, dtype)
        self.cache.buffer.fill_(0xff)                   # every slot a NaN until it is written

    def packed(self, name, part="new"):
        """Rows of one part of every sequence, packed."""
        t = [x[p:] if part == "new" else x[:p] for x, p in zip(getattr(self, name), self.past)]
        t = torch.cat(t)
        more = self.T - sum(self.new) if part == "new" else 0
        return torch.cat([t, t.new_zeros((more,) + t.shape[1:])]) if more else t

    def fill_past(self):
        zero = torch.zeros_like(self.past_t)
        cu = torch.tensor([0] + np.cumsum(self.past).tolist(), dtype=torch.int32, device="cuda")
        self.cache.append(self.packed("k", "past"), self.packed("v", "past"), self.packed("f", "past"), cu, zero,
                          self.table)

    def append(self, **kw):
        self.cache.append(self.packed("k"), self.packed("v"), self.packed("f"), self.cu, self.past_t, self.table, **kw)

    def attend(self, eps=EPS, L_max=4096, **kw):
        kw.setdefault("max_new", max(self.new + [0]))
        return self.cache.attend(self.packed("q"), self.cu, self.past_t, self.table, gamma_q=self.gq, gamma_k=self.gk,
                                 eps=eps, L_max=L_max, **kw)

    def reference(self, s, h, eps, L_max):
        """(O, tolerance, lse, tolerance) of sequence s, head h in float64."""
        p0, L, hk = self.past[s], self.past[s] + self.new[s], h // (self.H // self.Hk)
        q, k, v = self.q[s][p0:, h].double(), self.k[s][:, hk].double(), self.v[s][:, hk].double()
        c = self.c[s][:, h]
        i, j = torch.arange(p0, L, device="cuda")[:, None], torch.arange(L, device="cuda")[None]
        decay = c[p0:, None] - c[None]
        x = q @ k.t() / math.sqrt(self.d) + decay
        seen = j <= i
        if eps > 0:
            u = float(self.gq[h].double() * self.gk[hk].double()) * math.sqrt(self.d)
            delta = -(2 * u + math.log(L_max) - math.log(eps))
            last = torch.minimum(j // 64 * 64 + 63, i)
            seen &= (j // 64 == i // 64) | (c[p0:, None] - c[last] >= delta)
        x = torch.where(seen, x, -math.inf)
        top = x.amax(1, keepdim=True)
        w = torch.exp(x - top)
        tot = w.sum(1, keepdim=True)
        p = w / tot
        v0 = torch.where(torch.isfinite(v), v, 0.0)
        o = p @ v0
        t = E * ((self.d / 4 + 8) * (q.abs() @ k.abs().t() / math.sqrt(self.d) + decay.abs()) + 8
                 + 2 * (top - x)) + (2.0 ** -8 if self.dtype == BF else 0.0)
        pt = torch.where(seen, p * (t + 200 * E), 0.0)
        err = pt.sum(1)
        return (o, pt @ v0.abs() + err[:, None] * o.abs() + 4 * E * o.abs(), (top + tot.log())[:, 0],
                torch.where(seen, p * (t - (2.0 ** -8 if self.dtype == BF else 0.0) + 200 * E), 0.0).sum(1)
                + 8 * E * ((top + tot.log()).abs()[:, 0] + 1))

    def check(self, o, lse, eps=EPS, L_max=4096, seqs=None):
        half = torch.finfo(self.dtype).eps / 2
        for s in range(len(self.new)) if seqs is None else seqs:
            at = int(self.cu[s])
            for h in range(self.H):
                if not self.new[s]:
                    continue
                ro, to, rl, tl = self.reference(s, h, eps, L_max)
                go, gl = o[at:at + self.new[s], h].double(), lse[at:at + self.new[s], h].double()
                eo, el = (go - ro).abs() / (to + half * ro.abs()), (gl - rl).abs() / tl
                assert torch.isfinite(go).all() and eo.max() <= 1, (s, h, "O", float(eo.max()))
                assert el.max() <= 1, (s, h, "lse", float(el.max()))

    def check_pages(self):
        v = {n: t for n, t in self.cache.views().items()}
        for s in range(len(self.new)):
            L = self.past[s] + self.new[s]
            pos = torch.arange(L, device="cuda")
            pg, sl = self.table[s].long()[pos // 64], pos % 64
            assert torch.equal(v["k"][pg, :, sl], self.k[s]) and torch.equal(v["v"][pg, :, sl], self.v[s])
            got = v["c"][pg, :, sl]
            # (128 runs, each added in turn, then their prefix sums; all terms of one sign)
            assert ((got - self.c[s]).abs() <= 2.0 ** -53 * (2 * L / 128 + 24) * self.c[s].abs()).all()


def serve(w, eps=EPS, **kw):
    w.fill_past()
    w.append()
    w.check_pages()
    o, lse = w.attend(eps, **kw)
    w.check(o, lse, eps)
    return o, lse


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new,past", [
    ([1], [0]), ([1], [63]), ([1], [64]), ([1, 1, 1], [500, 1, 1023]),       # single tokens
    ([5, 2, 16], [60, 0, 127]),                                              # short chunks over a page's end
    ([65], [0]), ([64], [64]), ([130, 130], [1, 190]), ([17, 63], [300, 65]),
    ([300, 1, 0, 200, 1], [700, 64, 10, 0, 2000]),                           # mixed, one without a row
])
def test_lengths(new, past, d, dtype):
    print(f"case: paged new={new} past={past} d={d} {dtype}", flush=True)
    serve(World(new, past, 3, 3, d, dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,Hk", [(1, 1), (2, 1), (6, 2), (8, 1), (32, 2), (21, 3)])
def test_shared_key_heads(H, Hk, dtype):
    for new, past in (([1, 1, 2], [100, 700, 64]), ([100, 3, 1], [130, 257, 64])):
        print(f"case: paged H={H} Hk={Hk} new={new} {dtype}", flush=True)
        serve(World(new, past, H, Hk, 64, dtype, seed=H, mu=(0.0, 6.0)))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("mu", [(-6.0, 2.0), (12.0, 20.0)])
def test_strong_and_weak_gates(mu, dtype):
    """From a decay that prunes all but a row's own page to none worth mentioning."""
    for eps in (EPS, 0.0):
        serve(World([150, 1, 9], [900, 1200, 333], 4, 2, 64, dtype, seed=3, mu=mu), eps)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_large_logits(dtype):
    serve(World([70, 1], [200, 300], 2, 2, 64, dtype, seed=4, scale=4.0))


@pytest.mark.parametrize("max_len", [1, 64, 3000, 1 << 20])
def test_any_division_of_the_keys(max_len):
    """max_len is a hint: the results stay within the tolerances for any."""
    for new, past in (([1, 2], [2500, 40]), ([200, 1], [2500, 40])):
        w = World(new, past, 2, 2, 64, BF, seed=5, mu=(6.0, 9.0))
        serve(w, max_len=max_len)


def test_token_by_token_equals_one_chunk_and_repeats():
    """Appending and attending token by token, in uneven chunks, or at once."""
    w = World([137], [0], 4, 2, 64, BF, seed=6)
    o, lse = serve(w)
    v = {n: t.clone() for n, t in w.cache.views().items()}
    w.append()                                           # the same rows again: the same pages
    for n, t in w.cache.views().items():
        assert torch.equal(t.view(torch.int16), v[n].view(torch.int16)), n
    q, k, vv, f = (w.packed(n) for n in "qkvf")
    for sizes in ([1] * 137, [3, 60, 1, 2, 71]):
        w.cache.buffer.fill_(0xff)
        at, outs = 0, []
        for n in sizes:
            cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
            past = torch.tensor([at], dtype=torch.int32, device="cuda")
            w.cache.append(k[at:at + n], vv[at:at + n], f[at:at + n], cu, past, w.table)
            outs.append(w.cache.attend(q[at:at + n], cu, past, w.table, n, gamma_q=w.gq, gamma_k=w.gk, eps=EPS,
                                       L_max=4096))
            at += n
        w.check(torch.cat([a for a, _ in outs]), torch.cat([b for _, b in outs]))
        # (one more rounding of c per chunk)
        pos = torch.arange(137, device="cuda")
        c = w.cache.views()["c"][w.table[0].long()[pos // 64], :, pos % 64]
        assert ((c - w.c[0]).abs() <= 2.0 ** -53 * 170 * w.c[0].abs()).all()


def test_strided_rows_and_rows_behind_the_last_sequence():
    w = World([40, 1, 7], [100, 64, 3], 4, 2, 64, BF, seed=7, extra_rows=9)
    w.fill_past()
    T, n = w.T, sum(w.new)
    qkv = torch.zeros((T, 8, 64), dtype=BF, device="cuda")
    qkv[:, :4], qkv[:, 4:6], qkv[:, 6:] = w.packed("q"), w.packed("k"), w.packed("v")
    qkv[n:] = float("nan")
    f = torch.full((4, T), float("nan"), device="cuda")
    f[:, :n] = w.packed("f")[:n].t()
    w.cache.append(qkv[:, 4:6], qkv[:, 6:], f.t(), w.cu, w.past_t, w.table)
    w.check_pages()
    o = torch.full((T, 4, 64), 7.0, dtype=BF, device="cuda")
    lse = torch.full((T, 4), 7.0, device="cuda")
    w.cache.attend(qkv[:, :4], w.cu, w.past_t, w.table, 40, gamma_q=w.gq, gamma_k=w.gk, eps=EPS, L_max=4096,
                   out=(o, lse))
    w.check(o, lse)
    assert (o[n:] == 7.0).all() and (lse[n:] == 7.0).all()


def test_no_sequences_and_no_rows():
    w = World([0, 0], [5, 0], 2, 2, 64, BF)
    w.fill_past()
    before = w.cache.buffer.clone()
    flags = torch.full((2, 2), -1, dtype=torch.int32, device="cuda")
    w.append(flags=flags)
    assert not flags.any() and torch.equal(before, w.cache.buffer)
    o, lse = w.attend()
    assert o.shape == (0, 2, 64) and lse.shape == (0, 2)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    o = torch.full((3, 2, 64), 7.0, dtype=BF, device="cuda")
    w.cache.attend(o, torch.zeros(1, dtype=torch.int32, device="cuda"), none, w.table[:0], 1,
                   out=(o, torch.zeros((3, 2), device="cuda")))
    assert (o == 7.0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new", [[6], [100]])
def test_values_that_are_not_finite_reach_only_their_rows(new, dtype):
    """Infinities and NaN in K or V of a later position leave the rows before it alone and
    reach those after it; a page pruned for one row but kept for another likewise."""
    w = World(new, [70], 4, 2, 64, dtype, seed=8)
    w.fill_past()
    w.append()
    clean, clean_lse = w.attend()
    bad = 70 + new[0] // 2
    for name, value in (("v", float("inf")), ("v", float("nan")), ("k", float("nan")), ("v", -float("inf"))):
        keep = getattr(w, name)[0].clone()
        getattr(w, name)[0][bad, :, 5] = value
        w.append()
        o, lse = w.attend()
        n = new[0] // 2
        assert torch.equal(o[:n], clean[:n]) and torch.equal(lse[:n], clean_lse[:n]), name
        assert not torch.isfinite(o[n:, :, 5]).any(), name
        if name == "v":
            assert torch.equal(lse, clean_lse)
            keep_cols = [i for i in range(64) if i != 5]
            assert torch.equal(o[n:][..., keep_cols], clean[n:][..., keep_cols])
        setattr(w, name, [keep])
    # a NaN in a page that strongly forgetting heads prune: head 0 unaffected, head 3 not
    w = World(new, [200], 4, 2, 64, dtype, seed=9, mu=(-4.0, 15.0))
    w.v[0][3] = float("nan")
    w.fill_past()
    w.append()
    o, _ = w.attend()
    assert torch.isfinite(o[:, 0]).all() and torch.isnan(o[:, 3]).all()


def test_bad_pages_and_flags():
    w = World([3, 80, 1], [100, 10, 200], 2, 1, 64, BF, seed=10, mu=(9.0, 9.5))
    w.fill_past()
    flags = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    w.append(flags=flags)
    assert not flags.any()
    o, lse = w.attend(flags=flags)
    assert not flags.any()
    w.check(o, lse)
    good = w.cache.buffer.clone()
    # sequence 0 loses the page of its new rows, sequence 1 its first one
    keep = w.table.clone()
    w.table[0, 1], w.table[1, 0] = w.P, -3
    w.append(flags=flags)
    assert (flags[0] & ops.FLAG_BAD_PAGE).all() and (flags[1] & ops.FLAG_BAD_PAGE).all() and not flags[2].any()
    o2, lse2 = w.attend(eps=0.0, flags=flags)
    assert (flags[0] == ops.FLAG_BAD_PAGE).all() and (flags[1] == ops.FLAG_BAD_PAGE).all() and not flags[2].any()
    w.check(o2, lse2, 0.0, seqs=[2])
    assert torch.isfinite(o2).all()
    # all of sequence 2's pages gone, and a table too narrow for sequence 1
    w.cache.buffer.copy_(good)
    w.table.copy_(keep)
    w.table[2] = 1 << 30
    o3, lse3 = w.attend(flags=flags)
    assert not o3[-1].any() and (lse3[-1] == -math.inf).all() and (flags[2] == ops.FLAG_BAD_PAGE).all()
    w.check(o3, lse3, seqs=[0, 1])
    narrow = w.table[:, :1].contiguous()
    w.cache.attend(w.packed("q"), w.cu, w.past_t, narrow, 80, flags=flags)
    assert (flags == ops.FLAG_BAD_PAGE).all()
    # gates and scales
    w.table.copy_(keep)
    f = w.packed("f").clone()
    f[0, 0], f[3, 1], f[-1, 0] = 0.5, float("nan"), -math.inf
    w.cache.append(w.packed("k"), w.packed("v"), f, w.cu, w.past_t, w.table, flags=flags)
    assert flags.tolist() == [[1, 0], [0, 2], [2, 0]]
    w.append()
    w.gq[1] = -1.0
    w.attend(flags=flags)
    assert flags.tolist() == [[0, 8]] * 3
    w.gq[1] = 1.0
    # more rows than max_new: those rows are left and reported
    o, lse = torch.full((84, 2, 64), 7.0, dtype=BF, device="cuda"), torch.full((84, 2), 7.0, device="cuda")
    w.attend(flags=flags, max_new=3, out=(o, lse))
    assert flags.tolist() == [[0, 0], [ops.FLAG_MAX_NEW] * 2, [0, 0]]
    w.check(o, lse, seqs=[0, 2])
    assert (o[3:83] == 7.0).all() and (lse[3:83] == 7.0).all()


def test_dropped_and_shared_pages():
    """Pages that every head has left out may be gone from the table; a common prefix may be
    held once."""
    w = World([2, 70], [1500, 1500], 2, 2, 64, BF, seed=11, mu=(-2.0, 0.0))
    o, lse = serve(w)
    flags = torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    w.table[:, :10] = -1
    o2, lse2 = w.attend(flags=flags)
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and not flags.any()
    w = World([3, 3], [128, 128], 2, 2, 64, BF, seed=12)
    for n in "qkvf":
        getattr(w, n)[1][:128] = getattr(w, n)[0][:128]
    w.c = [torch.cumsum(f.double(), 0) for f in w.f]
    w.table[1, :2] = w.table[0, :2]
    cu = torch.tensor([0, 128], dtype=torch.int32, device="cuda")
    w.cache.append(w.k[0][:128], w.v[0][:128], w.f[0][:128], cu, torch.zeros(1, dtype=torch.int32, device="cuda"),
                   w.table[:1])
    w.append()
    w.check(*w.attend())


def test_corrupt_call_arrays_stay_inside():
    """cu, past and table of any content touch nothing outside the call's arrays."""
    w = World([5, 70], [64, 10], 2, 2, 64, BF, seed=13)
    w.fill_past()
    w.append()
    for cu in ([0, 1000, 75], [5, 0, -3], [-7, 200, 100], [80, 90, 95]):
        w.cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
        for past in ([-5, 1 << 30], [0x7fffffff, 0x7fffffff]):
            w.past_t = torch.tensor(past, dtype=torch.int32, device="cuda")
            q = torch.zeros((75, 2, 64), dtype=BF, device="cuda")
            w.cache.append(q, q, torch.zeros((75, 2), device="cuda"), w.cu, w.past_t, w.table)
            for eps in (EPS, 0.0):
                w.cache.attend(q, w.cu, w.past_t, w.table, 75, gamma_q=w.gq, gamma_k=w.gk, eps=eps)
    torch.cuda.synchronize()


def test_a_cache_past_32_bit_offsets():
    w = World([1, 40], [200, 70], 4, 4, 128, BF, seed=14, spare=5)
    need = w.P
    P = (1 << 32) // (4 * 64 * 128) + 9                  # the last pages start past 2^32 elements
    w.cache = ops.PagedCache(P, 4, 128, 4, BF)
    w.table = torch.where(w.table >= 0, P - 1 - w.table, w.table)
    assert int(w.table.max()) == P - 1 or need <= P
    serve(w)


def test_another_stream_and_a_captured_step():
    """append() and attend() captured into a graph and replayed with new contents between
    eager calls; and on a stream that is not the default."""
    w = World([1, 1, 30], [500, 63, 100], 4, 2, 64, BF, seed=15)
    o, lse = serve(w)
    q, k, v, f = (w.packed(n) for n in "qkvf")

    def step():
        w.cache.append(k, v, f, w.cu, w.past_t, w.table)
        return w.cache.attend(q, w.cu, w.past_t, w.table, 30, gamma_q=w.gq, gamma_k=w.gk, eps=EPS, L_max=4096)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a, b = step()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, o) and torch.equal(b, lse)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    for r in range(3):
        for x in (q, k, v):
            x.copy_(x.roll(1, 0))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        w.cache.buffer[:64].add_(0)
        for g, out in graphs:
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), r


@pytest.mark.parametrize("dtype", [BF, F32])
def test_sixteen_query_heads_of_128_features(dtype):
    """The most query heads per key head beside the widest rows, as single tokens and a chunk."""
    for new, past in (([1, 1], [700, 63]), ([20, 1], [300, 64])):
        serve(World(new, past, 32, 2, 128, dtype, seed=16, mu=(0.0, 7.0)))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new,past", [([1], [60000]), ([100], [20000]), ([3, 1], [30000, 1])])
def test_long_sequences_in_many_shares(new, past, dtype):
    """Few rows over many pages: their sums are merged from dozens of workgroups."""
    w = World(new, past, 2, 1, 64, dtype, seed=17, mu=(9.0, 11.0))
    w.fill_past()
    w.append()
    for eps in (0.0, EPS):
        w.check(*w.attend(eps, L_max=1 << 16), eps=eps, L_max=1 << 16)


@pytest.mark.parametrize("max_len", [1 << 12, 64])
def test_many_ragged_sequences(max_len):
    """More (sequence, head) items than are shared out, and as many that are, some without a
    row; then all of them with a chunk."""
    N = 1100
    new = [(0, 1, 1, 2, 1, 5, 1)[i % 7] for i in range(N)]
    past = [(i * 37) % 180 for i in range(N)]
    w = World(new, past, 4, 4, 64, BF, seed=18, mu=(1.0, 6.0))
    w.fill_past()
    w.append()
    some = [0, 1, 2, 3, 5, 6, 550, 1095, 1096, 1099]
    w.check(*w.attend(max_len=max_len), seqs=some)
    new = [(0, 1, 33, 70)[i % 4] for i in range(300)]
    w = World(new, [(i * 41) % 900 for i in range(300)], 8, 2, 64, BF, seed=19, mu=(1.0, 6.0))
    w.fill_past()
    w.append()
    w.check(*w.attend(max_len=max_len), seqs=[0, 1, 2, 3, 150, 151, 297, 298, 299])


def test_two_calls_at_once():
    """Calls on two streams at a time read the same cache and keep to their own scratch."""
    w = World([1, 40, 1, 9], [3000, 800, 64, 100], 4, 2, 64, BF, seed=20, mu=(5.0, 8.0))
    o, lse = serve(w)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for st in streams:
            with torch.cuda.stream(st):
                outs.append(w.attend())
    for st in streams:
        torch.cuda.current_stream().wait_stream(st)
    for a, b in outs:
        assert torch.equal(a, o) and torch.equal(b, lse)


def test_operator_timing_counts_calls():
    w = World([1, 30], [100, 20], 2, 2, 64, BF, seed=21)
    acp.acp_timing_reset()
    acp.acp_timing_enable(True)
    try:
        serve(w)
    finally:
        acp.acp_timing_enable(False)
    t = ops.acp_op_timing_read()
    acp.acp_timing_reset()
    assert t["append"][0] == 2 and t["attend"][0] == 1 and t["norm"] == (0, 0.0)
    assert 0.0 < t["attend"][1] < 1000.0 and 0.0 < t["append"][1] < 1000.0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,scale", [(64, 2.1), (64, 2.5), (64, 2.6), (128, 2.1), (128, 2.2)])
def test_scales_on_both_sides_of_a_known_reference(d, scale, dtype):
    """U = scale^2 sqrt(d) above 32 (35 to 50) and above 52: the two ways in which the weights of
    a chunk are kept in float32's range."""
    serve(World([100, 1], [300, 200], 2, 1, d, dtype, seed=22, scale=scale, mu=(2.0, 7.0)))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("forget", [5.0, 20.0])
@pytest.mark.parametrize("new,past", [([1], [63]), ([40], [24]), ([100], [60])])
def test_the_keys_that_count_come_after_forgotten_ones(new, past, forget, dtype):
    """Queries of one feature, gates that forget e^-5 or e^-20 a position: what the
    softmax is first scaled by is far below the row's own logit, which is k_5, below 5.  Its own key
    counts, and the one before with e^-5 times e^(k_5 - k_5') at most: a logit, one product and one
    decay, is rounded with 4 e |logit| + 4 e <= 24 e, a decay with 6 e times its weight, a power of
    two with 2 e, and sums of at most 16 + 8 terms, the scales of four waves and the division with
    40 e; the logits' bound as reference, 8, adds 20 e: 100 e covers lse, and O relative to max |v|
    but for the weights' and its own rounding to bfloat16."""
    w = World(new, past, 16, 16, 64, dtype, seed=23, mu=(-forget - 0.2, -forget + 0.2))
    w.q = [torch.zeros_like(t) for t in w.q]
    for t in w.q:
        t[..., 5] = 8.0
    assert max(float(k[..., 5].abs().max()) for k in w.k) < 5.0
    w.fill_past()
    w.append()
    for eps in (EPS, 0.0):
        o, lse = w.attend(eps)
        for h in range(16):
            ro, _, rl, _ = w.reference(0, h, eps, 4096)
            vmax = w.v[0][:, h].abs().max().double()
            assert (lse[:, h].double() - rl).abs().max() <= 100 * E, (h, float((lse[:, h].double() - rl).abs().max() / E))
            assert (o[:, h].double() - ro).abs().max() <= (100 * E + (2.0 ** -7 if dtype == BF else 0.0)) * vmax, h


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("new,past", [([100], [100]), ([1], [150]), ([12], [100]), ([3, 90], [110, 0])])
@pytest.mark.parametrize("gate", [-1e4, -1e7, float(torch.finfo(torch.float32).min)])
def test_a_gate_that_forgets_everything(new, past, dtype, gate):
    """As between two texts: no row after it attends to a position before it.  A gate whose sum
    leaves float64 too few bits for the gates after it is reported."""
    w = World(new, past, 4, 2, 64, dtype, seed=24, mu=(2.0, 7.0))
    for s in range(len(new)):
        w.f[s][past[s] + new[s] // 2 if new[s] > 1 else 70] = gate
    w.c = [torch.cumsum(f.double(), 0) for f in w.f]
    w.fill_past()
    flags = torch.zeros((len(new), 4), dtype=torch.int32, device="cuda")
    w.append(flags=flags)
    w.check_pages()
    far = gate < -2.0 ** 32
    assert (flags == (4 if far else 0)).all()
    for eps in (EPS, 0.0):
        w.check(*w.attend(eps), eps)


def test_sums_that_leave_the_range_are_reported():
    low = float(torch.finfo(torch.float32).min)
    for new in ([9], [100]):
        w = World(new, [3], 2, 2, 64, BF, seed=25)
        w.f[0][5, 0], w.f[0][8, 0] = low, low            # c = -6.8e38
        w.f[0][6, 1] = -2.0 ** 31
        w.fill_past()
        flags = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
        w.append(flags=flags)
        assert flags.tolist() == [[6, 0]]
        w.f[0][7, 1] = -2.0 ** 31
        w.append(flags=flags)
        assert flags.tolist() == [[6, 4]]


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_whose_own_page_is_bad(dtype):
    """They attend to the pages that the tile's first row keeps, with c_i = 0: logits far above
    the scales' bound.  Weights and O are off by 2^-8 and 2^-9 of max |v| in bfloat16, float32's
    logits, of at most 200, by 1000 e."""
    w = World([80], [300], 3, 3, 64, dtype, seed=26, mu=(0.3, 0.6))
    w.fill_past()
    w.append()
    w.table[0, 5] = -1                                   # positions 320 to 383
    flags = torch.zeros((1, 3), dtype=torch.int32, device="cuda")
    o, lse = w.attend(flags=flags)
    assert (flags == ops.FLAG_BAD_PAGE).all() and torch.isfinite(lse).all()
    for h in range(3):
        c, k, v = w.c[0][:, h], w.k[0][:, h].double(), w.v[0][:, h].double()
        assert float(c[300]) < -90.0
        delta = -(2 * 8.0 + math.log(4096) + 10.0)
        lo = next(n for n in range(5) if n == 4 or c[300] - c[64 * n + 63] >= delta)
        x = w.q[0][320:, h].double() @ k[64 * lo:320].t() / 8 - c[None, 64 * lo:320]
        p = torch.softmax(x, 1)
        lim = (2.0 ** -7 if dtype == BF else 1000 * E) * float(v.abs().max())
        assert (o[20:, h].double() - p @ v[64 * lo:320]).abs().max() <= lim, h
        assert (lse[20:, h].double() - torch.logsumexp(x, 1)).abs().max() <= 1000 * E * 200, h
