"""prq_tree_attention against the float64 oracle: head sizes and groups, page sizes, requests of no,
one and many rows and of no and many cached tokens, trees, chains, masks that leave rows empty, splits
of the keys, garbage where nothing may be read.

Bar, per element of out (P = sum_j p_j |v_j| and S = scale * max_j sum_d |q_d k_d| from the oracle):
  2^-8 |out|            the output's rounding to bf16
  2^-8 P                each probability's rounding to bf16
  2^-18 (S + 16) P      float32 scores (D products of relative error 2^-24 each, at most 256 of
                        them), the exponential's argument and the sums, all relative to P
lse: 2^-18 (S + 16) + 2^-22 |lse|."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention as at            # noqa: E402
from tests.gpu_util import say                # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _prq():
    from paper_2609_22106_amd import prq
    return prq


def _tree(rng, n):
    see = np.zeros((n, n), bool)
    for i in range(n):
        parent = int(rng.integers(-1, i)) if i else -1
        if parent >= 0:
            see[i] = see[parent]
        see[i, i] = True
    return see


class Case:
    """Requests [(cached, rows), ...] with their tokens on shuffled pages; everything that no row may
    see -- the rest of the last pages, unused pages, unused page-table entries -- is garbage."""

    def __init__(self, requests, Hq, Hk, D, page, seed=0, mask="tree", wide=None, garbage=float("nan"), size=1.5):
        rng = np.random.default_rng(seed)
        self.requests, self.Hq, self.Hk, self.D, self.page = requests, Hq, Hk, D, page
        n = [r for _, r in requests]
        M = sum(n)
        used = [-(-(c + r) // page) for c, r in requests]
        pages = sum(used) + 3
        order = rng.permutation(pages)
        width = max(used + [1]) + 1
        table = np.full((len(requests), width), 1 << 30, np.int32)      # past the pool
        K = torch.full((pages, Hk, page, D), garbage, dtype=BF16, device="cuda")
        V = torch.full((pages, Hk, page, D), garbage, dtype=BF16, device="cuda")
        self.keys, self.values, at_page = [], [], 0
        g = torch.Generator(device="cuda").manual_seed(seed)
        for b, (c, r) in enumerate(requests):
            ids = order[at_page:at_page + used[b]]
            at_page += used[b]
            table[b, :used[b]] = ids
            L = c + r
            k = torch.randn(L, Hk, D, generator=g, device="cuda").to(BF16)
            v = (torch.randn(L, Hk, D, generator=g, device="cuda") + 0.3).to(BF16)
            slot = torch.arange(L, device="cuda")
            at_ = torch.from_numpy(ids.astype(np.int64)).cuda()
            if L:
                K[at_[slot // page], :, slot % page] = k
                V[at_[slot // page], :, slot % page] = v
            self.keys.append(k)
            self.values.append(v)
        self.q = (size * torch.randn(M, Hq, D, generator=g, device="cuda")).to(BF16)
        self.cache = _prq().PagedKV(K, V)
        self.table = torch.from_numpy(table).cuda()
        self.cached = torch.tensor([c for c, _ in requests], dtype=torch.int32, device="cuda")
        self.offsets = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32, device="cuda")
        self.scale = 1.0 / D ** 0.5
        self.mask = None
        if mask is not None:
            w = max(n + [0]) if wide is None else wide
            m = np.ones((M, w), bool)                                   # columns past a request's rows: set
            row = 0
            for r in n:
                one = {"tree": lambda: _tree(rng, r), "self": lambda: np.eye(r, dtype=bool),
                       "none": lambda: np.zeros((r, r), bool),
                       "any": lambda: rng.random((r, r)) < 0.4}[mask]()
                m[row:row + r, :min(r, w)] = one[:, :w]
                row += r
            self.mask = torch.from_numpy(m).cuda()

    def run(self, **kw):
        kw.setdefault("max_kv_len", max([c + r for c, r in self.requests] + [0]))
        M = self.q.shape[0]
        kw.setdefault("out", torch.full((M, self.Hq, self.D), float("nan"), dtype=BF16, device="cuda"))
        kw.setdefault("lse", torch.full((M, self.Hq), float("nan"), device="cuda"))
        return _prq().prq_tree_attention(self.q, self.cache, self.table, self.cached, self.offsets, self.scale,
                                         tree_mask=self.mask, **kw)

    def check(self, out, lse, keys=None, values=None):
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        q = self.q.double().cpu().numpy()
        mask = None if self.mask is None else self.mask.cpu().numpy()
        row = 0
        for b, (c, r) in enumerate(self.requests):
            k = (self.keys[b] if keys is None else keys[b]).double().cpu().numpy()
            v = (self.values[b] if values is None else values[b]).double().cpu().numpy()
            rows = slice(row, row + r)
            want, wl, spread, size = at.tree_attention(q[rows], k, v, c, self.scale,
                                                       None if mask is None else mask[rows, :r])
            S = (self.scale * size + 16)[..., None]
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -18 * S) * spread
            err = np.abs(out[rows] - want)
            assert np.all(err <= tol), (b, float(np.max(err - tol)))
            empty = np.isneginf(wl)
            assert np.array_equal(np.isneginf(lse[rows]), empty)
            err = np.abs(lse[rows][~empty] - wl[~empty])
            assert np.all(err <= 2.0 ** -18 * S[..., 0][~empty] + 2.0 ** -22 * np.abs(wl[~empty])), float(err.max())
            row += r


CASES = [
    # requests, Hq, Hk, D, page
    ([(0, 1)], 1, 1, 64, 16), ([(1, 1)], 4, 1, 128, 16), ([(0, 0), (5, 1), (0, 0), (31, 1)], 8, 2, 64, 16),
    ([(33, 1)] * 5, 32, 8, 128, 64), ([(127, 1), (128, 1), (129, 1), (0, 1)], 8, 8, 128, 128),
    ([(700, 3), (15, 13), (16, 1), (0, 7)], 6, 2, 64, 32), ([(100, 16), (90, 5)], 12, 3, 128, 16),
    ([(1000, 64), (37, 33)], 8, 2, 128, 16), ([(1023, 65)], 4, 4, 64, 64), ([(250, 9), (3, 2)], 16, 1, 128, 16),
    ([(77, 5), (500, 20)], 4, 2, 256, 16), ([(40, 70)], 5, 1, 256, 32), ([(2000, 1), (3, 1)], 40, 2, 64, 256),
    ([(64, 3)], 64, 1, 128, 16), ([(5000, 2)], 2, 1, 128, 4096), ([(300, 17)] * 3, 21, 7, 64, 16)]


@pytest.mark.parametrize("requests,Hq,Hk,D,page", CASES)
@pytest.mark.parametrize("mask", ["tree", "any", None])
def test_matches_oracle(requests, Hq, Hk, D, page, mask):
    say("tree attention", requests, Hq, Hk, D, page, mask)
    c = Case(requests, Hq, Hk, D, page, seed=len(requests) + D, mask=mask)
    c.check(*c.run())


def test_many_requests_of_one_token():
    rng = np.random.default_rng(5)
    c = Case([(int(rng.integers(0, 200)), 1) for _ in range(150)], 8, 2, 64, 16, mask=None)
    c.check(*c.run())


def test_masks_that_leave_rows_empty():
    """No own token seen: the cached ones alone, or nothing at all (0 and -inf)."""
    for mask, wide in (("none", None), ("none", 0), ("self", 2)):
        say("empty rows", mask, wide)
        c = Case([(0, 5), (40, 3), (0, 1)], 4, 2, 128, 16, mask=mask, wide=wide)
        out, lse = c.run()
        c.check(out, lse)
        if mask == "none":
            assert not out[:5].any() and not out[8:].any() and bool(torch.isneginf(lse[:5]).all())


def test_a_long_chunk_of_a_prompt():
    c = Case([(50, 300), (0, 129)], 4, 2, 64, 16, mask=None)
    c.check(*c.run())


@pytest.mark.parametrize("max_kv", [0, 1, 64, 300, 10 ** 6])
def test_max_kv_len_is_only_a_plan(max_kv):
    c = Case([(300, 4), (2, 1)], 8, 2, 64, 16)
    c.check(*c.run(max_kv_len=max_kv))


def test_unseen_infinities_and_nan_do_not_reach_a_row():
    """Own token 3 holds NaN and infinities that rows 3.. do or do not see: a row that sees them has
    them where they are, every other row is as without them."""
    for D, Hq, Hk in ((64, 4, 2), (128, 32, 8), (256, 2, 2)):
        c = Case([(45, 8), (10, 4)], Hq, Hk, D, 16, mask="tree", seed=D)
        c.mask[:8, 3] = False
        c.mask[5, 3] = True
        page, at_ = c.table[0, 48 // 16].item(), 48 % 16
        c.check(*c.run())
        clean = c.run()
        V = c.cache.V
        V[page, :, at_, 7], V[page, :, at_, 8] = float("nan"), float("inf")
        out, lse = c.run()
        keep = torch.ones(12, Hq, D, dtype=torch.bool, device="cuda")
        keep[5, :, 7:9] = False
        assert bool(torch.isnan(out[5, :, 7]).all()) and bool((out[5, :, 8] == float("inf")).all())
        assert bool((out[keep].float() - clean[0][keep].float()).abs().max() < 2.0 ** -5)
        assert torch.equal(lse, clean[1])
        c.cache.K[page, :, at_] = float("nan")
        out, lse = c.run()
        assert bool(torch.isnan(out[5]).all()) and bool(torch.isnan(lse[5]).all())
        rows = [r for r in range(12) if r != 5]
        assert bool(torch.isfinite(out[rows]).all()) and torch.equal(lse[rows], clean[1][rows])


def test_large_scores_and_scores_of_minus_infinity():
    """Scores that pass the maximum by far, rising and falling along the keys; a seen key of -inf."""
    for falling in (False, True):
        c = Case([(600, 2)], 2, 1, 64, 16, mask=None, size=1.0)
        k = c.keys[0]
        ramp = torch.linspace(40 * falling, 40 * (not falling), 602, device="cuda")
        k[:, :, 0] = ramp[:, None].to(BF16)
        slot = torch.arange(602, device="cuda")
        c.cache.K[c.table[0].long()[slot // 16], :, slot % 16] = k
        c.q[:, :, 0] = 20
        c.check(*c.run())
    c = Case([(5, 1)], 1, 1, 64, 16, mask=None)
    c.cache.K[c.table[0, 0].item(), :, 2, 0] = float("-inf")
    c.q[:, :, 0] = 1.0
    out, lse = c.run()
    keep = [0, 1, 3, 4, 5]
    c.requests = [(4, 1)]
    c.check(out, lse, keys=[c.keys[0][keep]], values=[c.values[0][keep]])


def test_pages_outside_the_pool_are_not_seen():
    c = Case([(100, 1)], 4, 2, 64, 16, mask=None)
    for bad in (-1, c.cache.pages, -(1 << 31)):
        t = c.table.clone()
        t[0, 2] = bad
        keep = [i for i in range(101) if not 32 <= i < 48]
        M = c.q.shape[0]
        out, lse = _prq().prq_tree_attention(c.q, c.cache, t, c.cached, c.offsets, c.scale, max_kv_len=101)
        one = Case.__new__(Case)
        one.__dict__.update(c.__dict__, requests=[(len(keep) - 1, 1)])
        assert M == 1
        one.check(out, lse, keys=[c.keys[0][keep]], values=[c.values[0][keep]])


def test_lengths_past_the_page_table_are_cut():
    c = Case([(60, 1)], 2, 1, 64, 16, mask=None)
    c.cached[0] = 1 << 30
    out, lse = _prq().prq_tree_attention(c.q, c.cache, c.table[:, :2], c.cached, c.offsets, c.scale)
    c.requests = [(32, 1)]
    c.check(out, lse, keys=[c.keys[0][:32]], values=[c.values[0][:32]])
    c.cached[0] = -5                                    # taken as 0: the row's own token alone, at slot 0
    out, lse = _prq().prq_tree_attention(c.q, c.cache, c.table[:, :2], c.cached, c.offsets, c.scale)
    c.requests = [(0, 1)]
    c.check(out, lse, keys=[c.keys[0][:1]], values=[c.values[0][:1]])


def test_offsets_outside_the_rows_are_clamped():
    c = Case([(20, 3), (9, 2)], 2, 1, 64, 16, mask=None)
    want = c.run()
    c.offsets = torch.tensor([0, 3, 99], dtype=torch.int32, device="cuda")
    got = c.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_strided_queries_masks_tables_and_pools():
    c = Case([(300, 7), (90, 12)], 8, 2, 128, 16, mask="tree")
    want = c.run()
    M = c.q.shape[0]
    wide = torch.randn(M, 13 * 128, device="cuda").to(BF16)
    wide[:, 128:9 * 128] = c.q.view(M, -1)
    c.q = wide[:, 128:9 * 128].unflatten(1, (8, 128))
    m = torch.ones(M, 40, dtype=torch.bool, device="cuda")
    m[:, 3:15] = c.mask
    c.mask = m[:, 3:15]
    t = torch.full((2, 99), -7, dtype=torch.int32, device="cuda")
    t[:, 5:5 + c.table.shape[1]] = c.table
    c.table = t[:, 5:5 + c.table.shape[1]]
    pool = torch.stack([c.cache.K, c.cache.V], 1)
    c.cache = _prq().PagedKV(pool[:, 0], pool[:, 1])
    got = c.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_pool_past_32_bits():
    Hk, page, D = 8, 16, 128
    c = Case([(70, 2), (33, 1)], 16, Hk, D, page, mask=None)
    want = c.run()
    pages = (1 << 31) // (Hk * page * D) + 700
    K = torch.empty(pages, Hk, page, D, dtype=BF16, device="cuda")
    V = torch.empty(pages, Hk, page, D, dtype=BF16, device="cuda")
    n = c.cache.pages
    K[-n:], V[-n:] = c.cache.K, c.cache.V
    c.table = torch.where(c.table < n, c.table + (pages - n), c.table)
    c.cache = _prq().PagedKV(K, V)
    got = c.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_calls_repeat_bit_for_bit_and_leave_the_state_head_zero():
    """Whatever the scratch behind the head held, and for calls of other sizes in between."""
    prq = _prq()
    c = Case([(3000, 2), (100, 1)], 32, 8, 128, 64)
    other = Case([(1500, 40)], 8, 2, 64, 16)
    need = prq.prq_tree_attention_workspace_bytes(3, 2, 32, 8, 128, 3002)
    assert need > 16384
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    a = c.run(workspace=ws)
    for fill in (255, 1):
        ws[16384:] = fill
        b = c.run(workspace=ws)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        other.check(*other.run(workspace=ws))
        assert not ws[:16384].any()
    d = c.run()
    assert torch.equal(a[0], d[0]) and torch.equal(a[1], d[1])
    with pytest.raises(prq.PRQError) as e:
        c.run(workspace=torch.zeros(need - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.status == prq.PRQ_EWORKSPACE


def test_uneven_requests_share_the_chip():
    """One long request among short ones, more requests than a wave has lanes, and both."""
    rng = np.random.default_rng(3)
    for requests in ([(9000, 1)] + [(int(rng.integers(0, 60)), 1) for _ in range(20)],
                     [(int(rng.integers(0, 400)), int(rng.integers(0, 3))) for _ in range(70)] + [(4000, 2)],
                     [(5000, 9), (0, 0), (17, 30), (2500, 3)]):
        say("uneven", requests[:3])
        c = Case(requests, 4, 1, 64, 16)
        c.check(*c.run())


def test_no_rows_and_no_requests():
    prq = _prq()
    c = Case([(3, 1)], 2, 1, 64, 16, mask=None)
    out, lse = prq.prq_tree_attention(c.q[:0], c.cache, c.table, c.cached, c.offsets * 0, c.scale)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)
    with pytest.raises(ValueError):
        prq.prq_tree_attention(c.q, c.cache, c.table, c.cached, c.offsets[:1], c.scale)
    with pytest.raises(ValueError):
        prq.prq_tree_attention(c.q, c.cache, c.table.long(), c.cached, c.offsets, c.scale)
    with pytest.raises(ValueError):
        prq.prq_tree_attention(c.q, c.cache, c.table, c.cached, c.offsets, c.scale,
                               tree_mask=torch.ones(2, 1, dtype=torch.bool, device="cuda"))           # rows


@pytest.mark.parametrize("rows,D,page", [(1, 128, 16), (5, 64, 64), (13, 128, 16), (13, 64, 32), (13, 256, 16),
                                         (20, 128, 64), (20, 64, 16), (40, 128, 16), (40, 64, 64), (64, 128, 128)])
def test_long_parts(rows, D, page):
    """Many kv heads leave few workgroups to a head, so that each goes through more than a thousand
    keys, of which one page is missing; against float64 products on the device (same bars)."""
    Hk, G = 32, 4
    g = torch.Generator(device="cuda").manual_seed(rows + D)
    cached = [2500 + 37 * i for i in range(7)] + [31]
    n = [rows - (i % 3 if rows > 3 else 0) for i in range(8)]
    used = [-(-(c + r) // page) for c, r in zip(cached, n)]
    order = torch.randperm(sum(used), generator=g, device="cuda").int()
    table = torch.full((8, max(used)), -1, dtype=torch.int32, device="cuda")
    for b in range(8):
        table[b, :used[b]] = order[sum(used[:b]):sum(used[:b + 1])]
    table[3, 1600 // page] = -1
    K, V = ((torch.randn(sum(used), Hk, page, D, generator=g, device="cuda") + 0.2 * i).to(BF16) for i in range(2))
    q = (1.5 * torch.randn(sum(n), Hk * G, D, generator=g, device="cuda")).to(BF16)
    mask = torch.rand(sum(n), rows, generator=g, device="cuda") < 0.5
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32, device="cuda")
    say("long parts", rows, D, page)
    out, lse = _prq().prq_tree_attention(q, _prq().PagedKV(K, V), table,
                                         torch.tensor(cached, dtype=torch.int32, device="cuda"), offsets, D ** -0.5,
                                         mask)
    at_ = 0
    for b in range(8):
        L, r = cached[b] + n[b], slice(at_, at_ + n[b])
        at_ += n[b]
        ids = table[b, :used[b]].long()
        there = (ids >= 0).repeat_interleave(page)[:L]
        k, v = (t[ids.clamp(min=0)].transpose(1, 2).reshape(-1, Hk, D)[:L].transpose(0, 1).double() for t in (K, V))
        qb = q[r].reshape(n[b], Hk, G, D).permute(1, 2, 0, 3).reshape(Hk, G * n[b], D).double()
        see = there.repeat(n[b], 1)
        see[:, cached[b]:] &= mask[r, :n[b]]
        s = (qb @ k.transpose(1, 2).contiguous()) * D ** -0.5
        s = s.masked_fill(~see.repeat(G, 1), float("-inf"))
        want_l = torch.logsumexp(s, -1)
        p = torch.exp(s - want_l[..., None])
        want, spread = p @ v, p @ v.abs()
        size = (qb.abs() @ k.abs().transpose(1, 2).contiguous()).amax(-1)
        S = (D ** -0.5 * size + 16)[..., None]
        rows_of = lambda t: t.reshape(n[b], Hk, G, -1).permute(1, 2, 0, 3).reshape(Hk, G * n[b], -1).double()  # noqa
        err = (rows_of(out[r]) - want).abs()
        assert bool((err <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -18 * S) * spread).all()), (b, float(err.max()))
        err = (rows_of(lse[r])[..., 0] - want_l).abs()
        assert bool((err <= 2.0 ** -18 * S[..., 0] + 2.0 ** -22 * want_l.abs()).all()), (b, float(err.max()))


@pytest.mark.parametrize("rows,D", [(3, 128), (10, 64), (20, 64), (20, 128), (24, 256), (40, 64), (40, 128)])
def test_infinities_and_nan_among_many_columns(rows, D):
    """NaN and infinities in an own token that few rows see, in a cached one that all see, and on a
    page that is missing."""
    Hq, Hk = 8, 2
    c = Case([(75, rows), (200, rows)], Hq, Hk, D, 16, mask="any", seed=rows)
    c.mask[:, 2] = False
    c.mask[1, 2] = c.mask[rows - 1, 2] = True
    c.check(*c.run())
    clean = c.run()
    V, slot = c.cache.V, 75 + 2
    page, at_ = c.table[0, slot // 16].item(), slot % 16
    V[page, :, at_, 3], V[page, :, at_, D - 1] = float("-inf"), float("nan")
    out, lse = c.run()
    sees = torch.zeros(2 * rows, dtype=torch.bool, device="cuda")
    sees[[1, rows - 1]] = True
    assert bool((out[sees][..., 3] == float("-inf")).all()) and bool(torch.isnan(out[sees][..., D - 1]).all())
    assert torch.equal(out[~sees], clean[0][~sees]) and torch.equal(lse, clean[1])
    between = torch.ones(D, dtype=torch.bool, device="cuda")
    between[[3, D - 1]] = False
    assert bool((out[sees][..., between].float() - clean[0][sees][..., between].float()).abs().max() < 2.0 ** -5)
    # an infinity that every row sees, among the cached tokens: all of the request's rows have it
    V[c.table[1, 100 // 16].item(), :, 100 % 16, 5] = float("inf")
    out, _ = c.run()
    assert bool((out[rows:, :, 5] == float("inf")).all())
    assert torch.equal(out[:rows][~sees[:rows]], clean[0][:rows][~sees[:rows]])
    # on a page that is missing from the table, nothing of it is left
    c.table[1, 100 // 16] = -1
    out, _ = c.run()
    assert bool(torch.isfinite(out[rows:]).all())


@pytest.mark.parametrize("rows,D", [(1, 64), (4, 128), (5, 64), (9, 256), (10, 64), (10, 128), (20, 64), (40, 128)])
def test_rows_of_no_request_are_left_alone(rows, D):
    """16, 64, 128 and 256 columns a workgroup, the keys split: rows before the first offset and from
    the last one on keep what out and lse held, whatever an earlier call or a program left in the
    workspace behind its head."""
    prq = _prq()
    c = Case([(600, rows), (900, rows), (700, rows)], 8, 2, D, 16, seed=rows)
    M = 3 * rows
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    assert prq.prq_tree_attention_workspace_bytes(M, 1, 8, 2, D, 940) > 16384
    outs = [torch.full(s, 7.0, dtype=t, device="cuda") for s, t in (((M, 8, D), BF16), ((M, 8), torch.float32))]

    def one(b, out, lse):                                            # request b's rows alone
        return prq.prq_tree_attention(c.q, c.cache, c.table[b:b + 1], c.cached[b:b + 1],
                                      c.offsets[b:b + 2].contiguous(), c.scale, tree_mask=c.mask, max_kv_len=940,
                                      out=out, lse=lse, workspace=ws)
    for fill in (0, 1, 255):
        say("rows of no request", rows, D, fill)
        ws[16384:] = fill
        for t in outs:
            t.fill_(7.0)
        one(1, *outs)
        assert bool((outs[0][:rows] == 7).all()) and bool((outs[0][2 * rows:] == 7).all())
        assert bool((outs[1][:rows] == 7).all()) and bool((outs[1][2 * rows:] == 7).all())
        mine = [t[rows:2 * rows].clone() for t in outs]
        one(2, *outs)                                                # (in the parts that the call before has left)
        one(0, *outs)
        assert torch.equal(outs[0][rows:2 * rows], mine[0]) and torch.equal(outs[1][rows:2 * rows], mine[1])
        c.check(*outs)
        assert not ws[:16384].any()


def test_offsets_that_rise_and_fall_leave_the_workspace_ready():
    """More than 64 requests, rows counted twice: more tiles and parts than the launch was planned for.
    Every part of a tile that is begun has its workgroup all the same, so the state head is zero again,
    and a call with a table in order is as on a workspace of its own."""
    prq = _prq()
    M, Hq, Hk, D, page, L = 70, 32, 8, 64, 256, 3840
    g = torch.Generator(device="cuda").manual_seed(1)
    K, V = (torch.randn(L // page + 1, Hk, page, D, generator=g, device="cuda").to(BF16) for _ in range(2))
    q = torch.randn(M, Hq, D, generator=g, device="cuda").to(BF16)
    offsets = torch.tensor([0, M] + list(range(M - 1)), dtype=torch.int32, device="cuda")
    B = len(offsets) - 1
    pages = torch.arange(L // page + 1, dtype=torch.int32, device="cuda").repeat(B, 1)
    # the first request has all rows and no cached tokens, 54 of those with a row have many
    cached = torch.tensor([0, 0] + [L - 1] * 54 + [0] * (B - 56), dtype=torch.int32, device="cuda")
    need = prq.prq_tree_attention_workspace_bytes(M, B, Hq, Hk, D, L)
    assert need > 16384

    def call(offsets, ws):
        return prq.prq_tree_attention(q, prq.PagedKV(K, V), pages, cached, offsets, D ** -0.5, max_kv_len=L,
                                      workspace=ws)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    say("offsets that rise and fall")
    out, lse = call(offsets, ws)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    assert not ws[:16384].any()
    in_order = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    got, want = call(in_order, ws), call(in_order, torch.zeros(need, dtype=torch.uint8, device="cuda"))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert not ws[:16384].any()


@pytest.mark.parametrize("max_kv", [(1 << 31) - 1, 1 << 40])
def test_no_bound_on_the_lengths(max_kv):
    """The plan of the longest requests there may be: the bits of one that is long enough."""
    c = Case([(900, 4), (2, 1)], 8, 2, 64, 16)
    want, got = c.run(max_kv_len=1 << 20), c.run(max_kv_len=max_kv)
    c.check(*got)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("rows", [1, 9, 30])
@pytest.mark.parametrize("scale", [-0.07, 0.0, -0.0, 1e-35, -2.5])
def test_scales_of_either_sign_and_zero(rows, scale):
    """Scores of either sign; with a scale of 0 every seen key weighs alike.  (Bars as above, the size
    of the scores with the scale's magnitude.)"""
    say("scale", scale, rows)
    c = Case([(200, rows), (0, rows)], 8, 2, 64, 16, seed=rows)
    c.scale = scale
    out, lse = c.run()
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    q, mask = c.q.double().cpu().numpy(), c.mask.cpu().numpy()
    for b, at_ in enumerate((slice(0, rows), slice(rows, 2 * rows))):
        k, v = c.keys[b].double().cpu().numpy(), c.values[b].double().cpu().numpy()
        want, wl, spread, size = at.tree_attention(q[at_], k, v, c.requests[b][0], float(np.float32(scale)), mask[at_])
        S = (abs(scale) * size + 16)[..., None]
        assert np.all(np.abs(out[at_] - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -18 * S) * spread)
        assert np.all(np.abs(lse[at_] - wl) <= 2.0 ** -18 * S[..., 0] + 2.0 ** -22 * np.abs(wl))
