"""prq_qk_norm_rope against the float64 oracle: every head size, both pair layouts, part of the
head, with and without norm, both input types, strides, padding rows, slots past 32 bits.

Bar, per element: one rounding to bf16 (2^-8 of the value) and the float32 chain behind it, whose
error is relative to the magnitudes that are added, not to their difference: 2^-18 of the head's
largest normed value (64 float32 roundings; the longest chain is the mean's 3 + log2 terms, the
root, two products and the sum of two)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention as at            # noqa: E402
from tests.gpu_util import say                # noqa: E402

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _prq():
    from paper_2609_22106_amd import prq
    return prq


def _make(M, Hq, Hk, D, rot, page, dtype, norm, seed, positions=64, w_dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    pages = M // page + 4
    c = dict(q=(3 * rnd(M, Hq * D)).to(dtype), k=(3 * rnd(M, Hk * D)).to(dtype), v=rnd(M, Hk * D).to(dtype),
             pos=torch.randint(0, positions, (M,), generator=g, device="cuda", dtype=torch.int32),
             slots=torch.randperm(pages * page, generator=g, device="cuda")[:M].contiguous(),
             wq=(1 + 0.3 * rnd(D)).to(w_dtype) if norm else None, wk=(1 + 0.3 * rnd(D)).to(w_dtype) if norm else None)
    c["table"] = _prq().prq_rope_table(positions, rot, theta=1e4) if rot else None
    c["cache"] = _prq().PagedKV(rnd(pages, Hk, page, D).bfloat16(), rnd(pages, Hk, page, D).bfloat16())
    return c


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _check(c, got, K0, V0, D, inter):
    """All of q, and all of the pool: written slots as the oracle, every other one untouched."""
    q, k, v, table = (_np(c[n]) for n in ("q", "k", "v", "table"))
    pos, slots = c["pos"].cpu().numpy(), c["slots"].cpu().numpy()
    cache = c["cache"]
    K, V = _np(cache.K), _np(cache.V)
    wantK, wantV = _np(K0), _np(V0)
    page = cache.page_size
    M = q.shape[0]

    def near(a, b):
        assert np.all(np.abs(a - b) <= 2.0 ** -8 * np.abs(b) + 2.0 ** -18 * np.max(np.abs(b)) * 2), \
            float(np.max(np.abs(a - b)))
    out = _np(got)
    for i in range(M):
        turn = [] if table is None else table[pos[i]]
        for h in range(q.shape[1] // D):
            near(out[i, h], at.norm_rotate(q[i, h * D:(h + 1) * D], _np(c["wq"]), EPS, turn, inter))
        s = slots[i]
        if not 0 <= s < K.shape[0] * page:
            continue
        for h in range(cache.heads):
            want = at.norm_rotate(k[i, h * D:(h + 1) * D], _np(c["wk"]), EPS, turn, inter)
            near(K[s // page, h, s % page], want)
            near(V[s // page, h, s % page], v[i, h * D:(h + 1) * D])
            wantK[s // page, h, s % page] = K[s // page, h, s % page]
            wantV[s // page, h, s % page] = V[s // page, h, s % page]
    np.testing.assert_array_equal(K, wantK)
    np.testing.assert_array_equal(V, wantV)


def _run(c, inter, **kw):
    return _prq().prq_qk_norm_rope(c["q"], c["k"], c["v"], c["pos"], c["table"], c["cache"], c["slots"],
                                   q_weight=c["wq"], k_weight=c["wk"], eps=EPS, interleaved=inter, **kw)


F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("M,Hq,Hk,D,rot,page,dtype,norm,inter", [
    (1, 32, 8, 128, 128, 64, F32, True, False), (1, 1, 1, 64, 64, 16, F32, True, True),
    (5, 3, 1, 64, 32, 16, BF16, True, True), (7, 8, 2, 128, 64, 32, BF16, False, False),
    (17, 6, 3, 256, 256, 16, F32, True, False), (9, 4, 4, 256, 8, 16, BF16, True, True),
    (33, 12, 12, 64, 8, 128, F32, True, False), (40, 8, 1, 128, 120, 16, F32, True, False),
    (3, 5, 5, 128, 24, 16, F32, False, True), (6, 4, 2, 128, 0, 16, F32, True, False),
    (6, 4, 2, 64, 0, 16, BF16, False, True), (700, 2, 1, 64, 64, 64, F32, True, False),
    (1300, 7, 1, 128, 128, 64, F32, True, False), (600, 30, 15, 64, 16, 16, BF16, True, True),
    (260, 33, 11, 256, 64, 16, F32, True, False)])
def test_matches_oracle(M, Hq, Hk, D, rot, page, dtype, norm, inter):
    say("norm rope", M, Hq, Hk, D, rot, dtype, norm, inter)
    c = _make(M, Hq, Hk, D, rot, page, dtype, norm, seed=M + D)
    K0, V0 = c["cache"].K.clone(), c["cache"].V.clone()
    got = _run(c, inter, out=torch.full((M, Hq, D), float("nan"), dtype=BF16, device="cuda"))
    _check(c, got, K0, V0, D, inter)


def test_one_weight_and_float32_weights():
    c = _make(4, 4, 2, 64, 64, 16, F32, True, 3, w_dtype=F32)
    c["wq"] = None
    K0, V0 = c["cache"].K.clone(), c["cache"].V.clone()
    _check(c, _run(c, False), K0, V0, 64, False)


def test_rows_of_a_merged_projection_and_of_an_interleaved_pool():
    """q, k, v as slices of one [M, (Hq + 2 Hk) D] projection; K and V pages in one allocation."""
    Hq, Hk, D, M = 8, 2, 128, 21
    c = _make(M, Hq, Hk, D, 128, 16, F32, True, 4)
    whole = torch.cat([c["q"], c["k"], c["v"]], 1)
    c["q"], c["k"], c["v"] = whole[:, :Hq * D], whole[:, Hq * D:(Hq + Hk) * D], whole[:, (Hq + Hk) * D:]
    pool = torch.randn(5, 2, Hk, 16, D, device="cuda").bfloat16()
    c["cache"] = _prq().PagedKV(pool[:, 0], pool[:, 1])
    K0, V0 = pool[:, 0].clone(), pool[:, 1].clone()
    _check(c, _run(c, False), K0, V0, D, False)


def test_padding_rows_and_slots_outside_the_pool_write_nothing():
    c = _make(6, 4, 2, 64, 64, 16, F32, True, 5)
    n = c["cache"].pages * 16
    c["slots"] = torch.tensor([-1, 3, n, n + 5, -(1 << 40), 1 << 40], device="cuda")
    K0, V0 = c["cache"].K.clone(), c["cache"].V.clone()
    _check(c, _run(c, False), K0, V0, 64, False)


def test_positions_outside_the_table_are_nan_in_the_rotated_dims_only():
    c = _make(4, 2, 1, 64, 32, 16, F32, True, 6)
    c["pos"] = torch.tensor([64, -1, 1 << 30, 63], dtype=torch.int32, device="cuda")
    out = _run(c, False).float()
    assert bool(torch.isnan(out[:3, :, :32]).all()) and bool(torch.isfinite(out[:3, :, 32:]).all())
    assert bool(torch.isfinite(out[3]).all())
    s = c["slots"].tolist()
    K = c["cache"].K.float()
    assert bool(torch.isnan(K[s[0] // 16, :, s[0] % 16, :32]).all())
    assert bool(torch.isfinite(c["cache"].V.float()).all())


def test_nan_and_infinity_stay_in_their_head():
    c = _make(3, 4, 2, 128, 128, 16, F32, True, 7)
    want = _run(c, False).clone()
    c["q"][1, 128 + 5], c["q"][2, 300] = float("nan"), float("inf")
    got = _run(c, False)
    assert bool(torch.isnan(got[1, 1]).all())           # the norm spreads it over its own head
    keep = torch.ones(3, 4, dtype=torch.bool, device="cuda")
    keep[1, 1] = keep[2, 2] = False
    assert torch.equal(got[keep], want[keep])


def test_zero_rows_and_zero_heads():
    c = _make(2, 2, 1, 64, 64, 16, F32, True, 8)
    c["q"].zero_()
    assert not _run(c, False).any()                      # 0 / sqrt(0 + eps) = 0
    e = torch.empty(0, 128, device="cuda")
    out = _prq().prq_qk_norm_rope(e, e[:, :64], e[:, :64], c["pos"][:0], c["table"], c["cache"], c["slots"][:0])
    assert out.shape == (0, 2, 64)


def test_slots_past_32_bits():
    """A pool of 2^31 + elements: the last pages lie past every 32-bit element offset."""
    Hk, page, D, M = 8, 16, 128, 3
    pages = (1 << 31) // (Hk * page * D) + 700
    prq = _prq()
    K = torch.empty(pages, Hk, page, D, dtype=BF16, device="cuda")
    V = torch.empty(pages, Hk, page, D, dtype=BF16, device="cuda")
    c = _make(M, 8, Hk, D, 128, page, F32, True, 9)
    small = c["cache"]
    c["slots"] = torch.tensor([0, 17, 35], device="cuda")
    want_q = _run(c, False).clone()
    c["cache"] = prq.PagedKV(K, V)
    first = pages - 4
    c["slots"] = c["slots"] + first * page
    assert torch.equal(_run(c, False), want_q)
    for s in (0, 17, 35):
        assert torch.equal(K[first + s // page, :, s % page], small.K[s // page, :, s % page])
        assert torch.equal(V[first + s // page, :, s % page], small.V[s // page, :, s % page])
