"""prq_block_norm against the float64 oracle: types, widths, norms on either side, gates, strides, in
place, rows without a block or a residual.

Bar: one rounding of each output to its type (half a step: bf16 2^-8, float32 2^-24 of the value) and
the float32 chain behind it.  The chain of r' is at most a square sum of H / 8 <= 2048 additions a
lane and 8 over lanes, the root and quotient and 5 products; a sum of squares has no cancellation, so
its relative error, halved by the root, is below (2048 + 8 + 2) 2^-25 only for adversarial input and
2^-20 with 16 lanes' partial sums of H / 64 = 256 terms; 2^-18 of the magnitudes that are added covers
it and the rest."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import moe                        # noqa: E402
from tests import moe_plans                   # noqa: E402
from tests.gpu_util import say                # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
CHAIN = 2.0 ** -18


def _prq():
    from paper_2609_22106_amd import prq
    return prq


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _make(M, H, y_type, r_type, post, gates, seed, w_type=BF16, index=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")   # noqa: E731
    return dict(y=(3 * rnd(M, H)).to(y_type), r=(2 * rnd(M, H)).to(r_type),
                post=(1 + 0.3 * rnd(H)).to(w_type) if post else None, pre=(1 + 0.3 * rnd(H)).to(w_type),
                gate=rnd(gates, H).to(w_type) if gates else None,
                index=torch.randint(-1, gates + 1, (M,), generator=g, device="cuda", dtype=torch.int32) if index else None)


def _check(c, got, eps=1e-6, offset=0.0, a=1.0, b=1.0, r0=None):
    h, r = got
    y, res = _np(c["y"]), _np(c["r"] if r0 is None else r0)
    want_r, want_h = moe.block_norm(y, res, _np(c["post"]), _np(c["pre"]), _np(c["gate"]), _np(c["index"]), eps, offset,
                                    a, b)
    part, _ = moe.block_norm(y, None, _np(c["post"]), None, _np(c["gate"]), _np(c["index"]), eps, offset, a, b)
    added = np.abs(part) + np.abs(a * res)
    half = 2.0 ** -8 if r.dtype is BF16 else 2.0 ** -24
    assert np.all(np.abs(_np(r) - want_r) <= half * np.abs(want_r) + CHAIN * added)
    if h is not None:
        # h's own chain, and r' moved by its error: h moves with it, and through the row's root
        rms = np.sqrt(np.mean(want_r ** 2, 1, keepdims=True) + eps)
        w = np.abs(offset + _np(c["pre"]))
        moved = CHAIN * added / rms * w + np.abs(want_h) * CHAIN * np.sqrt(np.mean(added ** 2, 1, keepdims=True)) / rms
        assert np.all(np.abs(_np(h) - want_h) <= 2.0 ** -8 * np.abs(want_h) + CHAIN * np.abs(want_h) + moved)


@pytest.mark.parametrize("M,H,y_type,r_type,post,gates,index,w_type", [
    (1, 8, F32, F32, True, 0, False, BF16), (1, 2048, F32, BF16, True, 1, False, BF16), (3, 16, BF16, BF16, False, 3, False, F32),
    (7, 1032, BF16, F32, True, 2, True, BF16), (61, 2560, F32, BF16, True, 5, True, F32), (5, 16384, F32, F32, True, 0, False, F32),
    (4, 12296, BF16, BF16, False, 4, True, BF16), (2050, 2560, F32, F32, True, 3, True, BF16),
    (2049, 1056, BF16, BF16, True, 2049, False, BF16), (2053, 2568, F32, BF16, False, 1, False, BF16),
    (4099, 40, BF16, F32, True, 1, True, BF16), (2301, 256, F32, F32, False, 0, False, F32), (6, 5128, BF16, BF16, True, 0, False, BF16)])
def test_matches_oracle(M, H, y_type, r_type, post, gates, index, w_type):
    say("block norm", M, H, y_type, r_type, post, gates, index)
    c = _make(M, H, y_type, r_type, post, gates, M + H, w_type, index)
    out = torch.full((M, H), float("nan"), dtype=BF16, device="cuda")
    r = torch.full((M, H), float("nan"), dtype=r_type, device="cuda")
    r0 = c["r"].clone()
    got = _prq().prq_block_norm(c["y"], c["r"], c["pre"], post_weight=c["post"], gate=c["gate"], gate_index=c["index"],
                                out=out, residual_out=r, residual_scale=0.75, block_scale=-0.5)
    assert got[0] is out and got[1] is r and torch.equal(c["r"], r0)
    _check(c, got, a=0.75, b=-0.5)


@pytest.mark.parametrize("M,H,y_type,r_type,post,gates", [
    (1024, 520, F32, BF16, True, 1), (1025, 1056, BF16, BF16, True, 7), (1601, 1536, F32, F32, True, 0),
    (1023, 1536, BF16, F32, False, 0), (1027, 1544, F32, F32, True, 3), (3333, 1024, F32, F32, False, 0)])
def test_rows_by_half_a_workgroup(M, H, y_type, r_type, post, gates):
    """1024 rows and more of 513 to 1536 elements, and their neighbours, in place: the last row alone."""
    say("block norm", M, H, y_type, r_type, post, gates)
    c = _make(M, H, y_type, r_type, post, gates, M + H, index=gates > 1)
    r0 = c["r"].clone()
    got = _prq().prq_block_norm(c["y"], c["r"], c["pre"], post_weight=c["post"], gate=c["gate"], gate_index=c["index"])
    assert got[1] is c["r"]
    _check(c, got, r0=r0)


def test_in_place_and_offset_weights():
    c = _make(9, 264, F32, BF16, True, 0, 1)
    r0 = c["r"].clone()
    got = _prq().prq_block_norm(c["y"], c["r"], c["pre"], post_weight=c["post"], weight_offset=1.0, eps=1e-3)
    assert got[1] is c["r"]
    _check(c, got, eps=1e-3, offset=1.0, r0=r0)


@pytest.mark.parametrize("M", [3, 2100])
def test_strided_rows(M):
    """Slices of wider tensors: y of a merged projection, the outputs in padded buffers whose gaps stay."""
    c = _make(M, 128, F32, F32, True, 2, 2, index=True)
    wide = torch.cat([c["y"], c["y"]], 1)
    c["y"] = wide[:, 128:]
    r_buf, h_buf = torch.full((M, 160), 7.0, device="cuda"), torch.full((M, 136), 7.0, dtype=BF16, device="cuda")
    got = _prq().prq_block_norm(c["y"], c["r"], c["pre"], post_weight=c["post"], gate=c["gate"], gate_index=c["index"],
                                out=h_buf[:, :128], residual_out=r_buf[:, :128])
    _check(c, got)
    assert bool((r_buf[:, 128:] == 7).all()) and bool((h_buf[:, 128:] == 7).all())


def test_without_a_block_without_a_residual_and_without_a_next_norm():
    prq = _prq()
    c = _make(5, 512, F32, F32, True, 0, 3)
    r0 = c["r"].clone()
    h, r = prq.prq_block_norm(None, c["r"], c["pre"])               # the first norm of a model
    assert r is c["r"] and torch.equal(r, r0)
    z = dict(c, y=torch.zeros_like(c["y"]), post=None)
    _check(z, (h, r))
    h, r = prq.prq_block_norm(None, c["r"], c["pre"], residual_scale=0.5)
    assert torch.equal(c["r"], 0.5 * r0)
    h, r = prq.prq_block_norm(c["y"], None, c["pre"], post_weight=c["post"])
    assert r is None
    want = prq.prq_block_norm(c["y"], torch.zeros_like(r0), c["pre"], post_weight=c["post"])
    assert torch.equal(h, want[0])
    c["r"] = r0.clone()
    h, r = prq.prq_block_norm(c["y"], c["r"])                        # the last sum of a model
    assert h is None and torch.equal(r, r0 + c["y"])


def test_zero_rows_and_rows_of_zeros():
    prq = _prq()
    e = torch.empty(0, 64, device="cuda")
    h, r = prq.prq_block_norm(e, e.clone(), torch.ones(64, device="cuda"))
    assert h.shape == r.shape == (0, 64)
    z = torch.zeros(3, 64, device="cuda")
    h, r = prq.prq_block_norm(z, z.clone(), torch.ones(64, device="cuda"), post_weight=torch.ones(64, device="cuda"))
    assert not h.any() and not r.any()                               # 0 / sqrt(0 + eps) = 0


@pytest.mark.parametrize("M", [4, 2052])
def test_nan_and_infinity_stay_in_their_row(M):
    prq = _prq()
    c = _make(M, 320, F32, F32, True, 1, 4)
    call = lambda: prq.prq_block_norm(c["y"], c["r"], c["pre"], post_weight=c["post"], gate=c["gate"],       # noqa: E731
                                      residual_out=torch.empty_like(c["r"]))
    want = [t.clone() for t in call()]
    c["y"][1, 7], c["r"][2, 300] = float("nan"), float("inf")
    got = call()
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[1] = keep[2] = False
    for g, w in zip(got, want):
        assert torch.equal(g[keep], w[keep])
    assert bool(torch.isnan(got[0][1]).all()) and bool(torch.isnan(got[1][1]).all())
    assert float(got[1][2, 300]) == float("inf") and not bool(torch.isfinite(got[0][2, 300]))


def test_a_gate_index_outside_the_gate_gates_nothing():
    c = _make(6, 64, BF16, F32, False, 2, 5)
    c["index"] = torch.tensor([-1, 2, 1 << 30, -(1 << 31), 0, 1], dtype=torch.int32, device="cuda")
    got = _prq().prq_block_norm(c["y"], c["r"], c["pre"], gate=c["gate"], gate_index=c["index"],
                                residual_out=torch.empty_like(c["r"]))
    _check(c, got)
    assert torch.equal(got[1][:4], (c["r"] + c["y"].float())[:4])


def test_rows_past_32_bits():
    """2^31 + elements of residual: the last rows lie past every 32-bit element offset."""
    prq = _prq()
    H, M = 16384, (1 << 31) // 16384 + 3
    r = torch.empty(M, H, dtype=BF16, device="cuda")
    h = torch.empty(M, H, dtype=BF16, device="cuda")
    y = torch.empty(M, H, dtype=BF16, device="cuda")
    c = _make(3, H, BF16, BF16, True, 0, 6)
    r[-3:], y[-3:] = c["r"], c["y"]
    prq.prq_block_norm(y, r, c["pre"], post_weight=c["post"], out=h)
    want = prq.prq_block_norm(c["y"], c["r"], c["pre"], post_weight=c["post"])
    assert torch.equal(h[-3:], want[0]) and torch.equal(r[-3:], want[1])


# A lane adds at most 64 squares in 16 sums of 4; a wave's lanes meet in 6 steps and the waves in 2, so a sum of
# squares is off by at most 1 + 2 + 16 + 6 + 2 = 27 roundings of it, the root of the mean by half of those and of
# the quotient's and eps's, and its own, 1 / it one more: 17.  u takes 3 more, the gate 1, the scaled sum 3: 24
# roundings of b u at most and 2 of a r.  Without a norm behind the block 4 are left.
STEP = 2.0 ** -24


def _check_rows(rows, c, got, a, b, eps=1e-6):
    """Rows against the oracle, with the roundings that there are."""
    pick = lambda t: None if t is None else _np(t[rows])                      # noqa: E731
    post, pre, gate = _np(c["post"]), _np(c["pre"]), _np(c["gate"])
    index = None if c["index"] is None else pick(c["index"])
    want_r, want_h = moe.block_norm(pick(c["y"]), pick(c["r"]), post, pre, gate, index, eps, 0.0, a, b)
    part, _ = moe.block_norm(pick(c["y"]), None, post, None, gate, index, eps, 0.0, a, b)
    far = STEP * ((24 if post is not None else 4) * np.abs(part) + 2 * np.abs(a * pick(c["r"])))
    far = (1 + 2.0 ** -7) * far                                                # second order, and of what is rounded
    half = 2.0 ** -8 if got[1].dtype is BF16 else STEP
    assert np.all(np.abs(pick(got[1]) - want_r) <= half * np.abs(want_r) + far)
    rms = np.sqrt(np.mean(want_r ** 2, 1, keepdims=True) + eps)
    moved = far / rms * np.abs(pre) + np.abs(want_h) * np.sqrt(np.mean(far ** 2, 1, keepdims=True)) / rms
    assert np.all(np.abs(pick(got[0]) - want_h) <= 2.0 ** -8 * np.abs(want_h) + (1 + 2.0 ** -7) * (moved + 20 * STEP * np.abs(want_h)))


def _form(M, H, y_bf16, r_bf16, post, gates, index):
    say("block norm", M, H, y_bf16, r_bf16, post, gates, index)
    c = _make(M, H, BF16 if y_bf16 else F32, BF16 if r_bf16 else F32, post, gates, M + H, index=index)
    out = torch.full((M, H), float("nan"), dtype=BF16, device="cuda")
    r = torch.full((M, H), float("nan"), dtype=c["r"].dtype, device="cuda")
    return c, _prq().prq_block_norm(c["y"], c["r"], c["pre"], post_weight=c["post"], gate=c["gate"], gate_index=c["index"],
                                    out=out, residual_out=r, residual_scale=0.75, block_scale=-0.5)


@pytest.mark.parametrize("M,H,y_bf16,r_bf16,plan", moe_plans.NORM_FORMS)
@pytest.mark.parametrize("post,gates,index", [(True, 3, True), (False, 1, False)])
def test_every_form(M, H, y_bf16, r_bf16, plan, post, gates, index):
    c, got = _form(M, H, y_bf16, r_bf16, post, gates, index)
    _check_rows(slice(None), c, got, 0.75, -0.5)


@pytest.mark.parametrize("M,H,y_bf16,r_bf16,plan", moe_plans.NORM_PAST_THE_CACHE)
@pytest.mark.parametrize("post", [True, False])
def test_past_the_last_cache(M, H, y_bf16, r_bf16, plan, post):
    c, got = _form(M, H, y_bf16, r_bf16, post, 2, True)
    g = torch.Generator().manual_seed(M)
    rows = torch.unique(torch.cat([torch.randint(0, M, (30,), generator=g), torch.tensor([0, 1, M - 2, M - 1])])).cuda()
    _check_rows(rows, c, got, 0.75, -0.5)
    assert not bool(torch.isnan(got[0]).any()) and not bool(torch.isnan(got[1]).any())      # all rows are written
