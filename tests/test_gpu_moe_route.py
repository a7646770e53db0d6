"""prq_moe_route against the float64 oracle.

Logits whose sums are exact in float32 (x and W on a grid of few bits) make the choice exact too: ids
are compared for equality, ties among them.  Weights: expf (2^-23) and the sum of its values, two and six
roundings of the chosen, ten of all, a quotient and a product: below 2^-20 of the value.  Before that the
logit's distance d to the largest one is rounded to float32, which is d 2^-24 of the exponent and so
of the weight (d is below 8 for the logits on the grid; logits of deviation 45 reach 150, and 150 * 2^-24
alone is 9 * 2^-20); a weight below float32's normal numbers may be anything down to 0, 2^-126.  The
sigmoid's are float64 rounded once (2^-24, with 2^-40 for its own chain).  Logits of other inputs: sums of H
products in float32, 2^-24 H of the magnitudes that are added."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import moe                        # noqa: E402
from tests import moe_plans                   # noqa: E402
from tests.gpu_util import say                # noqa: E402

pytestmark = pytest.mark.gpu


def _prq():
    from paper_2609_22106_amd import prq
    return prq


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _grid(M, E, H, seed):
    """Products are multiples of 2^-13 and sums stay below 2^11: 24 bits hold them in any order."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.round(torch.randn(M, H, generator=g, device="cuda") * 16) / 16).clamp(-7, 7)
    w = torch.round(torch.randn(E, H, generator=g, device="cuda") * (512 / H ** 0.5)).clamp(-255, 255) / 512
    bias = 0.1 * torch.randn(E, generator=g, device="cuda")
    assert float((x.abs() @ w.abs().t()).max()) < 2 ** 11 if M else True
    return x.bfloat16(), w.bfloat16(), bias


def _check(got, logits, k, sigmoid=False, bias=None, renormalize=True, scale=1.0):
    ids, weights = got
    want_ids, want = moe.route(logits, k, sigmoid, _np(bias), renormalize, scale)
    np.testing.assert_array_equal(ids.cpu().numpy(), want_ids)
    tol = 2.0 ** -23
    if not sigmoid:
        chosen = np.take_along_axis(logits, want_ids, 1)
        tol = 2.0 ** -20 + 2.0 ** -24 * (chosen[:, :1] - chosen)
    assert np.all(np.abs(_np(weights) - want) <= tol * np.abs(want) + 2.0 ** -126)


SIZES = [(1, 128, 8, 2048), (1, 1, 1, 8), (3, 5, 5, 40), (17, 16, 2, 1056), (16, 17, 3, 136), (64, 64, 6, 2560),
         (33, 1024, 32, 256), (1000, 250, 8, 512), (1025, 128, 8, 256), (1100, 16, 4, 1056), (1030, 32, 32, 64),
         (1027, 40, 1, 328), (1033, 1000, 10, 128), (1029, 512, 8, 64), (4100, 128, 8, 128), (2048, 60, 4, 24)]


@pytest.mark.parametrize("M,E,k,H", SIZES)
@pytest.mark.parametrize("sigmoid,renormalize", [(False, True), (False, False), (True, True), (True, False)])
def test_matches_oracle(M, E, k, H, sigmoid, renormalize):
    say("route", M, E, k, H, sigmoid, renormalize)
    x, w, bias = _grid(M, E, H, M + E + H)
    logits = torch.full((M, E), float("nan"), device="cuda")
    got = _prq().prq_moe_route(x, w, k, scoring="sigmoid" if sigmoid else "softmax", bias=bias if sigmoid else None,
                               renormalize=renormalize, scale=2.5, logits=logits)
    want = _np(x) @ _np(w).T
    np.testing.assert_array_equal(_np(logits), want)
    _check(got, want, k, sigmoid, bias if sigmoid else None, renormalize, 2.5)


@pytest.mark.parametrize("M,E,k,H", [(2, 257, 8, 64), (9, 300, 31, 64), (40, 512, 8, 72), (1300, 300, 32, 16),
                                     (1150, 257, 3, 136), (8200, 520, 8, 8), (4096, 512, 2, 8), (4099, 500, 8, 24),
                                     (5470, 300, 4, 16)])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_more_experts_than_a_group(M, E, k, H, sigmoid):
    """Past 256 experts a token has 32 keys a lane, past 512 a wave; past 8192 tokens of those, two launches."""
    say("route", M, E, k, H, sigmoid)
    x, w, bias = _grid(M, E, H, M + E + H)
    got = _prq().prq_moe_route(x, w, k, scoring="sigmoid" if sigmoid else "softmax", bias=bias if sigmoid else None,
                               renormalize=False)
    _check(got, _np(x) @ _np(w).T, k, sigmoid, bias if sigmoid else None, False)


@pytest.mark.parametrize("M", [5, 1200])
def test_sums_of_any_values(M):
    g = torch.Generator(device="cuda").manual_seed(M)
    x, w = torch.randn(M, 2048, generator=g, device="cuda").bfloat16(), torch.randn(128, 2048, generator=g, device="cuda").bfloat16()
    logits = torch.empty(M, 128, device="cuda")
    got = _prq().prq_moe_route(x, w, 8, logits=logits)
    far = 2.0 ** -24 * 2048 * (np.abs(_np(x)) @ np.abs(_np(w)).T)
    assert np.all(np.abs(_np(logits) - _np(x) @ _np(w).T) <= far)
    _check(got, _np(logits), 8)                                     # the choice from what the sums came to


@pytest.mark.parametrize("M", [4, 1400])
def test_ties_go_to_the_lowest_index(M):
    x = torch.zeros(M, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.randn(130, 64, device="cuda").bfloat16()
    for kw in (dict(), dict(scoring="sigmoid")):
        ids, weights = _prq().prq_moe_route(x, w, 7, **kw)
        assert bool((ids == torch.arange(7, device="cuda")).all()) and bool((weights == weights[0, 0]).all())
    # a logit of -0 is 0
    x[:, 0] = 1
    w.zero_()
    w[::2, 0] = -0.0
    assert bool((_prq().prq_moe_route(x, w, 7)[0] == torch.arange(7, device="cuda")).all())
    # scores that are 1 in 32 bits differ in 64
    w[:, 0] = 20 + torch.arange(130, device="cuda") % 64 / 8
    ids, _ = _prq().prq_moe_route(x, w, 4, scoring="sigmoid")
    assert ids[0].tolist() == [63, 127, 62, 126]


@pytest.mark.parametrize("M", [6, 1300])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_nan_and_infinite_logits(M, sigmoid):
    """NaN behind everything, infinities in their place; other rows are as they were."""
    x = torch.zeros(M, 8, dtype=torch.bfloat16, device="cuda")
    x[:, 0] = 1
    w = torch.zeros(70, 8, dtype=torch.bfloat16, device="cuda")
    w[:, 0] = torch.arange(70, device="cuda") / 8
    run = lambda **kw: _prq().prq_moe_route(x, w, 5, scoring="sigmoid" if sigmoid else "softmax", **kw)   # noqa: E731
    want = [t.clone() for t in run()]
    x[2, 1] = float("nan")
    x[3, 1] = 1                                  # row 3 alone meets these
    w[69, 1], w[3, 1], w[68, 1] = float("nan"), float("inf"), -float("inf")
    # 0 * inf and 0 * nan are NaN for the other rows: give them their own column
    ids, weights = run()
    assert ids[2].tolist() == [0, 1, 2, 3, 4]    # all NaN
    assert bool(torch.isnan(weights[2]).all())
    assert ids[3].tolist() == [3, 67, 66, 65, 64]
    if sigmoid:
        assert bool(torch.isfinite(weights[3]).all())
    # experts 3, 68 and 69 are NaN for everybody else
    assert ids[0].tolist() == [67, 66, 65, 64, 63] and torch.equal(ids[0], ids[-1])
    w[:, 1] = 0
    x[2, 1] = 0
    for g, t in zip(run(), want):
        assert torch.equal(g, t)


@pytest.mark.parametrize("M", [20, 1280])
def test_strides_and_a_shared_workspace(M):
    """Rows of wider tensors; one workspace for calls of several sizes in turn, left ready by each."""
    prq = _prq()
    x, w, _ = _grid(M, 96, 128, 11)
    wide, w_wide = torch.full((M, 200), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.cat([w, w], 1)
    wide[:, :128] = x
    ws = torch.zeros(4 << 20, dtype=torch.uint8, device="cuda")
    logits = torch.full((M, 100), 7.0, device="cuda")
    ids = torch.full((M + 1, 4), -7, dtype=torch.int32, device="cuda")
    for m in (M, 1, M, 3):
        got = prq.prq_moe_route(wide[:m, :128], w_wide[:, :128], 4, logits=logits[:m, :96], workspace=ws, ids=ids[:m])
        _check(got, _np(x[:m]) @ _np(w).T, 4)
        assert bool((logits[:, 96:] == 7).all()) and bool((ids[M:] == -7).all())
        assert not ws[:16384].any()


@pytest.mark.parametrize("M,ld", [(20, 1 << 27), (1100, 1 << 21)])
def test_rows_past_32_bits(M, ld):
    """Rows of x, and of the logits, more than 2^31 elements apart, first to last."""
    x, w, _ = _grid(M, 40, 64, 7)
    far = torch.empty((M - 1) * ld + 16384, dtype=torch.bfloat16, device="cuda")
    rows = far.as_strided((M, 64), (ld, 1))
    rows.copy_(x)
    logits = far.view(torch.float32)[4096:].as_strided((M, 40), (ld // 2, 1))
    got = _prq().prq_moe_route(rows, w, 4, logits=logits)
    _check(got, _np(x) @ _np(w).T, 4)
    np.testing.assert_array_equal(_np(logits), _np(x) @ _np(w).T)
    assert torch.equal(rows, x)


def test_zero_tokens():
    x, w, _ = _grid(0, 8, 64, 1)
    ids, weights = _prq().prq_moe_route(x, w, 2)
    assert ids.shape == weights.shape == (0, 2)


def _same(got, logits, k, sigmoid=False, bias=None, renormalize=True, scale=1.0):
    """_check, where weights may be NaN: in the same places."""
    ids, weights = got
    with np.errstate(invalid="ignore"):
        want_ids, want = moe.route(logits, k, sigmoid, _np(bias), renormalize, scale)
        np.testing.assert_array_equal(ids.cpu().numpy(), want_ids)
        nan = np.isnan(want)
        np.testing.assert_array_equal(np.isnan(_np(weights)), nan)
        tol = 2.0 ** -23
        if not sigmoid:
            chosen = np.take_along_axis(logits, want_ids, 1)
            tol = 2.0 ** -20 + 2.0 ** -24 * np.where(want > 0, chosen[:, :1] - chosen, 0)
        assert np.all((np.abs(_np(weights) - want) <= tol * np.abs(want) + 2.0 ** -126)[~nan])


@pytest.mark.parametrize("M,E,k,H,plan", moe_plans.ROUTE_FORMS)
@pytest.mark.parametrize("sigmoid,renormalize", [(False, False), (True, True)])
def test_every_form(M, E, k, H, plan, sigmoid, renormalize):
    say("route", M, E, k, H, sigmoid, renormalize)
    x, w, bias = _grid(M, E, H, M + E + H)
    bias = bias if sigmoid else None
    kw = dict(scoring="sigmoid" if sigmoid else "softmax", bias=bias, renormalize=renormalize, scale=0.5)
    logits = torch.full((M, E), float("nan"), device="cuda")
    got = _prq().prq_moe_route(x, w, k, logits=logits, **kw)
    want = _np(x) @ _np(w).T
    np.testing.assert_array_equal(_np(logits), want)
    _check(got, want, k, sigmoid, bias, renormalize, 0.5)
    for again, t in zip(_prq().prq_moe_route(x, w, k, **kw), got):                 # without logits
        assert torch.equal(again, t)


@pytest.mark.parametrize("M,E", moe_plans.ROUTE_KINDS)
def test_ties_of_every_form(M, E):
    x = torch.zeros(M, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.randn(E, 64, device="cuda").bfloat16()
    k = min(E, 9)
    for kw in (dict(), dict(scoring="sigmoid"), dict(scoring="sigmoid", bias=torch.full((E,), 0.25, device="cuda"))):
        ids, weights = _prq().prq_moe_route(x, w, k, **kw)
        assert bool((ids == torch.arange(k, device="cuda")).all()) and bool((weights == weights[0, 0]).all())
    # two values in turn: the experts of the larger one first, each in order
    x[:, 0] = 1
    w.zero_()
    w[1::2, 0] = 1
    want = torch.cat([torch.arange(1, E, 2), torch.arange(0, E, 2)])[:k].cuda()
    assert bool((_prq().prq_moe_route(x, w, k)[0] == want).all())


@pytest.mark.parametrize("M,E", moe_plans.ROUTE_KINDS)
@pytest.mark.parametrize("kw", [dict(renormalize=True), dict(renormalize=False), dict(scoring="sigmoid", renormalize=False)])
def test_nan_and_infinite_logits_of_every_form(M, E, kw):
    """Rows with a logit of +inf, of -inf and of NaN, among the chosen and not, and rows of nothing else; the
    weights too: a softmax over all is NaN wherever a logit is, the chosen alone are not where that is not chosen."""
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.zeros(M, 8, dtype=torch.bfloat16, device="cuda")
    x[:, 0] = 1
    w = torch.zeros(E, 8, dtype=torch.bfloat16, device="cuda")
    w[:, 0] = torch.randperm(E, generator=g, device="cuda") / 32                     # (8 bits at most)
    inf, nan = float("inf"), float("nan")
    at = [m for m in (0, 3, M // 2, M - 1)]
    for m, v in zip(at, (inf, nan, -inf, inf)):
        x[m, 1] = v                                                                # times column 1
    w[0, 1], w[E // 2, 1], w[E - 1, 1] = 1, -1, 0.5                                 # 0 times inf and NaN: NaN for the others
    with np.errstate(invalid="ignore"):
        logits = _np(x) @ _np(w).T
    k, rows = min(E, 5), sorted({*at, *range(1, M, 37)})

    def check():
        got = _prq().prq_moe_route(x, w, k, **kw)
        _same([t[rows] for t in got], logits[rows], k, "scoring" in kw, renormalize=kw["renormalize"])
    check()
    x[:, 1] = 0
    x[at, 2] = 1
    w[E // 3, 2], w[2 * E // 3, 2] = nan, -inf                                      # NaN for every row: 0 times those
    w[:, 1] = 0
    with np.errstate(invalid="ignore"):
        logits = _np(x) @ _np(w).T
    check()


@pytest.mark.parametrize("M,E", moe_plans.ROUTE_KINDS)
def test_strides_and_a_poisoned_workspace_of_every_form(M, E):
    """Rows of wider tensors; one workspace for calls of several sizes in turn, whose scratch holds NaN."""
    prq = _prq()
    k = min(E, 6)
    x, w, _ = _grid(M, E, 136, M + E)
    wide, w_wide = torch.full((M, 200), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.cat([w, w + 1], 1)
    wide[:, 8:144] = x
    ws = torch.zeros(max(prq.prq_moe_route_workspace_bytes(m, E, 136) for m in (1, 3, M)) + 16384, dtype=torch.uint8, device="cuda")
    logits = torch.full((M + 1, E + 4), 7.0, device="cuda")[:, :(E + 3) // 4 * 4]
    ids, weights = torch.full((M + 1, k), -7, dtype=torch.int32, device="cuda"), torch.full((M + 1, k), -7.0, device="cuda")
    for m in (M, 1, M, 3):
        ws[16384:] = 255
        got = prq.prq_moe_route(wide[:m, 8:144], w_wide[:, :136], k, workspace=ws, ids=ids[:m], weights=weights[:m],
                                logits=logits[:m, :E] if E % 4 == 0 else None)
        _check(got, _np(x[:m]) @ _np(w).T, k)
        assert not ws[:16384].any() and bool((logits[M:] == 7).all())
        assert bool((ids[M:] == -7).all()) and bool((weights[M:] == -7).all())


@pytest.mark.parametrize("M,E,ld", [(8200, 16, 1 << 18), (2800, 40, 1 << 20), (1400, 96, 1 << 21), (1029, 250, 1 << 21),
                                    (1000, 300, 1 << 22)])
def test_rows_past_32_bits_of_every_form(M, E, ld):
    """Rows of x, and of the logits, more than 2^31 elements apart, first to last."""
    x, w, _ = _grid(M, E, 64, 7)
    far = torch.empty((M - 1) * ld + 16384, dtype=torch.bfloat16, device="cuda")
    rows = far.as_strided((M, 64), (ld, 1))
    rows.copy_(x)
    logits = far.view(torch.float32)[4096:].as_strided((M, E), (ld // 2, 1))
    got = _prq().prq_moe_route(rows, w, 4, logits=logits)
    want = _np(x) @ _np(w).T
    _check(got, want, 4)
    np.testing.assert_array_equal(_np(logits), want)
    assert torch.equal(rows, x)
