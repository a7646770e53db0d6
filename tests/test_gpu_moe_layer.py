"""prq_moe_layer against the float64 oracle.

Bar, per output: its rounding (bf16, 2^-8 of the value); the roundings of w h to bf16, each at most
2^-8 of its value and independent of each other, uniform within their step: a standard deviation of
at most 2^-8 / sqrt(3) of the root of the squares' sum, six of which cover the outputs checked here;
and float32 sums: 2^-24 times the number of terms times the magnitudes that are added, in the first
product (whose errors reach y through h) and the second, with 8 more for SiLU and the products."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import moe                                  # noqa: E402
from paper_2609_22106_amd import inputs                 # noqa: E402
from tests import moe_plans                             # noqa: E402
from tests.gpu_util import dev, say                     # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _prq():
    from paper_2609_22106_amd import prq
    return prq


def _np(t):
    return t.double().cpu().numpy()


class Layer:
    def __init__(self, E, H, I, tail, N, seed, scale_lo=118, scale_hi=124):
        rng = np.random.default_rng(seed)
        up, down = (inputs.random_mxfp4(rng, (E, n), K, scale_lo, scale_hi) for n, K in ((2 * I, H), (N, I + tail)))
        self.up, self.down = moe.dequantized(*up), moe.dequantized(*down)
        self.gate_up, self.down_w = (_prq().prq_pack_weight(dev(q), dev(s)) for q, s in (up, down))
        self.E, self.H, self.I, self.tail, self.N = E, H, I, tail, N

    def __call__(self, x, ids, weights, **kw):
        return _prq().prq_moe_layer(x, ids, weights, self.gate_up, self.down_w, k_tail=self.tail, **kw)

    def check(self, got, x, ids, weights):
        y, size, root, reach = moe.layer(_np(x), ids.cpu().numpy(), _np(weights), self.up, self.down, self.tail)
        k = ids.shape[1]
        tol = (2.0 ** -8 * np.abs(y) + 6 * 2.0 ** -8 / np.sqrt(3) * root
               + 2.0 ** -24 * ((self.H + 8) * reach + (k * (self.I + self.tail) + 8) * size))
        err = np.abs(_np(got) - y)
        assert np.all(err <= tol), (float(np.max(err / np.maximum(tol, 1e-300))), np.argwhere(err > tol)[:4])


def _routed(M, E, k, seed, H):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.argsort(torch.rand(M, E, generator=g, device="cuda"), dim=1)[:, :k].to(torch.int32).contiguous()
    return ((torch.randn(M, H, generator=g, device="cuda") / 4).to(BF16), ids,
            torch.rand(M, k, generator=g, device="cuda") + 0.1)


@pytest.mark.parametrize("M,E,k,H,I,tail,N", [
    (1, 1, 1, 32, 32, 0, 16), (1, 128, 8, 2048, 96, 32, 64), (2, 3, 2, 160, 64, 64, 48), (7, 16, 2, 1056, 352, 32, 1056),
    (16, 4, 3, 128, 128, 0, 256), (17, 9, 5, 384, 160, 32, 112), (31, 2, 1, 96, 32, 0, 32), (33, 64, 6, 256, 192, 64, 320),
    (48, 8, 8, 64, 32, 32, 16), (64, 128, 8, 512, 96, 32, 128), (64, 1, 1, 288, 64, 0, 64), (64, 5, 4, 2080, 416, 96, 80),
    (64, 300, 32, 64, 32, 0, 32), (3, 4096, 4, 64, 32, 0, 16), (40, 40, 20, 1120, 32, 0, 48), (64, 16, 2, 128, 1408, 0, 1040)])
def test_matches_oracle(M, E, k, H, I, tail, N):
    say("experts", M, E, k, H, I, tail, N)
    layer = Layer(E, H, I, tail, N, seed=M + E)
    x, ids, w = _routed(M, E, k, M + H, H)
    out = torch.full((M, N), float("nan"), dtype=BF16, device="cuda")
    got = layer(x, ids, w, out=out)
    assert got is out
    layer.check(got, x, ids, w)


@pytest.mark.parametrize("M,E,k,H,I,tail,N", [
    (20, 64, 6, 160, 352, 32, 48), (50, 64, 6, 2144, 288, 0, 32), (64, 60, 9, 96, 448, 64, 80),      # two waves a tile
    (12, 128, 9, 288, 480, 32, 32), (40, 128, 8, 1184, 416, 0, 48), (64, 130, 8, 64, 544, 96, 16)])   # one
def test_many_tiles(M, E, k, H, I, tail, N):
    """More intermediate features of all experts: fewer waves of the first launch share a tile."""
    say("experts", M, E, k, H, I, tail, N)
    layer = Layer(E, H, I, tail, N, seed=M + E + H)
    x, ids, w = _routed(M, E, k, M + 1, H)
    layer.check(layer(x, ids, w), x, ids, w)


@pytest.mark.parametrize("M", [1, 20, 64])
def test_ids_that_name_nothing_rows_without_experts_and_an_expert_named_twice(M):
    layer = Layer(6, 128, 64, 32, 96, seed=3)
    x, ids, w = _routed(M, 6, 4, 5, 128)
    full = layer(x, ids, w).clone()
    ids[0, 1], ids[0, 2] = -1, 6
    ids[0, 3] = ids[0, 0]
    if M > 8:
        ids[3] = torch.tensor([1 << 30, -(1 << 31), 7, -5], dtype=torch.int32)
        ids[8] = 2
    got = layer(x, ids, w, out=torch.full((M, 96), float("nan"), dtype=BF16, device="cuda"))
    layer.check(got, x, ids, w)
    if M > 8:
        assert not got[3].any()
        keep = [i for i in range(M) if i not in (0, 3, 8)]
        layer.check(full, *(_routed(M, 6, 4, 5, 128)))
        # sums over other numbers of experts may be split elsewhere: equal to rounding, which check has shown
        assert torch.allclose(got[keep].float(), full[keep].float(), rtol=2 ** -6, atol=1e-3)
    ids.fill_(-1)
    assert not layer(x, ids, w, out=torch.full((M, 96), float("nan"), dtype=BF16, device="cuda")).any()


def test_all_tokens_at_one_expert():
    layer = Layer(32, 256, 96, 32, 64, seed=4)
    x, ids, w = _routed(64, 32, 2, 6, 256)
    ids[:, 0], ids[:, 1] = 31, -1
    layer.check(layer(x, ids, w), x, ids, w)


def test_nan_and_infinity_stay_in_their_token():
    layer = Layer(8, 96, 64, 0, 48, seed=5)
    x, ids, w = _routed(40, 8, 3, 7, 96)
    want = layer(x, ids, w).clone()
    x[3, 5], x[17, 95], w[20, 1] = float("nan"), float("inf"), float("nan")
    got = layer(x, ids, w)
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[[3, 17, 20]] = False
    assert torch.equal(got[keep], want[keep])
    assert bool(torch.isnan(got[3]).all()) and bool(torch.isnan(got[20]).all()) and not bool(torch.isfinite(got[17]).all())


@pytest.mark.parametrize("lo,hi", [(0, 0), (1, 20), (60, 70), (127, 127), (150, 180), (230, 242)])
def test_scale_codes_far_from_one(lo, hi):
    """Each E8M0 code as the power of two that it is: one weight of ones in either product."""
    prq = _prq()
    H = I = 32
    N = 16
    for code in range(lo, hi + 1):
        up_q, up_s = np.zeros((1, 2 * I, H // 2), np.uint8), np.full((1, 2 * I, 1), 127, np.uint8)
        for r in range(2 * I):                                       # row r: 1 at column r % 32
            up_q[0, r, (r % 32) // 2] = 2 << (4 * (r % 2))
        up_s[0, I:] = code                                           # the up-projection's rows: 2^(code - 127)
        down_q, down_s = np.zeros((1, N, I // 2), np.uint8), np.full((1, N, 1), 127, np.uint8)
        for r in range(N):
            down_q[0, r, r // 2] = 2 << (4 * (r % 2))
        x = torch.full((1, H), 64.0, dtype=BF16, device="cuda")       # SiLU(64) is 64 in bf16
        ids, w = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, 1, device="cuda")
        pack = lambda q, s: prq.prq_pack_weight(dev(q), dev(s))       # noqa: E731
        got = prq.prq_moe_layer(x, ids, w, pack(up_q, up_s), pack(down_q, down_s))
        assert bool((got.double() == 4096.0 * 2.0 ** (code - 127)).all()), code
        down_s[:] = code
        up_s[:] = 127
        got = prq.prq_moe_layer(x, ids, w, pack(up_q, up_s), pack(down_q, down_s))
        assert bool((got.double() == 4096.0 * 2.0 ** (code - 127)).all()), code


def test_strides_and_a_shared_workspace():
    """Rows of wider tensors; one workspace for layers of several sizes in turn, left ready by each."""
    prq = _prq()
    a, b = Layer(64, 256, 224, 32, 512, seed=8), Layer(3, 64, 32, 0, 16, seed=9)
    ws = torch.zeros(8 << 20, dtype=torch.uint8, device="cuda")
    for M, layer in ((64, a), (1, b), (33, a), (64, b), (64, a)):
        x, ids, w = _routed(M, layer.E, 3, M, layer.H)
        wide = torch.full((M, layer.H + 8), float("nan"), dtype=BF16, device="cuda")
        wide[:, :layer.H] = x
        buf = torch.full((M + 1, layer.N + 24), 7.0, dtype=BF16, device="cuda")
        got = layer(wide[:, :layer.H], ids, w, out=buf[:M, :layer.N], workspace=ws)
        layer.check(got, x, ids, w)
        assert bool((buf[:, layer.N:] == 7).all()) and bool((buf[M:] == 7).all())
        assert not ws[:16384].any()
        assert torch.equal(layer(x, ids, w, workspace=ws), got)      # the same bits again
        ws[16384:] = 255                                             # (NaN) nothing is read that was not written
    assert prq.prq_moe_layer_workspace_bytes(64, 3, 64, 256, 224, 32, 512) <= ws.numel()


@pytest.mark.parametrize("M,E,k,H,I,tail,N", [(2, 1, 1, 65536, 32, 0, 16), (64, 2, 2, 32, 32768, 32, 16),
                                              (35, 2, 1, 32, 32, 0, 65536)])
def test_largest_widths(M, E, k, H, I, tail, N):
    say("experts", M, E, k, H, I, tail, N)
    layer = Layer(E, H, I, tail, N, seed=M + E)
    x, ids, w = _routed(M, E, k, M, H)
    layer.check(layer(x, ids, w), x, ids, w)


def test_rows_past_32_bits():
    """Rows of x and out more than 2^31 elements apart, first to last."""
    M, ld = 20, 1 << 27
    layer = Layer(8, 64, 32, 0, 48, seed=4)
    x, ids, w = _routed(M, 8, 2, 6, 64)
    far = torch.empty((M - 1) * ld + 16384, dtype=BF16, device="cuda")
    rows, out = far.as_strided((M, 64), (ld, 1)), far[8192:].as_strided((M, 48), (ld, 1))
    rows.copy_(x)
    layer(rows, ids, w, out=out)
    layer.check(out, x, ids, w)
    assert torch.equal(rows, x)


def test_zero_tokens():
    layer = Layer(2, 32, 32, 0, 16, seed=1)
    x, ids, w = (torch.empty(0, 32, dtype=BF16, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"),
                 torch.empty(0, 2, device="cuda"))
    assert layer(x, ids, w).shape == (0, 16)


def test_tail_of_a_prepared_weight():
    """Gate and up rows from prq_expand_producer (its first I), the down-projection from prq_prepare: the
    layer computes the augmented product on unquantized activations."""
    from oracle import prquant as pq
    prq = _prq()
    rng = np.random.default_rng(12)
    H, I, N, tail = 128, 96, 64, 32
    bits = lambda *s: inputs.f32_to_bf16_bits((0.1 * rng.standard_normal(s)).astype(np.float32))   # noqa: E731
    down, xcal, up, gate = bits(N, I), bits(16, I), bits(I, H), bits(I, H)
    art = prq.prq_prepare(down, xcal, 0.5, tail)
    up_aug, gate_aug = prq.prq_expand_producer(up, gate, art["inv_scale"], art["perm"], tail)
    both = np.concatenate([gate_aug[:I], up_aug[:I]])
    first = prq.prq_prepare(both, both[:1], 0.0, 0, "none")
    layer = object.__new__(Layer)
    layer.E, layer.H, layer.I, layer.tail, layer.N = 1, H, I, tail, N
    layer.up = moe.dequantized(first["Wq"], first["Wsc"])[None]
    layer.down = moe.dequantized(art["Wq"], art["Wsc"])[None]
    layer.gate_up = prq.prq_pack_weight(dev(first["Wq"]), dev(first["Wsc"]))
    layer.down_w = prq.prq_pack_weight(dev(art["Wq"]), dev(art["Wsc"]))
    x, ids, w = _routed(5, 1, 1, 13, H)
    layer.check(layer(x, ids, w), x, ids, w)
    np.testing.assert_array_equal(first["perm"], np.arange(H))       # own order
    assert np.all(first["scale"] == 1)
    assert pq.prepare(both, both[:1], 0.0, 0, "none")["Wq"].shape == first["Wq"].shape


def _check_between(layer, got, x, ids, weights):
    """Without the roundings to 8 bits of the bar above: w h between the launches is off by less than 2^-15 of
    it, and is summed as two operands.  An output's own rounding, and 2^-7 of the errors for their products."""
    y, size, _, reach = moe.layer(_np(x), ids.cpu().numpy(), _np(weights), layer.up, layer.down, layer.tail)
    terms = 2 * ids.shape[1] * (layer.I + layer.tail)
    far = 2.0 ** -15 * size + 2.0 ** -24 * ((layer.H + 8) * reach + (terms + 16) * size)
    tol = 2.0 ** -8 * np.abs(y) + (1 + 2.0 ** -7) * far
    err = np.abs(_np(got) - y)
    assert np.all(err <= tol), (float(np.max(err / np.maximum(tol, 1e-300))), np.mean(err > tol))


@pytest.mark.parametrize("M,E,k,H,I,tail,N", [
    (1, 1, 1, 32, 32, 0, 64), (64, 4, 1, 32, 32, 32, 64), (40, 3, 2, 64, 64, 32, 80), (5, 128, 4, 96, 32, 0, 256),
    (64, 16, 2, 32, 96, 96, 48), (17, 1, 1, 160, 256, 64, 32)])
def test_little_is_lost_between_the_launches(M, E, k, H, I, tail, N):
    say("experts", M, E, k, H, I, tail, N)
    layer = Layer(E, H, I, tail, N, seed=M + N)
    x, ids, w = _routed(M, E, k, M + H, H)
    _check_between(layer, layer(x, ids, w), x, ids, w)


def _one_feature(up_code, down_code, weight):
    """One token, H = I = 32, N = 16: SiLU(64) * (64 2^(up_code - 127)) * weight as feature 0, and that times
    2^(down_code - 127) as output 0; all else is 0."""
    prq = _prq()
    up_q, up_s = np.zeros((1, 64, 16), np.uint8), np.full((1, 64, 1), 127, np.uint8)
    up_q[0, 0, 0] = up_q[0, 32, 0] = 2                               # a weight of 1 in column 0
    up_s[0, 32] = up_code
    down_q, down_s = np.zeros((1, 16, 16), np.uint8), np.full((1, 16, 1), 127, np.uint8)
    down_q[0, 0, 0], down_s[0, 0] = 2, down_code
    x = torch.zeros(1, 32, dtype=BF16, device="cuda")
    x[0, 0] = 64
    ids, w = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.full((1, 1), weight, device="cuda")
    return prq.prq_moe_layer(x, ids, w, prq.prq_pack_weight(dev(up_q), dev(up_s)), prq.prq_pack_weight(dev(down_q), dev(down_s)))[0]


def test_the_largest_values_between_the_launches():
    """The largest float32 stays finite, an infinity infinite."""
    below_two = float(np.nextafter(np.float32(2), np.float32(0)))
    assert float(_one_feature(242, 125, below_two)[0]) == 2.0 ** 126       # 2^127 of those, a quarter of it
    assert float(_one_feature(243, 125, 1.0)[0]) == float("inf")
    assert float(_one_feature(243, 125, -1.0)[0]) == -float("inf")


def _check_some(layer, got, x, ids, w, seed):
    """Twelve rows (the oracle takes a row at a time); all are written."""
    g = torch.Generator().manual_seed(seed)
    rows = torch.unique(torch.cat([torch.randint(0, len(x), (10,), generator=g), torch.tensor([0, len(x) - 1])])).cuda()
    layer.check(got[rows], x[rows], ids[rows], w[rows])
    assert not bool(torch.isnan(got).any())


@pytest.mark.parametrize("M,E,k,H,I,tail,N,plan", moe_plans.LAYER_FORMS + moe_plans.LAYER_WINDOWS)
def test_every_form(M, E, k, H, I, tail, N, plan):
    """As many experts as tokens ask for, then one of them asked for by all, with a workspace of NaN."""
    say("experts", M, E, k, H, I, tail, N)
    layer = Layer(E, H, I, tail, N, seed=M + E + H)
    x, ids, w = _routed(M, E, k, M + N, H)
    ws = torch.zeros(_prq().prq_moe_layer_workspace_bytes(M, k, E, H, I, tail, N), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        ws[16384:] = 255
        out = torch.full((M, N), float("nan"), dtype=BF16, device="cuda")
        layer(x, ids, w, out=out, workspace=ws)
        _check_some(layer, out, x, ids, w, M)
        assert not ws[:16384].any()
        ids[:, 0] = E // 2


@pytest.mark.parametrize("M,E,k,H,I,tail,N", [(64, 64, 32, 32, 32, 32, 48), (64, 1024, 32, 64, 32, 0, 48), (50, 600, 20, 64, 64, 32, 64)])
def test_an_expert_named_by_every_choice(M, E, k, H, I, tail, N):
    """Room for as many tokens as choices, most of it empty: behind an expert of lower number and before others."""
    layer = Layer(E, H, I, tail, N, seed=M + E)
    x, ids, w = _routed(M, E, k, M + H, H)
    ids[:] = E // 2
    _check_some(layer, layer(x, ids, w, out=torch.full((M, N), float("nan"), dtype=BF16, device="cuda")), x, ids, w, 1)
    ids[::3, 1], ids[1::5, 2], ids[:, k - 1] = 3, E - 1, -1
    _check_some(layer, layer(x, ids, w, out=torch.full((M, N), float("nan"), dtype=BF16, device="cuda")), x, ids, w, 2)


@pytest.mark.parametrize("code", [0, 1, 127, 242, 243, 250, 251, 252, 253, 254])
def test_every_weight_of_a_scale_code(code):
    """In either product a weight is its value times the power of two; of 2^128 and more, which codes of 253 and
    254 have and float32 has not, it is infinite.  An output that meets one is not finite: infinity times the
    part 0 of a w h that fits 8 bits, as here, is NaN."""
    prq = _prq()
    values = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])
    small = 2.0 ** -100 if code > 127 else 2.0 ** 60                  # with which 64 times it stays within bf16
    want = values * 2.0 ** (code - 127)
    finite = np.abs(want) < 2.0 ** 128
    want = want * 64 * small
    pack = lambda q, s: prq.prq_pack_weight(dev(q), dev(s))           # noqa: E731
    x = torch.zeros(1, 32, dtype=BF16, device="cuda")
    x[0, 0], x[0, 1] = 64, small                                      # gate and up columns
    ids, w = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, 1, device="cuda")

    def run(up_row, up_code, down_q, down_code):
        up_q, up_s = np.zeros((1, 64, 16), np.uint8), np.full((1, 64, 1), 127, np.uint8)
        up_q[0, 0, 0] = 2                                             # SiLU(64), feature 0
        up_q[0, 32, 0], up_s[0, 32] = up_row << 4, up_code
        return prq.prq_moe_layer(x, ids, w, pack(up_q, up_s), pack(down_q, np.full((1, 16, 1), down_code, np.uint8)))[0]

    ones, codes = np.zeros((1, 16, 16), np.uint8), np.zeros((1, 16, 16), np.uint8)
    ones[0, :, 0], codes[0, :, 0] = 2, np.arange(16)                  # column 0
    got = _np(run(2, 127, codes, code))
    assert np.array_equal(got[finite], want[finite]) and not np.isfinite(got[~finite]).any()
    for v in range(16):
        got = _np(run(v, code, ones, 127))
        assert (got == want[v]).all() if finite[v] else not np.isfinite(got).any()
