"""prq_lora against the float64 oracle: ranks, ragged segments, segments without an adapter, long K,
strides, in place and not, bad tables.

Bar, per element: float32 sums of bf16 products, n terms, error at most n 2^-24 of the sum of the
terms' magnitudes: (K + 3 rank + 32) 2^-24 of the oracle's magnitude sum (each bf16 term of A x is
exact; 32 for the partial sums and the scale)."""
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


class Case:
    def __init__(self, rows, of, ranks, N, K, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda")    # noqa: E731
        M = sum(rows)
        self.x, self.Y = rnd(M, K).to(BF16), rnd(M, N)
        self.pairs = [((rnd(r, K) / K ** 0.5).to(BF16), rnd(N, r).to(BF16)) for r in ranks]
        self.scales = [0.5 + 0.25 * i for i in range(len(ranks))]
        self.adapters = _prq().prq_lora_adapters(self.pairs, self.scales)
        self.off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.of_host = of
        self.offsets = torch.from_numpy(self.off).cuda()
        self.of = torch.tensor(of, dtype=torch.int32, device="cuda")
        self.K, self.ranks = K, ranks

    def check(self, out, Y=None):
        a = [(A.double().cpu().numpy(), B.double().cpu().numpy(), s)
             for (A, B), s in zip(self.pairs, self.scales)]
        want, size = at.lora(self.x.double().cpu().numpy(), (self.Y if Y is None else Y).double().cpu().numpy(), a,
                             self.off, self.of_host)
        err = np.abs(out.double().cpu().numpy() - want)
        tol = (self.K + 3 * max(self.ranks) + 32) * 2.0 ** -24 * size
        assert np.all(err <= tol), float(np.max(err / np.maximum(tol, 1e-30)))

    def run(self, out=None, **kw):
        if out is None:
            out = torch.full_like(self.Y, float("nan"))
        return _prq().prq_lora(self.x, self.adapters, self.offsets, self.of, self.Y, out=out, **kw)


@pytest.mark.parametrize("rows,of,ranks,N,K", [
    ([1], [0], [8], 16, 8), ([1], [0], [16], 4096, 2560), ([1, 1, 1], [1, -1, 0], [8, 24], 48, 264),
    ([3, 0, 17, 16, 1], [0, 1, 1, 0, -1], [64, 8], 1024, 520), ([15, 33], [2, 0], [5, 128, 40], 320, 1000),
    ([40, 2], [0, 1], [256, 72], 208, 328), ([0, 0, 9], [0, 0, 0], [16], 64, 64), ([100], [0], [32], 2560, 9728),
    ([64, 65, 1, 190], [0, 1, 2, -1], [64, 16, 8], 1936, 5216), ([500], [0], [48], 4096, 256),
    ([70, 90, 200], [1, 0, 1], [128, 136], 512, 96), ([1] * 64, list(range(8)) * 8, [8, 16, 32, 64] * 2, 2560, 2568)])
def test_matches_oracle(rows, of, ranks, N, K):
    say("adapters", rows[:6], ranks, N, K)
    c = Case(rows, of, ranks, N, K, seed=N + K)
    out = c.run()
    c.check(out)
    # in place: the same bits
    Y = c.Y.clone()
    assert _prq().prq_lora(c.x, c.adapters, c.offsets, c.of, Y) is Y
    assert torch.equal(Y, out)


def test_more_segments_than_a_wave():
    rng = np.random.default_rng(1)
    rows = rng.integers(0, 4, 300).tolist()
    c = Case(rows, rng.integers(-1, 3, 300).tolist(), [8, 16, 24], 64, 128)
    c.check(c.run())


def test_strided_rows():
    c = Case([20, 30], [0, 1], [16, 32], 96, 200)
    want = c.run()
    M = 50
    x = torch.zeros(M, 256, dtype=BF16, device="cuda")
    x[:, 24:224] = c.x
    Y = torch.zeros(M, 132, device="cuda")
    Y[:, 4:100] = c.Y
    out = torch.full((M, 200), 7.0, device="cuda")
    c.x, c.Y = x[:, 24:224], Y[:, 4:100]
    got = c.run(out=out[:, 100:196])
    assert torch.equal(got, want)
    assert bool((out[:, :100] == 7).all()) and bool((out[:, 196:] == 7).all())


def test_tables_that_name_what_is_not_there_count_as_no_adapter():
    c = Case([4, 4, 4, 4], [0, 1, 2, 1 << 30], [16, 8], 64, 128)
    c.adapters.rank_offsets = torch.tensor([0, 16, 4000], dtype=torch.int32, device="cuda")   # past A
    c.of_host = [0, -1, -1, -1]
    c.check(c.run())
    for bad in ([0, 12, 24], [-8, 8, 24], [16, 0, 24], [0, 24, 24]):           # unaligned, before A, descending, too large
        c.adapters.rank_offsets = torch.tensor(bad, dtype=torch.int32, device="cuda")
        got = c.run()
        assert bool(torch.isfinite(got).all()) and torch.equal(got[:4], c.Y[:4])


def test_offsets_outside_the_rows_are_clamped_and_uncovered_rows_left_alone():
    c = Case([5, 6], [0, 0], [16], 64, 128)
    want = c.run()
    c.offsets = torch.tensor([0, 5, 400], dtype=torch.int32, device="cuda")
    assert torch.equal(c.run(), want)
    c.offsets = torch.tensor([-3, 5, 5], dtype=torch.int32, device="cuda")
    got = c.run()
    assert torch.equal(got[:5], want[:5]) and bool(torch.isnan(got[5:]).all())


def test_nan_and_infinity_stay_in_their_row():
    c = Case([20], [0], [16], 64, 128)
    want = c.run()
    c.x[3, 7], c.x[9, 0] = float("nan"), float("inf")
    got = c.run()
    assert bool(torch.isnan(got[3]).all()) and not bool(torch.isfinite(got[9]).any())
    rows = [r for r in range(20) if r not in (3, 9)]
    assert torch.equal(got[rows], want[rows])


def test_values_beyond_bf16_of_the_product_keep_float32():
    """A x of 2^12 + 1 (13 bits): a rounding to bf16 would lose the 1."""
    c = Case([1], [0], [8], 16, 64)
    c.x.zero_()
    c.x[0, 0], c.x[0, 1] = 4096, 1
    A, B = torch.zeros(8, 64), torch.zeros(16, 8)
    A[0, :2], B[:, 0] = 1, 1
    c.adapters = _prq().prq_lora_adapters([(A, B)], [1.0])
    c.Y.zero_()
    assert bool((c.run() == 4097).all())


def test_calls_repeat_bit_for_bit_and_need_no_clean_workspace():
    prq = _prq()
    c = Case([3, 2], [0, 1], [64, 16], 256, 9728)
    need = prq.prq_lora_workspace_bytes(5, 2, 256, 9728, 64)
    a = c.run(workspace=torch.zeros(need, dtype=torch.uint8, device="cuda"))
    b = c.run(workspace=torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    assert torch.equal(a, b)
    with pytest.raises(prq.PRQError) as e:
        c.run(workspace=torch.zeros(max(need - 1, 0), dtype=torch.uint8, device="cuda"))
    assert e.value.status == prq.PRQ_EWORKSPACE


def test_no_rows_and_refused_shapes():
    prq = _prq()
    c = Case([4], [0], [16], 64, 128)
    assert prq.prq_lora(c.x[:0], c.adapters, c.offsets * 0, c.of, c.Y[:0]).shape == (0, 64)
    with pytest.raises(ValueError):
        prq.prq_lora(c.x, c.adapters, c.offsets[:1], c.of, c.Y)
    with pytest.raises(ValueError):
        prq.prq_lora(c.x[:, :120], c.adapters, c.offsets, c.of, c.Y)          # K of the adapters
    with pytest.raises(ValueError):
        prq.prq_lora(c.x, c.adapters, c.offsets, c.of, torch.zeros(4, 4096, device="cuda"))   # B too small
    with pytest.raises(ValueError):
        prq.prq_lora(c.x, c.adapters, c.offsets, c.of, c.Y.cpu())


@pytest.mark.parametrize("rows,of,ranks,N,K", [
    ([1] * 64, [i * 7 % 3 for i in range(64)], [16, 8, 64], 272, 2560),            # more than 16 rows of one
    ([1] * 64, [0] * 64, [32], 64, 6000), ([1] * 9, [1, 0, -1, 1, 5, 1, 0, -3, 1 << 30], [8, 200], 96, 264),
    ([0, 2, 0, 3, 1, 0, 5, 1, 1, 7], [0, 1, 1, 0, 2, 0, 1, -1, 0, 2], [48, 8, 24], 512, 4104),
    ([i % 2 for i in range(100)], [i // 2 % 4 for i in range(100)], [16, 16, 8, 40], 1040, 520),
    ([1] * 37, [36 - i if i % 5 else -1 for i in range(37)], [8 + 8 * (i % 3) for i in range(35)], 128, 9728)])
def test_rows_of_an_adapter_in_many_segments(rows, of, ranks, N, K):
    say("adapters of many segments", len(rows), ranks[:4], N, K)
    c = Case(rows, of, ranks, N, K, seed=N)
    out = c.run()
    c.check(out)
    Y = c.Y.clone()
    _prq().prq_lora(c.x, c.adapters, c.offsets, c.of, Y)
    assert torch.equal(Y, out)
    # a row's result does not depend on the rows beside it
    order = torch.from_numpy(np.random.default_rng(0).permutation(out.shape[0])).cuda()
    by_row = torch.repeat_interleave(c.of.long(), torch.tensor(rows, device="cuda"))
    d = Case([1] * out.shape[0], [0] * out.shape[0], [8], N, K)
    d.x, d.Y, d.adapters = c.x[order].contiguous(), c.Y[order].contiguous(), c.adapters
    d.of = by_row[order].int().contiguous()
    c.check(d.run()[torch.argsort(order)])


def test_rows_in_no_segment_are_left_alone_among_many_segments():
    c = Case([1] * 20, [0, 1] * 10, [16, 8], 64, 128)
    want = c.run()
    off = torch.arange(21, dtype=torch.int32, device="cuda")
    off[:3] = 2                                                    # rows 0 and 1: nobody's
    off[20] = 400
    c.offsets = off
    got = c.run()
    assert torch.equal(got[2:], want[2:]) and bool(torch.isnan(got[:2]).all())
    c.offsets = torch.flip(torch.arange(21, dtype=torch.int32, device="cuda"), [0]).contiguous()       # descending
    assert bool(torch.isnan(c.run()).all())


@pytest.mark.parametrize("rows,of,ranks,N,K", [
    ([1], [0], [1], 64, 128), ([3, 20], [1, 0], [5, 17], 64, 2560), ([100], [0], [33], 256, 264),
    ([2, 40], [0, 1], [3, 63], 128, 9728), ([300, 70], [1, 0], [100, 129], 64, 96), ([1] * 20, [0, 1] * 10, [12, 2], 64, 128),
    ([1] * 20, [0, 1] * 10, [200, 1], 64, 520)])
def test_an_infinity_meets_the_ranks_there_are(rows, of, ranks, N, K):
    """A is positive and a column of B has one sign, so that a row of x with an infinity becomes one of
    that sign everywhere: what pads a rank to a multiple of 8 does not make it 0 x inf."""
    say("infinity and padded ranks", len(rows), ranks, N, K)
    prq = _prq()
    c = Case(rows, of, ranks, N, K, seed=K)
    sign = torch.where(torch.arange(N, device="cuda") % 3 == 0, -1.0, 1.0)
    c.pairs = [(A.abs() + 2.0 ** -6, ((B.float().abs() + 0.5) * sign[:, None]).to(BF16)) for A, B in c.pairs]
    c.adapters = prq.prq_lora_adapters(c.pairs, c.scales)
    want = c.run()
    c.check(want)
    M = sum(rows)
    for r in {0, M // 2, M - 1}:
        c.x[r, (7 * r) % K] = float("inf")
    got = c.run()
    for r in range(M):
        if r in (0, M // 2, M - 1):
            assert torch.equal(got[r], sign * float("inf")), r
        else:
            assert torch.equal(got[r], want[r]), r


def test_ranks_that_do_not_fit_the_offsets():
    """A rank beyond what the offsets hold is what they hold, one below 1 is none; what the others pad
    a rank with is not read as one of its own, whatever it is."""
    prq = _prq()
    for rows, K in ([5, 6, 7], 128), ([1] * 3, 5000), ([100, 64, 40], 264):
        c = Case(rows, [0, 1, 2], [16, 16, 24], 64, K, seed=K)
        want = c.run()
        a = c.adapters
        ranks = torch.tensor([99, 16, 1 << 30], dtype=torch.int32, device="cuda")
        c.adapters = prq.LoraAdapters(a.A, a.B, a.rank_offsets, a.scales, a.max_rank, ranks)
        assert torch.equal(c.run(), want)
        ranks[:] = torch.tensor([0, 11, -(1 << 31)], dtype=torch.int32, device="cuda")
        got, n = c.run(), rows[0] + rows[1]
        assert torch.equal(got[:rows[0]], c.Y[:rows[0]]) and torch.equal(got[n:], c.Y[n:])
        c.of_host, c.pairs[1] = [-1, 1, -1], (c.pairs[1][0][:11], c.pairs[1][1][:, :11])
        c.check(got)
        a.A[a.rank_offsets[1] + 11:a.rank_offsets[1] + 16] = float("nan")
        assert torch.equal(c.run(), got)
        with pytest.raises(ValueError):
            c.adapters = prq.LoraAdapters(a.A, a.B, a.rank_offsets, a.scales, a.max_rank, ranks[:2])
            c.run()
