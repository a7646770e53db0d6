"""The attention block's calls on the host (no GPU): the oracle's pins, the rotation
tables, argument checks of the C calls and of the binding."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import attention as at
from paper_2609_22106_amd import prq

FAKE, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4104)   # never dereferenced
S = ctypes.c_void_p(0)


# ----------------------------------------------------------------- oracle pins ---
def test_oracle_rotation_keeps_lengths_and_depends_on_distance_only():
    rng = np.random.default_rng(0)
    f, _ = at.rope_frequencies(16, 100.0)
    q, k = rng.standard_normal((2, 16))

    def turned(x, p, inter):
        return at.norm_rotate(x, None, 0.0, [(np.cos(p * w), np.sin(p * w)) for w in f], inter)
    for inter in (False, True):
        a = turned(q, 9, inter) @ turned(k, 4, inter)
        b = turned(q, 105, inter) @ turned(k, 100, inter)
        assert abs(a - b) < 1e-10
        assert abs(np.linalg.norm(turned(q, 9, inter)) - np.linalg.norm(q)) < 1e-12
        # a pair turned by its angle is a product of complex numbers
        i, j = (6, 7) if inter else (3, 11)
        z = (q[i] + 1j * q[j]) * np.exp(9j * f[3])
        got = turned(q, 9, inter)
        assert abs(got[i] + 1j * got[j] - z) < 1e-12


def test_oracle_norm_makes_unit_mean_square():
    x = 7 * np.random.default_rng(1).standard_normal(64)
    y = at.norm_rotate(x, np.ones(64), 0.0, [], False)
    assert abs(np.mean(y * y) - 1) < 1e-12


def test_oracle_attention_special_cases():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 7, 2, 8))
    q = rng.standard_normal((3, 4, 8))
    # equal scores: the mean of what is seen (4 cached and own tokens 0 .. i)
    out, lse, _, _ = at.tree_attention(0 * q, k, v, 4, 1.0)
    for i in range(3):
        np.testing.assert_allclose(out[i, 3], v[:5 + i, 1].mean(0))
        np.testing.assert_allclose(lse[i], np.log(5 + i))
    # a mask of the lower triangle is the chain; an empty row without cached tokens is 0
    tri = np.tril(np.ones((3, 3), bool))
    np.testing.assert_array_equal(at.tree_attention(q, k, v, 4, 0.3, tri)[0], at.tree_attention(q, k, v, 4, 0.3)[0])
    out, lse, _, _ = at.tree_attention(q, k[:3], v[:3], 0, 0.3, np.zeros((3, 3), bool))
    assert not out.any() and np.all(lse == -np.inf)


def test_oracle_adapters_are_a_low_rank_weight():
    rng = np.random.default_rng(3)
    x, Y = rng.standard_normal((5, 12)), rng.standard_normal((5, 6))
    A, B = rng.standard_normal((2, 12)), rng.standard_normal((6, 2))
    out, _ = at.lora(x, Y, [(A, B, 0.5)], [0, 2, 5], [-1, 0])
    np.testing.assert_array_equal(out[:2], Y[:2])
    np.testing.assert_allclose(out[2:], Y[2:] + x[2:] @ (0.5 * B @ A).T)


# ---------------------------------------------------------------------- tables ---
@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0),
                                dict(scaling="yarn", factor=4.0, original_positions=4096),
                                dict(scaling="yarn", factor=1.0, original_positions=64, theta=100.0)])
@pytest.mark.parametrize("rot", [8, 64, 128])
def test_rope_table_matches_oracle(rot, kw):
    theta = kw.pop("theta", 1e6)
    t = prq.prq_rope_table(300, rot, theta=theta, device="cpu", **kw).numpy()
    f, gain = at.rope_frequencies(rot, theta, kw.get("scaling", "none"), kw.get("factor", 1.0),
                                  kw.get("original_positions"))
    assert t.shape == (300, rot // 2, 2) and t.dtype == np.float32
    angle = np.arange(300)[:, None] * f
    # angles differ by rounding of float64 products and powers only; then one float32 rounding
    tol = 2.0 ** -24 * gain + 300 * 2.0 ** -48
    assert np.max(np.abs(t[..., 0] - gain * np.cos(angle))) <= tol
    assert np.max(np.abs(t[..., 1] - gain * np.sin(angle))) <= tol


def test_rope_table_scalings_at_their_ends():
    """linear and ntk slow the slowest pair by the factor, ntk leaves the fastest; yarn leaves the
    fastest and slows the slowest."""
    f0, _ = at.rope_frequencies(64, 1e4)
    for kind, first, last in (("linear", 8, 8), ("ntk", 1, 8), ("yarn", 1, 8)):
        f, _ = at.rope_frequencies(64, 1e4, kind, 8.0, 2048)
        np.testing.assert_allclose([f0[0] / f[0], f0[-1] / f[-1]], [first, last], rtol=1e-9)


@pytest.mark.parametrize("bad", [dict(rotary_dim=12), dict(rotary_dim=0), dict(rotary_dim=8, scaling="no"),
                                 dict(rotary_dim=8, factor=0.5), dict(rotary_dim=8, theta=1.0),
                                 dict(rotary_dim=8, scaling="yarn", factor=2.0)])
def test_rope_table_refuses(bad):
    with pytest.raises(ValueError):
        prq.prq_rope_table(16, device="cpu", **bad)


# ------------------------------------------------------------------ C refusals ---
ROPE = dict(q=FAKE, ld_q=4096, k=FAKE, ld_k=1024, v=FAKE, ld_v=1024, in_type=0, M=4, Hq=32, Hk=8, D=128, wq=FAKE,
            wk=FAKE, w_type=1, eps=1e-6, pos=FAKE, table=FAKE, rows=100, rot=128, inter=0, out=FAKE, K=FAKE, V=FAKE,
            stride=8 * 64 * 128, pages=10, page=64, slots=FAKE, stream=S)
TREE = dict(q=FAKE, ld_q=4096, M=4, Hq=32, Hk=8, D=128, K=FAKE, V=FAKE, stride=8 * 64 * 128, pages=10, page=64,
            table=FAKE, ld_pages=6, wide=6, cached=FAKE, offsets=FAKE, B=2, max_kv=300, scale=0.1, mask=FAKE,
            ld_mask=4, mask_wide=4, out=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 40, stream=S)
LORA = dict(x=FAKE, ld_x=256, M=4, K=256, A=FAKE, B=FAKE, rank_offsets=FAKE, scales=FAKE, adapters=2, rank_rows=32,
            max_rank=16, offsets=FAKE, of=FAKE, segments=2, N=64, Y=FAKE, ld_y=64, out=FAKE, ld_out=64, ws=FAKE,
            ws_bytes=1 << 40, stream=S)
EINVAL, EALIGN, EUNSUP, EWS = prq.PRQ_EINVAL, prq.PRQ_EALIGN, prq.PRQ_EUNSUPPORTED, prq.PRQ_EWORKSPACE


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), EINVAL), (dict(q=None), EINVAL), (dict(slots=None), EINVAL), (dict(pos=None), EINVAL),
    (dict(table=None), EINVAL), (dict(in_type=2), EINVAL), (dict(w_type=-1), EINVAL), (dict(inter=3), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(eps=-1.0), EINVAL), (dict(Hq=30), EINVAL), (dict(Hk=0), EINVAL),
    (dict(ld_q=4095), EINVAL), (dict(ld_v=1020), EINVAL), (dict(stride=8 * 64 * 128 - 8), EINVAL),
    (dict(pages=0), EINVAL), (dict(K=None), EINVAL), (dict(D=96, rot=96), EUNSUP), (dict(page=48), EUNSUP),
    (dict(page=8), EUNSUP), (dict(page=8192), EUNSUP), (dict(Hq=2048, ld_q=1 << 20), EUNSUP), (dict(M=1 << 24), EUNSUP),
    (dict(rot=12), EALIGN), (dict(rot=136), EALIGN), (dict(k=ODD), EALIGN), (dict(ld_q=4098), EALIGN),
    (dict(in_type=1, ld_k=1028), EALIGN), (dict(table=ODD), EALIGN), (dict(wk=ODD), EALIGN), (dict(V=ODD), EALIGN),
    (dict(stride=8 * 64 * 128 + 4), EALIGN), (dict(M=0, q=None, k=None, v=None, slots=None, out=None), 0)])
def test_norm_rope_refuses_before_touching_the_gpu(change, status):
    assert prq._qk_norm_rope(*{**ROPE, **change}.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), EINVAL), (dict(B=-1), EINVAL), (dict(max_kv=-1), EINVAL), (dict(q=None), EINVAL),
    (dict(out=None), EINVAL), (dict(cached=None), EINVAL), (dict(offsets=None), EINVAL), (dict(table=None), EINVAL),
    (dict(ld_pages=5), EINVAL), (dict(wide=-1), EINVAL), (dict(ld_mask=3), EINVAL), (dict(mask_wide=-1), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(ld_q=4000), EINVAL), (dict(Hq=12), EINVAL), (dict(D=80), EUNSUP),
    (dict(page=100), EUNSUP), (dict(B=5000), EUNSUP), (dict(M=1 << 21), EUNSUP),
    (dict(wide=1 << 25, ld_pages=1 << 25), EUNSUP), (dict(q=ODD), EALIGN), (dict(out=ODD), EALIGN),
    (dict(ld_q=4100), EALIGN), (dict(K=ODD), EALIGN), (dict(M=0, q=None, out=None), 0), (dict(B=0, table=None), 0)])
def test_tree_attention_refuses_before_touching_the_gpu(change, status):
    assert prq._tree(*{**TREE, **change}.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), EINVAL), (dict(segments=-1), EINVAL), (dict(N=0), EINVAL), (dict(K=-8), EINVAL),
    (dict(max_rank=-8), EINVAL), (dict(adapters=-1), EINVAL), (dict(rank_rows=-1), EINVAL), (dict(x=None), EINVAL),
    (dict(Y=None), EINVAL), (dict(out=None), EINVAL), (dict(A=None), EINVAL), (dict(scales=None), EINVAL),
    (dict(offsets=None), EINVAL), (dict(of=None), EINVAL), (dict(ld_x=248), EINVAL), (dict(ld_out=60), EINVAL),
    (dict(ld_y=68), EINVAL), (dict(N=56), EALIGN), (dict(K=252), EALIGN), (dict(max_rank=12), EALIGN),
    (dict(x=ODD), EALIGN), (dict(B=ODD), EALIGN), (dict(ld_x=260), EALIGN), (dict(ld_y=66, ld_out=66), EALIGN),
    (dict(max_rank=264), EUNSUP), (dict(segments=4097), EUNSUP), (dict(M=(1 << 19) + 1), EUNSUP),
    (dict(M=0, x=None, Y=None, out=None), 0), (dict(segments=0, offsets=None, of=None), 0)])
def test_lora_refuses_before_touching_the_gpu(change, status):
    assert prq._lora(*{**LORA, **change}.values()) == status


def test_workspace_sizes_of_refused_sizes_are_zero():
    assert prq.prq_tree_attention_workspace_bytes(-1, 1, 32, 8, 128, 100) == 0
    assert prq.prq_tree_attention_workspace_bytes(1, 1, 32, 8, 80, 100) == 0
    assert prq.prq_tree_attention_workspace_bytes(0, 1, 32, 8, 128, 100) == 0
    assert prq.prq_lora_workspace_bytes(4, 2, 60, 256, 16) == 0
    assert prq.prq_lora_workspace_bytes(0, 2, 64, 256, 16) == 0
    # a few rows over many keys, or a long K, are split: there is something to join
    assert prq.prq_tree_attention_workspace_bytes(1, 1, 32, 8, 128, 4096) > 0
    assert prq.prq_lora_workspace_bytes(64, 64, 2560, 9728, 64) > 0


# ------------------------------------------------------------ binding refusals ---
def test_binding_refuses_host_tensors_and_wrong_shapes():
    K = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        prq.PagedKV(K, K)                                            # not on a GPU
    with pytest.raises(ValueError):
        prq.PagedKV(K.float(), K.float())
    cache = object.__new__(prq.PagedKV)
    cache.K, cache.V, cache.pages, cache.heads, cache.page_size, cache.D, cache.stride = K, K, 4, 2, 16, 64, 2048
    q, kv = torch.zeros(3, 256), torch.zeros(3, 128)
    i32, i64 = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    table = torch.zeros(10, 32, 2)
    with pytest.raises(ValueError, match="q must"):
        prq.prq_qk_norm_rope(q, kv, kv, i32, table, cache, i64)      # not on a GPU
    with pytest.raises(ValueError, match="heads"):
        prq.prq_qk_norm_rope(q[:, :100], kv, kv, i32, table, cache, i64)
    with pytest.raises(ValueError, match="q must"):
        prq.prq_tree_attention(q.view(3, 4, 64), cache, i32.view(3, 1), i32, i32, 1.0)
    with pytest.raises(ValueError):
        prq.prq_lora(kv.bfloat16(), None, i32, i32, q)
    with pytest.raises(ValueError):
        prq.prq_lora_adapters([], [])
    with pytest.raises(ValueError):
        prq.prq_lora_adapters([(torch.zeros(4, 32), torch.zeros(16, 5))], [1.0], device="cpu")


def test_adapters_are_laid_out_padded():
    g = torch.Generator().manual_seed(0)
    pairs = [(torch.randn(r, 32, generator=g), torch.randn(16, r, generator=g)) for r in (3, 8, 16)]
    a = prq.prq_lora_adapters(pairs, [1.0, 2.0, 0.5], device="cpu")
    assert a.rank_offsets.tolist() == [0, 8, 16, 32] and a.max_rank == 16 and a.scales.tolist() == [1.0, 2.0, 0.5]
    for i, (A, B) in enumerate(pairs):
        lo, hi = a.rank_offsets[i], a.rank_offsets[i + 1]
        r = A.shape[0]
        assert torch.equal(a.A[lo:lo + r], A.bfloat16()) and not a.A[lo + r:hi].any()
        got = a.B[16 * lo:16 * hi].view(16, -1)
        assert torch.equal(got[:, :r], B.bfloat16()) and not got[:, r:].any()


@pytest.mark.parametrize("M,B,Hq,Hk,D", [(1, 1, 32, 8, 128), (377, 8, 32, 8, 128), (3, 2, 4, 2, 256), (40, 40, 12, 12, 64)])
def test_workspace_does_not_shrink_as_requests_may_be_longer(M, B, Hq, Hk, D):
    """Up to the largest length, which says that none is known."""
    top = (1 << 31) - 1
    sizes = [prq.prq_tree_attention_workspace_bytes(M, B, Hq, Hk, D, kv)
             for kv in (0, 1, 100, 1 << 12, 10 ** 6, 1 << 30, top - 255, top - 127, top - 1, top, top + 1, 1 << 32, 1 << 40)]
    assert sizes == sorted(sizes) and sizes[-1] > 0


def test_a_wave_barrier_stands_between_fences():
    """The barrier builtin orders no memory for the compiler: wherever lanes of a wave hand values to
    each other through LDS, a release comes before it and an acquire behind it."""
    found = 0
    for root, _, files in os.walk(os.path.dirname(prq.__file__)):
        for name in files:
            if name.endswith((".hip", ".hpp", ".h", ".cpp")):
                lines = [s.strip() for s in open(os.path.join(root, name))]
                for i, line in enumerate(lines):
                    if line.startswith("__builtin_amdgcn_wave_barrier"):
                        found += 1
                        assert lines[i - 1].startswith("__builtin_amdgcn_fence(__ATOMIC_RELEASE"), (name, i + 1)
                        assert lines[i + 1].startswith("__builtin_amdgcn_fence(__ATOMIC_ACQUIRE"), (name, i + 1)
    assert found


def test_adapters_carry_the_ranks_that_are_their_own():
    pairs = [(torch.ones(r, 32), torch.ones(16, r)) for r in (3, 8, 16)]
    assert prq.prq_lora_adapters(pairs, [1.0] * 3, device="cpu").ranks.tolist() == [3, 8, 16]
    assert prq.prq_lora_adapters(pairs[1:], [1.0] * 2, device="cpu").ranks is None          # nothing is padded


@pytest.mark.parametrize("ranks", [None, FAKE])
@pytest.mark.parametrize("change,status", [
    (dict(M=-1), EINVAL), (dict(x=None), EINVAL), (dict(scales=None), EINVAL), (dict(N=56), EALIGN),
    (dict(max_rank=264), EUNSUP), (dict(M=0, x=None, Y=None, out=None), 0), (dict(segments=0, offsets=None, of=None), 0)])
def test_lora_with_ranks_refuses_as_without(change, status, ranks):
    args = list({**LORA, **change}.values())
    assert prq._lora_ex(*args[:7], ranks, *args[7:]) == status


@pytest.mark.parametrize("dtype,kind", [(torch.float32, prq.PRQ_F32), (torch.bfloat16, prq.PRQ_BF16)])
@pytest.mark.parametrize("own", [lambda t: t, lambda t: torch.nn.Parameter(t)])
def test_a_norm_weight_has_its_own_type(monkeypatch, dtype, kind, own):
    """A module's Parameter too, which takes the checks' other way: its bf16 values are not float32."""
    monkeypatch.setattr(prq, "_on_gpu", lambda **t: None)
    w = own(torch.ones(64, dtype=dtype))
    assert prq._head_weight(w, "q_weight", 64) == (w.data_ptr(), kind)
