"""The calls of a mixture-of-experts half layer on the host (no GPU): the oracle's pins, argument checks
of the C calls and of the binding, workspace sizes."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import moe
from paper_2609_22106_amd import prq

FAKE, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4104)   # never dereferenced
S = ctypes.c_void_p(0)
EINVAL, EALIGN, EUNSUP, EWS = prq.PRQ_EINVAL, prq.PRQ_EALIGN, prq.PRQ_EUNSUPPORTED, prq.PRQ_EWORKSPACE


# ----------------------------------------------------------------- oracle pins ---
def test_oracle_norms():
    rng = np.random.default_rng(0)
    y, r = rng.standard_normal((2, 5, 16))
    s, h = moe.block_norm(y, r, pre=np.ones(16), eps=0.0)
    np.testing.assert_array_equal(s, r + y)
    np.testing.assert_allclose(np.mean(h * h, 1), 1)
    # the norm behind a block does not see its size, nor does the next one the sum's
    s2, h2 = moe.block_norm(7 * y, 3 * r, post=np.ones(16), pre=np.ones(16), eps=0.0, a=2.0, b=6.0)
    s1, h1 = moe.block_norm(y, r, post=np.ones(16), pre=np.ones(16), eps=0.0)
    np.testing.assert_allclose(s2, 6 * s1)
    np.testing.assert_allclose(h2, h1)
    # offset 1 and weight 0: the norm alone; a gate of zeros leaves the residual; none outside
    np.testing.assert_allclose(moe.block_norm(y, r, pre=np.zeros(16), eps=0.0, offset=1.0)[1], h)
    s, _ = moe.block_norm(y, r, gate=np.zeros((2, 16)), index=np.array([0, 1, -1, 2, 0]))
    np.testing.assert_array_equal(s, r + y * np.array([0, 0, 1, 1, 0])[:, None])


def test_oracle_route():
    l = np.array([[0.0, 3, 3, -1], [1, 1, 1, 1], [np.nan, 2, -np.inf, np.nan]])
    ids, w = moe.route(l[:2], 2)
    assert ids.tolist() == [[1, 2], [0, 1]]
    np.testing.assert_allclose(w, 0.5)
    np.testing.assert_allclose(moe.route(l[:2], 4, renormalize=False)[1].sum(1), 1)
    assert moe.route(l[2:], 4)[0].tolist() == [[1, 2, 0, 3]]                 # NaN last, in order
    # a bias moves the choice and not the weights
    ids, w = moe.route(l[:1], 2, sigmoid=True, bias=np.array([9.0, 0, 0, 8]), renormalize=False, scale=3.0)
    assert ids.tolist() == [[0, 3]]
    np.testing.assert_allclose(w, 3 / (1 + np.exp([[0.0, 1]])))


def test_oracle_layer_is_a_gated_mlp():
    rng = np.random.default_rng(1)
    x, up, down = rng.standard_normal((3, 8)), rng.standard_normal((2, 12, 8)), rng.standard_normal((2, 5, 8))
    ids, w = np.array([[0, 1], [1, -1], [1, 1]]), np.array([[0.3, 0.7], [0.5, 9], [0.25, 0.5]])

    def expert(e, v):
        g = up[e, :6] @ v
        h = g / (1 + np.exp(-g)) * (up[e, 6:] @ v)
        return down[e, :, :6] @ h + down[e, :, 6:] @ h[4:]
    y, size, root, reach = moe.layer(x, ids, w, up, down, 2)
    np.testing.assert_allclose(y, [0.3 * expert(0, x[0]) + 0.7 * expert(1, x[0]), 0.5 * expert(1, x[1]),
                                   0.75 * expert(1, x[2])])
    assert np.all(np.abs(y) <= size) and np.all(root <= size) and np.all(reach >= 0)


# ------------------------------------------------------------------ C refusals ---
NORM = dict(y=FAKE, ld_y=256, y_type=0, r=FAKE, ld_r=256, r_type=1, M=4, H=256, post=FAKE, pre=FAKE, w_type=1, offset=0.0,
            gate=FAKE, ld_gate=256, gate_type=1, gate_rows=2, index=FAKE, eps=1e-6, a=1.0, b=1.0, r_out=FAKE, ld_ro=256,
            h=FAKE, ld_h=256, stream=S)
ROUTE = dict(x=FAKE, ld_x=256, M=4, H=256, W=FAKE, ld_w=256, E=32, k=4, scoring=1, bias=FAKE, renorm=1, scale=1.0, ids=FAKE,
             weights=FAKE, logits=FAKE, ld_l=32, ws=FAKE, ws_bytes=1 << 30, stream=S)
LAYER = dict(x=FAKE, ld_x=256, M=4, ids=FAKE, weights=FAKE, k=2, up=FAKE, up_s=FAKE, down=FAKE, down_s=FAKE, E=8, H=256,
             I=64, tail=32, N=256, out=FAKE, ld_out=256, ws=FAKE, ws_bytes=1 << 30, stream=S)
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), EINVAL), (dict(H=0), EINVAL), (dict(eps=-1.0), EINVAL), (dict(eps=NAN), EINVAL), (dict(offset=INF), EINVAL),
    (dict(a=NAN), EINVAL), (dict(b=-INF), EINVAL), (dict(y_type=2), EINVAL), (dict(r_type=-1), EINVAL), (dict(w_type=7), EINVAL),
    (dict(gate_type=2), EINVAL), (dict(y=None), EINVAL), (dict(y=None, post=None), EINVAL),
    (dict(y=None, post=None, gate=None, index=None, r=None), EINVAL), (dict(pre=None), EINVAL), (dict(h=None), EINVAL),
    (dict(pre=None, h=None, r_out=None), EINVAL), (dict(gate=None), EINVAL), (dict(gate_rows=0), EINVAL),
    (dict(index=None, gate_rows=2), EINVAL), (dict(index=None, gate_rows=5), EINVAL), (dict(ld_y=248), EINVAL),
    (dict(ld_r=255), EINVAL), (dict(ld_gate=8), EINVAL), (dict(ld_ro=248), EINVAL), (dict(ld_ro=264), EINVAL),
    (dict(ld_h=0), EINVAL), (dict(H=252), EALIGN), (dict(y=ODD), EALIGN), (dict(r_out=ODD), EALIGN), (dict(h=ODD), EALIGN),
    (dict(gate=ODD), EALIGN), (dict(post=ODD), EALIGN), (dict(ld_y=258), EALIGN), (dict(ld_h=260), EALIGN),
    (dict(ld_gate=260), EALIGN), (dict(H=16392, ld_y=20000, ld_r=20000), EUNSUP), (dict(M=1 << 24), EUNSUP),
    (dict(M=0, y=None, r=None, h=None, r_out=None), 0)])
def test_block_norm_refuses_before_touching_the_gpu(change, status):
    assert prq._block_norm(*{**NORM, **change}.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), EINVAL), (dict(H=0), EINVAL), (dict(E=0), EINVAL), (dict(k=0), EINVAL), (dict(k=33), EINVAL),
    (dict(scoring=2), EINVAL), (dict(scoring=0), EINVAL), (dict(renorm=2), EINVAL), (dict(scale=NAN), EINVAL),
    (dict(x=None), EINVAL), (dict(W=None), EINVAL), (dict(ids=None), EINVAL), (dict(weights=None), EINVAL),
    (dict(ld_x=248), EINVAL), (dict(ld_w=8), EINVAL), (dict(ld_l=31), EINVAL), (dict(H=252), EALIGN), (dict(x=ODD), EALIGN),
    (dict(W=ODD), EALIGN), (dict(ld_x=260), EALIGN), (dict(ld_w=257), EALIGN), (dict(E=1025), EUNSUP),
    (dict(E=64, k=33, ld_l=64), EUNSUP), (dict(H=65544, ld_x=70000, ld_w=70000), EUNSUP), (dict(M=1 << 24), EUNSUP),
    (dict(M=0, x=None, ids=None, weights=None), 0)])
def test_route_refuses_before_touching_the_gpu(change, status):
    assert prq._route(*{**ROUTE, **change}.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(M=-1), EINVAL), (dict(k=0), EINVAL), (dict(E=0), EINVAL), (dict(H=0), EINVAL), (dict(I=0), EINVAL),
    (dict(tail=-32), EINVAL), (dict(N=0), EINVAL), (dict(x=None), EINVAL), (dict(ids=None), EINVAL), (dict(weights=None), EINVAL),
    (dict(up=None), EINVAL), (dict(up_s=None), EINVAL), (dict(down=None), EINVAL), (dict(down_s=None), EINVAL),
    (dict(out=None), EINVAL), (dict(ld_x=248), EINVAL), (dict(ld_out=248), EINVAL), (dict(H=248, ld_x=256), EALIGN),
    (dict(I=48), EALIGN), (dict(tail=16), EALIGN), (dict(tail=96), EALIGN), (dict(N=248), EALIGN), (dict(x=ODD), EALIGN),
    (dict(out=ODD), EALIGN), (dict(up=ODD), EALIGN), (dict(down_s=ODD), EALIGN), (dict(ld_x=260), EALIGN),
    (dict(ld_out=260), EALIGN), (dict(M=65), EUNSUP), (dict(k=33), EUNSUP), (dict(E=4097), EUNSUP),
    (dict(H=65568, ld_x=70000), EUNSUP), (dict(N=65552, ld_out=70000), EUNSUP), (dict(I=32800), EUNSUP),
    (dict(M=0, x=None, ids=None, out=None, ws=None), 0)])
def test_layer_refuses_before_touching_the_gpu(change, status):
    assert prq._moe(*{**LAYER, **change}.values()) == status


@pytest.mark.parametrize("call,pack,arguments,changes", [
    (prq._block_norm_call, prq._block_norm_pack, NORM,
     [(dict(M=-1), EINVAL), (dict(eps=NAN), EINVAL), (dict(a=1e300), EINVAL), (dict(H=252), EALIGN), (dict(M=1 << 24), EUNSUP),
      (dict(M=1 << 32), EINVAL), (dict(H=256 - (1 << 32)), EINVAL), (dict(M=0, y=None, r=None, h=None, r_out=None), 0)]),
    (prq._route_call, prq._route_pack, ROUTE,
     [(dict(k=0), EINVAL), (dict(scale=NAN), EINVAL), (dict(ld_x=260), EALIGN), (dict(E=1025), EUNSUP),
      (dict(E=(1 << 32) + 32), EINVAL), (dict(M=0, x=None, ids=None, weights=None), 0)]),
    (prq._moe_call, prq._moe_pack, LAYER,
     [(dict(tail=-32), EINVAL), (dict(out=ODD), EALIGN), (dict(M=65), EUNSUP), (dict(M=1 << 33), EINVAL),
      (dict(M=0, x=None, ids=None, out=None, ws=None), 0)])])
def test_records_are_the_calls(call, pack, arguments, changes):
    """The arguments in a record of 8 bytes each; integers past their parameter's range are refused, not cut."""
    for change, status in changes:
        values = [getattr(v, "value", v) or 0 for v in {**arguments, **change}.values()]      # (pointers as numbers)
        assert call(pack(*values)) == status, change
    assert call(None) == EINVAL


def test_workspace_sizes():
    assert prq.prq_moe_route_workspace_bytes(-1, 8, 64) == prq.prq_moe_route_workspace_bytes(4, 8, 60) == 0
    assert prq.prq_moe_route_workspace_bytes(0, 128, 2048) == prq.prq_moe_route_workspace_bytes(4, 2000, 64) == 0
    assert prq.prq_moe_route_workspace_bytes(1, 128, 2048) >= 16384 + 512   # tiles of experts meet there
    assert prq.prq_moe_route_workspace_bytes(1, 16, 2048) == 0              # one tile
    assert prq.prq_moe_route_workspace_bytes(1 << 20, 128, 2048) == 0       # a workgroup has all experts
    ws = prq.prq_moe_layer_workspace_bytes
    assert ws(65, 8, 128, 2048, 768, 64, 2048) == ws(0, 8, 128, 2048, 768, 64, 2048) == ws(4, 8, 128, 2048, 760, 0, 2048) == 0
    assert ws(64, 8, 128, 2048, 768, 64, 2048) >= 16384 + 64 * 8 * 768 * 2


# ------------------------------------------------------------ binding refusals ---
BF16 = torch.bfloat16


def test_binding_refuses_host_tensors_and_wrong_shapes():
    y, r, w = torch.zeros(3, 64), torch.zeros(3, 64, dtype=BF16), torch.ones(64)
    for args, kw in (((y, r, w), {}), ((None, r, w), {}), ((y, None, w), {}), ((None, None, w), {}), ((y[0], r, w), {})):
        with pytest.raises(ValueError):
            prq.prq_block_norm(*args, **kw)
    for kw in (dict(post_weight=w), dict(gate=torch.zeros(1, 64))):      # also where nothing would be launched
        with pytest.raises(ValueError, match="need y"):
            prq.prq_block_norm(None, r, **kw)
    W = torch.zeros(8, 64, dtype=BF16)
    with pytest.raises(ValueError, match="x must be"):
        prq.prq_moe_route(r, W, 2)                                       # not on a GPU
    with pytest.raises(ValueError, match="scoring"):
        prq.prq_moe_route(r, W, 2, scoring="top")
    up, down = prq.PackedWeight(w, w, 8, 128, 64), prq.PackedWeight(w, w, 8, 48, 96)
    ids = torch.zeros(3, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="x must be"):
        prq.prq_moe_layer(r, ids, torch.zeros(3, 2), up, down, k_tail=32)
    for bad in (dict(k_tail=0), dict(k_tail=64)):
        with pytest.raises(ValueError, match="fit"):
            prq.prq_moe_layer(r, ids, torch.zeros(3, 2), up, down, **bad)
    with pytest.raises(ValueError, match="fit"):
        prq.prq_moe_layer(r, ids, torch.zeros(3, 2), up, prq.PackedWeight(w, w, 9, 48, 96), k_tail=32)


class _At(torch.Tensor):
    """A tensor that says it is elsewhere."""

    def get_device(self):
        return self.index


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(prq, "_cur_device", lambda: 1)
    monkeypatch.setattr(prq, "_rows", lambda t, *a: t.shape[1])
    monkeypatch.setattr(prq, "_on_gpu", lambda **t: None)

    def at(index, *shape, dtype=BF16):
        t = torch.zeros(shape, dtype=dtype).as_subclass(_At)
        t.index = index
        return t
    w = at(1, 64, dtype=torch.float32)
    for y, r, g in ((at(0, 3, 64), at(1, 3, 64), None), (at(1, 3, 64), at(0, 3, 64), None),
                    (at(1, 3, 64), at(1, 3, 64), at(0, 1, 64))):
        with pytest.raises(ValueError, match="not the current device"):
            prq.prq_block_norm(y, r, w, gate=g)
    with pytest.raises(ValueError, match="W is on"):
        prq.prq_moe_route(at(1, 3, 64), at(0, 8, 64), 2)
    up, down = (prq.PackedWeight(at(1, n, dtype=torch.uint8), at(1, s, dtype=torch.uint8), 8, *size)
                for n, s, size in ((8 * 8 * 1024, 8 * 8 * 256, (128, 64)), (8 * 3 * 1024, 8 * 3 * 256, (48, 96))))
    ids = at(1, 3, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="weights is on"):
        prq.prq_moe_layer(at(1, 3, 64), ids, at(0, 3, 2, dtype=torch.float32), up, down, k_tail=32)
    down.Wps.index = 0
    with pytest.raises(ValueError, match="down.Wps is on"):
        prq.prq_moe_layer(at(1, 3, 64), ids, at(1, 3, 2, dtype=torch.float32), up, down, k_tail=32)


def test_oracle_route_with_a_nan_that_is_not_chosen():
    """What the header says: the chosen logits alone with renormalize, NaN without; a chosen infinity either way."""
    l = np.array([[2.0, np.nan, 3, 1], [np.inf, 0, 1, 2]])
    with np.errstate(invalid="ignore"):
        ids, w = moe.route(l, 2)
        of_all = moe.route(l, 2, renormalize=False)[1]
    assert ids.tolist() == [[2, 0], [0, 3]]
    np.testing.assert_allclose(w[0], np.exp([0, -1]) / (1 + np.exp(-1)))
    assert np.isnan(of_all).all() and np.isnan(w[1]).all()
