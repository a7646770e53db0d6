"""The mixture-of-experts half of a layer as one path: every stage against the oracle on what the stage
before it gave, in a graph with other inputs, on another stream, with inputs made late, two blocks at
once, behind the attention half; all within the bars of the operators' own tests."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import moe                                             # noqa: E402
from tests.gpu_util import say                                     # noqa: E402
from tests.test_gpu_moe_layer import Layer                         # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def _np(t):
    return t.double().cpu().numpy()


def _block(seed, hidden=256, E=24, k=4, I=96, k_tail=32, max_rows=150, **routing):
    from paper_2609_22106_amd import moe_block
    layer = Layer(E, hidden, I, k_tail, hidden, seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")    # noqa: E731
    block = moe_block.MoEBlock((rnd(E, hidden) * hidden ** -0.5).to(BF16), layer.gate_up, layer.down_w, k, k_tail,
                               1 + 0.1 * rnd(hidden), 1 + 0.1 * rnd(hidden), max_rows, **routing)
    return block, layer


def _inputs(M, hidden, seed, dtype=F32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(M, hidden, generator=g, device="cuda"), (2 * torch.randn(M, hidden, generator=g, device="cuda")).to(dtype)


def _check(block, layer, y, r0, residual, out, sigmoid=False):
    """Every stage on the values that the stage before it left."""
    M = y.shape[0]
    h, ids, weights, experts = block.h[:M], block.ids[:M], block.weights[:M], block.out[:M]
    half = 2.0 ** -8
    want_r, want_h = moe.block_norm(_np(y), _np(r0), pre=_np(block.norm_weight))
    assert np.all(np.abs(_np(h) - want_h) <= half * np.abs(want_h) + 2.0 ** -16 * np.max(np.abs(want_h)))
    logits = _np(h) @ _np(block.router).T
    want_ids, want_w = moe.route(logits, block.k, sigmoid)
    # a sum of 256 float32 products is off by less than 2^-16 of the largest logits here: wherever the
    # chosen ones and the next differ by more, the choice is the oracle's
    order = np.sort(logits, 1)[:, ::-1][:, :block.k + 1]
    clear = np.min(order[:, :-1] - order[:, 1:], 1) > 2.0 ** -14
    assert np.mean(clear) > 0.9
    np.testing.assert_array_equal(ids.cpu().numpy()[clear], want_ids[clear])
    assert np.all(np.abs(_np(weights) - want_w)[clear] <= 2.0 ** -13 * want_w[clear])
    for i in range(0, M, 64):
        layer.check(experts[i:i + 64], h[i:i + 64], ids[i:i + 64], weights[i:i + 64])
    want_r2, want_out = moe.block_norm(_np(experts), want_r, pre=_np(block.next_weight))
    # the residual lies between the two norms in its own type
    step = 2.0 ** -8 if residual.dtype is BF16 else 2.0 ** -22
    assert np.all(np.abs(_np(residual) - want_r2) <= 2 * step * (np.abs(want_r) + np.abs(want_r2)) + 2.0 ** -20)
    assert np.all(np.abs(_np(out) - want_out) <= half * np.abs(want_out) + 4 * step * np.max(np.abs(want_out)))


@pytest.mark.parametrize("M,dtype,routing", [(1, F32, {}), (7, BF16, {}), (64, F32, dict(scoring="sigmoid")), (150, F32, {})])
def test_stages_against_the_oracle(M, dtype, routing):
    say("moe block", M, dtype, routing)
    block, layer = _block(M, **routing)
    y, residual = _inputs(M, 256, M, dtype)
    r0 = residual.clone()
    out = block(y, residual)
    _check(block, layer, y, r0, residual, out, "scoring" in routing)
    assert not block.ws[:16384].any()


def test_graph_replays_equal_the_eager_result_with_other_inputs():
    block, _ = _block(3)
    y, residual = _inputs(40, 256, 1)
    block(y, residual.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block(y, residual)
    other, _ = _block(3)                                          # the same weights, buffers of its own
    for step in range(5):
        a, b = _inputs(40, 256, 10 + step)
        y.copy_(a)
        residual.copy_(b)
        graph.replay()
        want_r = b.clone()
        want = other(a, want_r)                                   # eager work between the replays
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(residual, want_r)


def test_two_graphs_share_a_workspace():
    """Of other sizes, replayed in turn: each leaves the workspace ready for the other."""
    small, big = _block(4)[0], _block(4)[0]
    big.ws = small.ws
    got, graphs = [], []
    inputs = [_inputs(m, 256, m) for m in (3, 64)]
    for block, (y, r) in zip((small, big), inputs):
        block(y, r.clone())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(block.experts(y.to(BF16)))
        graphs.append(graph)
    want = []
    for _ in range(3):
        for i, graph in enumerate(graphs):
            graph.replay()
            torch.cuda.synchronize()
            if len(want) <= i:
                want.append(got[i].clone())
            assert torch.equal(got[i], want[i])
    fresh = _block(4)[0]
    for i, (y, _) in enumerate(inputs):
        assert torch.equal(fresh.experts(y.to(BF16)), want[i])


def test_another_stream_and_inputs_made_late():
    """All calls on a side stream, inputs written there behind a long kernel; outputs and workspaces that the
    calls make themselves."""
    from paper_2609_22106_amd import prq
    block, layer = _block(5)
    y, residual = _inputs(33, 256, 2)
    want = block(y, residual.clone()).clone()
    side = torch.cuda.Stream()
    late_y, late_r = torch.zeros_like(y), torch.zeros_like(residual)
    side.wait_stream(torch.cuda.current_stream())
    a = torch.randn(4096, 4096, device="cuda")
    with torch.cuda.stream(side):
        for _ in range(4):
            a = a @ a * 1e-3
        late_y.copy_(y)
        late_r.copy_(residual)
    h, r = prq.prq_block_norm(late_y, late_r, block.norm_weight, stream=side)
    ids, weights = prq.prq_moe_route(h, block.router, block.k, stream=side)
    out = prq.prq_moe_layer(h, ids, weights, block.gate_up, block.down, k_tail=block.k_tail, stream=side)
    got, _ = prq.prq_block_norm(out, r, block.next_weight, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    (a, _), (b, _) = _block(6), _block(7)
    ya, ra = _inputs(64, 256, 1)
    yb, rb = _inputs(17, 256, 2)
    want_a, want_b = a(ya, ra.clone()).clone(), b(yb, rb.clone()).clone()
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in range(2)]
    copies = [(ra.clone(), rb.clone()) for _ in range(8)]
    torch.cuda.synchronize()
    for ca, cb in copies:
        with torch.cuda.stream(sides[0]):
            got_a = a(ya, ca)
        with torch.cuda.stream(sides[1]):
            got_b = b(yb, cb)
    torch.cuda.synchronize()
    assert torch.equal(got_a, want_a) and torch.equal(got_b, want_b)


def test_parameters_are_taken_where_tensors_are():
    from paper_2609_22106_amd import prq
    own = lambda t: torch.nn.Parameter(t, requires_grad=False)     # noqa: E731
    block, _ = _block(8)
    y, residual = _inputs(9, 256, 3)
    want = block(y, residual.clone()).clone()
    block.router, block.norm_weight, block.next_weight = own(block.router), own(block.norm_weight), own(block.next_weight)
    block.gate_up = prq.PackedWeight(own(block.gate_up.Wp), own(block.gate_up.Wps), block.gate_up.E, block.gate_up.N,
                                     block.gate_up.K_aug)
    assert torch.equal(block(y, residual.clone()), want)


def test_layer_behind_the_attention_half():
    """A decoding step through both halves, eager and as a graph."""
    from paper_2609_22106_amd import attention_block
    rng = np.random.default_rng(9)
    hidden, B = 256, 6
    attention = attention_block.random_block(rng, hidden, 4, 2, 64, 12, 16, [8], B, B, 32)
    block, layer = _block(10)
    pages = rng.permutation(12).astype(np.int32).reshape(B, 2)
    batch = attention_block.Batch([(int(c), [-1]) for c in rng.integers(0, 30, B)], pages, 16, [0, -1, 0, 0, -1, 0])
    x = torch.randn(B, hidden, device="cuda").to(BF16)
    residual = torch.randn(B, hidden, device="cuda")
    r0 = residual.clone()
    y = attention(x, batch).clone()
    out = block(y, residual).clone()
    _check(block, layer, y, r0, residual, out)
    graph = torch.cuda.CUDAGraph()
    live = r0.clone()
    with torch.cuda.graph(graph):
        got = block(attention(x, batch), live)
    for _ in range(3):
        live.copy_(r0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(live, residual)


def test_the_command_runs(capsys):
    import json
    from paper_2609_22106_amd import moe_block
    assert moe_block.main([]) == 0
    lines = [json.loads(s) for s in capsys.readouterr().out.splitlines() if s.startswith("{")]
    assert [s["sequences"] for s in lines] == [1, 64] and all(s["us"] > 0 for s in lines)


def test_workspaces_of_the_calls_own_in_a_graph():
    """Calls without a workspace inside a capture: made and cleared there, on every replay."""
    from paper_2609_22106_amd import prq
    block, _ = _block(11, E=300)
    y, residual = _inputs(40, 256, 4)

    def step(r):
        h, _ = prq.prq_block_norm(y, r, block.norm_weight)
        ids, weights = prq.prq_moe_route(h, block.router, block.k)
        return prq.prq_moe_layer(h, ids, weights, block.gate_up, block.down, k_tail=block.k_tail)
    want = step(residual.clone()).clone()
    torch.cuda.synchronize()
    live = residual.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(live)
    for _ in range(4):
        live.copy_(residual)
        graph.replay()
        assert torch.equal(step(residual.clone()), want)           # eager work between the replays
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("M", [0, 1])
def test_no_token_and_one(M):
    block, layer = _block(12, max_rows=4)
    y, residual = _inputs(M, 256, 5)
    r0 = residual.clone()
    out = block(y, residual)
    assert out.shape == (M, 256)
    if M:
        _check(block, layer, y, r0, residual, out)
    with pytest.raises(ValueError):
        block(*_inputs(5, 256, 6))                                 # more rows than the block has room for
