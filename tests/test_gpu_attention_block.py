"""The attention half of a layer: every stage against the float64 oracle on the stage's own input, a
tree against the chain of one of its paths, and the operators as they are used in a program: in a HIP
graph replayed beside eager work, and on a stream that is not the current one.

Bars: the projections' products 1e-3 of their largest value, and for the adapters, the norm and
rotation and the attention the bars that are derived beside their own tests."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention as at                     # noqa: E402
from oracle import prquant as pq                       # noqa: E402
from paper_2609_22106_amd import inputs                # noqa: E402
from tests.gpu_util import GEMM_RTOL_OF_MAX, say       # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
HIDDEN, HEADS, KV, D, PAGE = 256, 6, 2, 64, 16
RANKS, SCALES = [8, 40, 16], [0.5, 2.0, -1.0]


def _np(t):
    return t.double().cpu().numpy()


class Layer:
    """A small block and what the oracle needs of it."""

    def __init__(self, seed=0, max_rows=96, max_requests=4, longest=128):
        from paper_2609_22106_amd import attention_block as ab
        from paper_2609_22106_amd import prq
        rng = np.random.default_rng(seed)
        self.W, self.pairs, proj = [], [], []
        for N, K in (((HEADS + 2 * KV) * D, HIDDEN), (HIDDEN, HEADS * D)):
            W = inputs.f32_to_bf16_bits(rng.standard_normal((N, K), dtype=np.float32) * K ** -0.5)
            Xcal = inputs.f32_to_bf16_bits(rng.standard_normal((32, K), dtype=np.float32))
            pairs = [(torch.from_numpy(rng.standard_normal((r, K), dtype=np.float32) * K ** -0.5).to(BF16),
                      torch.from_numpy(rng.standard_normal((N, r), dtype=np.float32) * r ** -0.5).to(BF16))
                     for r in RANKS]
            proj.append(ab.Projection(W, Xcal, 0.5, 32, prq.prq_lora_adapters(pairs, SCALES), max_rows, max_requests))
            self.W.append(pq.prepare(W, Xcal, 0.5, 32))
            self.pairs.append([(_np(A), _np(B), s) for (A, B), s in zip(pairs, SCALES)])
        self.per = longest // PAGE
        self.weights = [torch.from_numpy((1 + 0.2 * rng.standard_normal(D)).astype(np.float32)).cuda()
                        for _ in range(2)]
        self.table = prq.prq_rope_table(longest, D, theta=1e4)
        self.cache = prq.prq_paged_kv(max_requests * self.per, KV, PAGE, D)
        self.block = ab.AttentionBlock(*proj, HEADS, self.cache, self.table, *self.weights, max_rows, max_requests,
                                       longest)
        self.pages = rng.permutation(max_requests * self.per).astype(np.int32).reshape(max_requests, self.per)

    def batch(self, requests, adapter):
        from paper_2609_22106_amd import attention_block as ab
        return ab.Batch(requests, self.pages[:len(requests)], PAGE, adapter)

    def project(self, i, x, offsets, of):
        """Projection i with adapters -> (values, error bound)."""
        w = self.W[i]
        bits = x.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
        y = pq.gemm(*pq.quant_act(bits, w["inv_scale"], w["perm"], 32), w["Wq"], w["Wsc"])
        out, size = at.lora(_np(x), y, self.pairs[i], offsets, of)
        return out, GEMM_RTOL_OF_MAX * np.max(np.abs(y)) + (x.shape[1] + 3 * max(RANKS) + 32) * 2.0 ** -24 * size

    def check(self, x, batch, requests, adapter):
        """Runs the block and checks each stage on the device's own input to it."""
        y = _np(self.block(x, batch))
        M, qkv = batch.M, _np(self.block.qkv.Y[:batch.M])
        off = np.concatenate([[0], np.cumsum([len(p) for _, p in requests])])
        want, tol = self.project(0, x, off, adapter)
        assert np.all(np.abs(qkv - want) <= tol)
        pos, slot, table = batch.position.cpu().numpy(), batch.slot.cpu().numpy(), _np(self.table)
        K, V = _np(self.cache.K), _np(self.cache.V)
        q = _np(self.block.q[:M])

        def near(a, b):
            assert np.all(np.abs(a - b) <= 2.0 ** -8 * np.abs(b) + 2.0 ** -17 * np.max(np.abs(b)))
        for i in range(M):
            heads = qkv[i].reshape(-1, D)
            for h in range(HEADS):
                near(q[i, h], at.norm_rotate(heads[h], _np(self.weights[0]), 1e-6, table[pos[i]], False))
            for h in range(KV):
                near(K[slot[i] // PAGE, h, slot[i] % PAGE],
                     at.norm_rotate(heads[HEADS + h], _np(self.weights[1]), 1e-6, table[pos[i]], False))
                near(V[slot[i] // PAGE, h, slot[i] % PAGE], heads[HEADS + KV + h])
        a = _np(self.block.attended[:M])
        for b, (cached, parents) in enumerate(requests):
            rows, L = slice(off[b], off[b + 1]), cached + len(parents)
            at_ = [self.pages[b, j // PAGE] for j in range(L)], slice(None), [j % PAGE for j in range(L)]
            see = np.zeros((len(parents),) * 2, bool)
            for i, p in enumerate(parents):
                see[i] = see[p] if p >= 0 else False
                see[i, i] = True
            out, _, spread, size = at.tree_attention(q[rows], K[at_], V[at_], cached, D ** -0.5, see)
            S = (D ** -0.5 * size + 16)[..., None]
            assert np.all(np.abs(a[rows] - out) <= 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2.0 ** -18 * S) * spread)
        want, tol = self.project(1, self.block.attended[:M].reshape(M, -1), off, adapter)
        assert np.all(np.abs(y - want) <= tol)
        return y


def _x(M, seed):
    return torch.randn((M, HIDDEN), generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(BF16)


def test_stages_match_oracle():
    layer = Layer()
    adapter = [2, -1, 0, 1]
    prompts = [(0, list(range(-1, n - 1))) for n in (17, 1, 40, 30)]
    mixed = [(17, [-1, 0, 0, 1, 2, -1]), (1, [-1]), (40, list(range(-1, 9))), (30, [-1, 0, 1, 0])]
    for step, requests in enumerate((prompts, mixed)):
        say("attention block, step", step)
        batch = layer.batch(requests, adapter)
        assert (batch.mask is None) == (requests is prompts)
        layer.check(_x(batch.M, step), batch, requests, adapter)


def test_a_path_of_a_tree_is_the_chain():
    """Rows 0, 1, 3 of the tree are a chain: as a chain of their own they are attended alike, at the
    same positions over the same cache (the rest of the tree sits in slots that they do not see).  Bar:
    both are within the attention's bar of the same q, keys and values where the projections agree bit
    for bit, which one row count for both gives."""
    layer = Layer(seed=1)
    layer.block(_x(20, 5), layer.batch([(0, list(range(-1, 19)))], [1]))
    K, V = layer.cache.K.clone(), layer.cache.V.clone()
    x = _x(5, 6)
    layer.block(x, layer.batch([(20, [-1, 0, 0, 1, 2])], [1]))
    tree, q = _np(layer.block.attended[:5]), _np(layer.block.q[:5])
    layer.cache.K.copy_(K)
    layer.cache.V.copy_(V)
    order = [0, 1, 3, 2, 4]
    layer.block(x[order].contiguous(), layer.batch([(20, [-1, 0, 1, 2, 3])], [1]))
    assert np.array_equal(_np(layer.block.q[:3]), q[order[:3]])
    chain = _np(layer.block.attended[:3])
    top = np.abs(_np(layer.cache.V)).max()
    assert np.all(np.abs(chain - tree[order[:3]]) <= 2 * (2.0 ** -7 + 2.0 ** -10) * top)


def _operators(seed):
    """[(call, its outputs)] of the three operators: the plans they have for few and many rows."""
    from paper_2609_22106_amd import prq
    g = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")       # noqa: E731
    ops = []
    # 600 tokens a request; one row each, trees of 5, chunks of 40
    cache = prq.PagedKV(rnd(40, KV, 64, 128).to(BF16), rnd(40, KV, 64, 128).to(BF16))
    pages = torch.arange(30, dtype=torch.int32, device="cuda").reshape(3, 10)
    for n in (1, 5, 40):
        M = 3 * n
        q = rnd(M, 8, 128).to(BF16)
        cached = torch.tensor([600 - n, 300, 17], dtype=torch.int32, device="cuda")
        off = torch.arange(0, M + 1, n, dtype=torch.int32, device="cuda")
        mask = rnd(M, n) > 0
        ws = torch.zeros(prq.prq_tree_attention_workspace_bytes(M, 3, 8, KV, 128, 640), dtype=torch.uint8,
                         device="cuda")
        assert ws.numel()                                             # the keys are split
        out = torch.empty((M, 8, 128), dtype=BF16, device="cuda")
        lse = torch.empty((M, 8), device="cuda")
        ops.append((lambda st=None, q=q, cached=cached, off=off, mask=mask, ws=ws, out=out, lse=lse:
                    prq.prq_tree_attention(q, cache, pages, cached, off, 0.1, mask, out=out, lse=lse, workspace=ws,
                                           stream=st), (out, lse)))
    pool = prq.prq_paged_kv(8, KV, 64, 128)
    table = prq.prq_rope_table(512, 128)
    for M in (1, 300):
        q, k, v = rnd(M, 8 * 128), rnd(M, KV * 128), rnd(M, KV * 128)
        pos = torch.arange(M, dtype=torch.int32, device="cuda")
        slots = torch.arange(M, device="cuda") + (300 if M == 1 else 0)
        out = torch.empty((M, 8, 128), dtype=BF16, device="cuda")
        ops.append((lambda st=None, a=(q, k, v, pos), slots=slots, out=out:
                    prq.prq_qk_norm_rope(*a, table, pool, slots, out=out, stream=st), (out, pool.K, pool.V)))
    for rows, N, K in (([1, 2], 512, 256), ([30, 33], 512, 5000), ([400, 0, 600], 1024, 256)):
        M = sum(rows)
        ad = prq.prq_lora_adapters([(rnd(r, K), rnd(N, r)) for r in (16, 64)], [0.5, 1.5])
        off = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device="cuda")
        of = torch.arange(len(rows), dtype=torch.int32, device="cuda") % 2
        x, Y, out = rnd(M, K).to(BF16), rnd(M, N), torch.empty((M, N), device="cuda")
        ws = torch.empty(max(1, prq.prq_lora_workspace_bytes(M, len(rows), N, K, 64)), dtype=torch.uint8,
                         device="cuda")
        ops.append((lambda st=None, x=x, ad=ad, off=off, of=of, Y=Y, out=out, ws=ws:
                    prq.prq_lora(x, ad, off, of, Y, out=out, workspace=ws, stream=st), (out,)))
    return ops


def _spoil(ops):
    for _, outs in ops:
        for t in outs:
            t.fill_(float("nan"))


def _run_and_keep(ops):
    for run, _ in ops:
        run()
    torch.cuda.synchronize()
    return [[t.clone() for t in outs] for _, outs in ops]


def _assert_same(ops, ref, what):
    torch.cuda.synchronize()
    for i, ((_, outs), want) in enumerate(zip(ops, ref)):
        for t, w in zip(outs, want):
            a, b = t.isnan(), w.isnan()                               # slots that nothing writes
            assert torch.equal(a, b) and torch.equal(t[~a], w[~b]), (what, i)


def test_graph_replays_match_eager():
    ops = _operators(3)
    say("graph of the attention block's operators")
    _spoil(ops)
    ref = _run_and_keep(ops)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for run, _ in ops:
            run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for run, _ in ops:
            run()
    other = _operators(4)
    for replay in range(5):
        _spoil(ops)
        graph.replay()
        _assert_same(ops, ref, f"replay {replay}")
        for run, _ in other:                                          # the program's own work
            run()
        torch.randn(1 << 20, device="cuda").sum().item()
    _spoil(ops)
    for run, _ in ops:
        run()
    _assert_same(ops, ref, "eager after the replays")


def test_another_stream():
    """Every call on a stream that is not the current one, behind work that is still running there:
    its inputs come from that stream."""
    from paper_2609_22106_amd import prq
    ops = _operators(7)
    _spoil(ops)
    ref = _run_and_keep(ops)
    _spoil(ops)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy = torch.randn((2048, 2048), device="cuda")
        for _ in range(20):
            busy = busy @ busy * 0.01
    for run, _ in ops:
        run(side)
    _assert_same(ops, ref, "side stream")
    # outputs and workspaces made by the call itself, as the side stream's own
    torch.cuda.synchronize()
    g = torch.Generator("cuda").manual_seed(9)
    M, N, K = 70, 256, 5000
    x, Y = torch.randn((M, K), generator=g, device="cuda").to(BF16), torch.randn((M, N), generator=g, device="cuda")
    ad = prq.prq_lora_adapters([(torch.randn((64, K), generator=g, device="cuda"),
                                 torch.randn((N, 64), generator=g, device="cuda"))], [1.0])
    off = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    of = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = prq.prq_lora(x, ad, off, of, Y, out=torch.empty_like(Y))
    torch.cuda.synchronize()
    late = torch.full_like(x, float("nan"))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy * 0.01
        late.copy_(x)
    got = prq.prq_lora(late, ad, off, of, Y, out=torch.empty_like(Y), stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_parameters_are_taken_as_tensors_are():
    """A module's Parameters in the place of inputs, tables and the cache: the bits of plain tensors."""
    from paper_2609_22106_amd import prq
    own = lambda t: torch.nn.Parameter(t.clone(), requires_grad=False)       # noqa: E731
    g = torch.Generator("cuda").manual_seed(31)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")       # noqa: E731
    M = 6
    pos, slots = torch.arange(M, dtype=torch.int32, device="cuda"), torch.arange(M, device="cuda")
    table, w = prq.prq_rope_table(64, 64), rnd(64).to(BF16)
    got = []
    for wrap in (lambda t: t.clone(), own):
        g.manual_seed(32)
        K, V = wrap(torch.zeros(4, KV, 16, 64, dtype=BF16, device="cuda")), wrap(torch.zeros(4, KV, 16, 64, dtype=BF16,
                                                                                        device="cuda"))
        cache = prq.PagedKV(K, V)
        q = prq.prq_qk_norm_rope(wrap(rnd(M, 8 * 64)), wrap(rnd(M, KV * 64)), wrap(rnd(M, KV * 64)), wrap(pos),
                                 wrap(table), cache, wrap(slots), wrap(w), wrap(w))
        pages = wrap(torch.arange(4, dtype=torch.int32, device="cuda")[None])
        one = torch.tensor([0, M], dtype=torch.int32, device="cuda")
        out, lse = prq.prq_tree_attention(wrap(q), cache, pages, wrap(one[:1]), wrap(one), 0.1,
                                          wrap(torch.ones(M, M, dtype=torch.bool, device="cuda")))
        ad = prq.prq_lora_adapters([(rnd(8, 128), rnd(64, 8))], [1.0])
        ad = prq.LoraAdapters(wrap(ad.A), wrap(ad.B), wrap(ad.rank_offsets), wrap(ad.scales), 8)
        y = prq.prq_lora(wrap(rnd(M, 128).to(BF16)), ad, wrap(one), wrap(one[:1]), wrap(rnd(M, 64)))
        got.append([t.detach().clone() for t in (q, K, V, out, lse, y)])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_a_captured_step_serves_other_tables():
    """One graph, replayed with other rows a request, lengths, pages, slots, positions, masks and
    adapters in its tables: each replay has an eager call's bits, and that call's stages match the
    oracle."""
    from paper_2609_22106_amd import prq
    layer = Layer(seed=2, longest=1024)
    rng = np.random.default_rng(12)
    g = torch.Generator("cuda").manual_seed(11)
    for t in (layer.cache.K, layer.cache.V):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))

    def step(M):
        """Tables of M rows of four requests; the mask M wide."""
        rows = np.diff(np.concatenate([[0], np.sort(rng.integers(0, M + 1, 3)), [M]]))
        requests = [(int(rng.integers(0, 1024 - M)), [int(rng.integers(-1, i)) if i else -1 for i in range(n)])
                    for n in rows]
        layer.pages = rng.permutation(layer.pages.size).astype(np.int32).reshape(layer.pages.shape)
        adapter = [int(a) for a in rng.integers(-1, len(RANKS), 4)]
        now = layer.batch(requests, adapter)
        see = torch.zeros((M, M), dtype=torch.bool, device="cuda")
        if now.mask is None:                                          # chains all of them
            row = 0
            for n in rows:
                see[row:row + n, :n] = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
                row += n
        else:
            see[:, :now.mask.shape[1]] = now.mask
        now.mask = see
        return now, requests, adapter

    for M in (4, 24, 70):                                             # 16, 64 and 64 columns a workgroup
        assert prq.prq_tree_attention_workspace_bytes(M, 4, HEADS, KV, D, 1024) > 16384       # keys are split
        static = step(M)[0]
        x = _x(M, M)
        layer.block(x, static)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = layer.block(x, static)
        for replay in range(5):
            say("captured step", M, "rows, replay", replay)
            now, requests, adapter = step(M)
            for name in ("position", "slot", "mask", "pages", "cached", "offsets", "adapter"):
                getattr(static, name).copy_(getattr(now, name))
            x.copy_(_x(M, 100 * M + replay))
            for t in (y, layer.block.q, layer.block.attended, layer.block.lse):
                t.fill_(float("nan"))
            graph.replay()
            got = [t.clone() for t in (y, layer.block.attended[:M], layer.block.lse[:M])]
            layer.check(x, now, requests, adapter)
            for a, b in zip(got, (y, layer.block.attended[:M], layer.block.lse[:M])):
                assert torch.equal(a, b)


def _calls(seed):
    """{name: (call(inputs, stream), inputs, the cache that it writes)} of the three operators' plans,
    with outputs and workspaces made by the call itself."""
    from paper_2609_22106_amd import prq
    g = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")       # noqa: E731
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")       # noqa: E731
    pages = torch.arange(30, dtype=torch.int32, device="cuda").reshape(3, 10)
    K, V = rnd(30, KV, 64, 128).to(BF16), rnd(30, KV, 64, 128).to(BF16)
    calls = {}
    for n in (1, 5, 40):                                              # 16, 64 and 256 columns a workgroup
        M, off, cached, mask = 3 * n, ints([0, n, 2 * n, 3 * n]), ints([600 - n, 300, 17]), rnd(3 * n, n) > 0
        assert prq.prq_tree_attention_workspace_bytes(M, 3, 8, KV, 128, 640) > 16384
        calls[f"attention, {n} rows a request"] = (
            lambda a, st, c=cached, o=off, m=mask: prq.prq_tree_attention(a[0], prq.PagedKV(a[1], a[2]), pages, c, o,
                                                                          0.1, m, max_kv_len=640, stream=st),
            (rnd(M, 8, 128).to(BF16), K, V), ())
    table = prq.prq_rope_table(512, 128)
    for M in (1, 300):
        pos, slots = torch.arange(M, dtype=torch.int32, device="cuda"), torch.arange(M, device="cuda")
        pool = prq.prq_paged_kv(8, KV, 64, 128)
        calls[f"norm and rotation, {M} rows"] = (
            lambda a, st, p=pos, s=slots, pool=pool: (prq.prq_qk_norm_rope(*a, p, table, pool, s, stream=st),
                                                      pool.K, pool.V),
            (rnd(M, 8 * 128), rnd(M, KV * 128), rnd(M, KV * 128)), (pool.K, pool.V))
    for rows, N, K_ in (([1, 2], 512, 256), ([30, 33], 512, 5000), ([400, 0, 600], 1024, 256)):
        M = sum(rows)
        ad = prq.prq_lora_adapters([(rnd(r, K_), rnd(N, r)) for r in (16, 64)], [0.5, 1.5])
        off, of = ints(np.concatenate([[0], np.cumsum(rows)])), ints([i % 2 for i in range(len(rows))])
        calls[f"adapters, {M} rows of {K_}"] = (
            lambda a, st, ad=ad, off=off, of=of: prq.prq_lora(a[0], ad, off, of, a[1], out=a[2], stream=st),
            (rnd(M, K_).to(BF16), rnd(M, N), torch.zeros((M, N), device="cuda")), ())
    return calls


def _outputs(result):
    return [t.clone() for t in (result if isinstance(result, tuple) else (result,))]


def _keep_busy(stream):
    with torch.cuda.stream(stream):
        busy = torch.randn((2048, 2048), device="cuda")
        for _ in range(40):
            busy = busy @ busy * 0.01


def test_inputs_made_late_on_the_calls_stream():
    """NaN until a stream that is not the current one, busy at first, writes them: a call on that
    stream waits for them, one on any other would read the NaN."""
    for name, (call, inputs, cache) in _calls(21).items():
        say("late inputs", name)
        want = _outputs(call([t.clone() for t in inputs], None))
        assert all(bool(torch.isfinite(t).all()) for t in want)
        late = [torch.full_like(t, float("nan")) for t in inputs]
        for t in cache:
            t.zero_()
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        _keep_busy(side)
        with torch.cuda.stream(side):
            for t, u in zip(late, inputs):
                t.copy_(u)
        got = call(late, side)
        torch.cuda.synchronize()
        for a, b in zip(_outputs(got), want):
            assert torch.equal(a, b), name


def test_a_call_on_another_stream_does_not_wait_for_the_current_one():
    """The current stream is busy while the call runs on its own: what the call makes for itself, a
    workspace that starts at zero among it, is ready there, also where both streams' memory was left
    full of ones."""
    for name, (call, inputs, cache) in _calls(22).items():
        say("busy current stream", name)
        want = _outputs(call([t.clone() for t in inputs], None))
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        for stream in (side, torch.cuda.current_stream()):
            with torch.cuda.stream(stream):
                dirty = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (1 << 14, 1 << 19, 1 << 21, 1 << 23)]
                del dirty
        args = [t.clone() for t in inputs]
        for t in cache:
            t.zero_()
        torch.cuda.synchronize()
        _keep_busy(torch.cuda.current_stream())
        got = call(args, side)
        side.synchronize()
        with torch.cuda.stream(side):
            got = _outputs(got)
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), name
