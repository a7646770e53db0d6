"""Performance cases of the operators of a mixture-of-experts half layer on one MI355X.

Three operators, each through the public calls of ``paper_2609_22106_amd.prq``:

* ``norm``: ``prq_block_norm`` -- the norm behind a block, its gate, the scaled residual sum and the
  norm before the next block, in one pass;
* ``route``: ``prq_moe_route`` -- the router's product, the experts of every token and their weights;
* ``experts``: ``prq_moe_layer`` -- all experts of a few tokens: gate and up products, SiLU, down product
  with its residual tail, weighted sum, MXFP4 weights and bf16 activations.

``run`` computes the plain form, elementary torch operations in 32 bits, or with ``own`` set the calls
above.  Layouts:

* rows row-major; ``gate`` [gate rows, H], ``gate_index`` int32 [M] the gate row of each row;
* router weight bf16 [E, H]; ids int32 [M, k] by descending score, weights float32 [M, k];
* expert weights in MXFP4 (E2M1 codes two a byte, an E8M0 scale for 32): gate_up [E, 2 I, H] (gate rows,
  then up rows), down [E, N, I + tail], whose last ``tail`` columns meet the last ``tail`` of the I
  intermediate values a second time.  A program keeps them packed as ``include/prq.h`` lays down.
"""
import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6
# (experts, experts a token, hidden, intermediate, tail): the expert shape that this repository
# benchmarks, and generic others: few wide experts, odd step counts, no tail
LAYERS = ((128, 8, 2048, 768, 64), (64, 6, 2560, 1408, 0), (16, 2, 1056, 352, 32), (8, 2, 2048, 2816, 64),
          (32, 4, 1024, 512, 32))
ROUTERS = ((128, 8, 2048), (64, 6, 2560), (16, 2, 1056), (8, 2, 4096), (250, 8, 1024))
HIDDEN = (2560, 2048, 1024, 4096, 1056, 5128)


def listed():
    return [
        # one sequence decoding: between the attention's output and the experts
        dict(name="norm 1 row", op="norm", M=1, H=2048, y32=True, r32=False, post=False, gates=0, a=1.0, b=1.0),
        # an odd batch decoding, norms on both sides of the block and one gate for all rows
        dict(name="norm 61 rows", op="norm", M=61, H=2560, y32=True, r32=False, post=True, gates=1, a=1.0, b=1.0),
        # ragged prompts, a gate for each of five requests, bf16 throughout, a width that is no power of two
        dict(name="norm ragged 1537 rows", op="norm", M=1537, H=1056, y32=False, r32=False, post=True, gates=5, a=1.0, b=0.22),
        # a long prompt, the residual kept in 32 bits and scaled
        dict(name="norm 8192 rows", op="norm", M=8192, H=2560, y32=True, r32=True, post=True, gates=0, a=0.9, b=0.5),
        # one token's eight of 128 experts
        dict(name="route 1 token", op="route", M=1, E=128, k=8, H=2048, sigmoid=False, renorm=True),
        # a decoding batch, scores by sigmoid with a correction of the selection
        dict(name="route 61 tokens", op="route", M=61, E=64, k=6, H=2560, sigmoid=True, renorm=True),
        # ragged prompts over more experts than a power of two, weights of the whole softmax
        dict(name="route 1537 tokens", op="route", M=1537, E=250, k=8, H=1024, sigmoid=False, renorm=False),
        # a long prompt
        dict(name="route 8192 tokens", op="route", M=8192, E=128, k=8, H=2048, sigmoid=False, renorm=True),
        # one sequence decoding: eight experts' weights
        dict(name="experts 1 token", op="experts", M=1, E=128, k=8, H=2048, I=768, tail=64),
        # seven tokens over few small experts, odd sizes
        dict(name="experts 7 tokens", op="experts", M=7, E=16, k=2, H=1056, I=352, tail=32),
        # a small batch over wider experts without a tail
        dict(name="experts 19 tokens", op="experts", M=19, E=64, k=6, H=2560, I=1408, tail=0),
        # a decoding batch that reaches nearly all experts: the largest
        dict(name="experts 64 tokens", op="experts", M=64, E=128, k=8, H=2048, I=768, tail=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm", "route", "experts"))
    if op == "norm":
        H = rng.choice(HIDDEN)
        M = _log_int(rng, 1, min(8192, 8192 * 2560 // H))
        return dict(op=op, M=M, H=H, y32=rng.random() < 0.6, r32=rng.random() < 0.4, post=rng.random() < 0.6,
                    gates=rng.choice((0, 0, 1, min(M, 7))), a=rng.choice((1.0, 0.9)), b=rng.choice((1.0, 0.22)))
    if op == "route":
        E, k, H = rng.choice(ROUTERS)
        M = _log_int(rng, 1, min(8192, 8192 * 2048 // max(H, 2048)))
        return dict(op=op, M=M, E=E, k=k, H=H, sigmoid=rng.random() < 0.4, renorm=rng.random() < 0.7)
    E, k, H, I, tail = rng.choice(LAYERS)
    return dict(op=op, M=_log_int(rng, 1, 64), E=E, k=k, H=H, I=I, tail=tail)


# ------------------------------------------------------------------- inputs ---
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * seed + stream)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _prepare_norm(c, seed):
    g = _gen(seed, 1)
    M, H = c["M"], c["H"]
    y, r = _randn(g, M, H), 2 * _randn(g, M, H)
    r[:, torch.randperm(H, generator=g, device=DEV)[:max(1, H // 200)]] *= 30.0       # outlier channels
    gates = c["gates"]
    index = None
    if gates > 1:
        at = torch.sort(torch.randint(0, M, (gates - 1,), generator=g, device=DEV)).values
        index = (torch.arange(M, device=DEV)[:, None] >= at).sum(1).to(torch.int32)
    return dict(case=c, y=y if c["y32"] else y.bfloat16(), r=r if c["r32"] else r.bfloat16(),
                post=(1 + 0.2 * _randn(g, H)).bfloat16() if c["post"] else None, pre=(1 + 0.2 * _randn(g, H)).bfloat16(),
                gate=(1 + 0.3 * _randn(g, gates, H)).bfloat16() if gates else None, index=index,
                r_out=torch.empty(M, H, dtype=torch.float32 if c["r32"] else torch.bfloat16, device=DEV),
                h=torch.empty(M, H, dtype=torch.bfloat16, device=DEV))


def _prepare_route(c, seed):
    """Activations and weights on a grid (steps of 2^-4 and 2^-9): their products' sums are exact in 32 bits, so
    that experts with nearly the same score come in one order, and equal ones do occur."""
    g = _gen(seed, 2)
    M, E, H = c["M"], c["E"], c["H"]
    x = (torch.round(_randn(g, M, H) * 16) / 16).clamp(-7, 7)
    w = torch.round(_randn(g, E, H) * (512 / math.sqrt(H))) / 512
    return dict(case=c, x=x.bfloat16(), w=w.bfloat16(), bias=0.1 * _randn(g, E) if c["sigmoid"] else None,
                ids=torch.empty(M, c["k"], dtype=torch.int32, device=DEV), weights=torch.empty(M, c["k"], device=DEV),
                workspace=torch.zeros(1 << 20, dtype=torch.uint8, device=DEV))


def _quantized(w):
    """MXFP4 codes and scales of w [..., K]: the scale puts a block's largest value into [4, 8), elements go to
    the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6, ties to the even code."""
    blocks = w.unflatten(-1, (-1, 32))
    code = (torch.frexp(blocks.abs().amax(-1)).exponent - 3 + 127).clamp(0, 254)
    t = torch.ldexp(blocks, (127 - code)[..., None]).abs()
    up = (t > 0.25).to(torch.uint8) + (t >= 0.75) + (t > 1.25) + (t >= 1.75) + (t > 2.5) + (t >= 3.5) + (t > 5)
    up = (up + 8 * (blocks < 0)).to(torch.uint8).flatten(-2)
    return up[..., 0::2] | (up[..., 1::2] << 4), code.to(torch.uint8)


def _packed(codes, scales):
    """include/prq.h's layout of [E, N, K / 2] codes and [E, N, K / 32] scales."""
    E, N, half = codes.shape
    steps = (half + 63) // 64
    codes = torch.nn.functional.pad(codes, (0, steps * 64 - half)).view(E, N // 16, 16, steps, 4, 16)
    groups = (steps + 3) // 4
    scales = torch.nn.functional.pad(scales, (0, groups * 16 - scales.shape[2]), value=127).view(E, N // 16, 16, groups, 4, 4)
    return codes.permute(0, 1, 3, 4, 2, 5).contiguous().view(-1), scales.permute(0, 1, 3, 5, 2, 4).contiguous().view(-1)


def _prepare_experts(c, seed):
    g = _gen(seed, 3)
    M, E, k, H, I, tail = c["M"], c["E"], c["k"], c["H"], c["I"], c["tail"]
    gate_up = _quantized(_randn(g, E, 2 * I, H) / math.sqrt(H))
    down = _quantized(_randn(g, E, H, I + tail) * torch.where(torch.arange(I + tail, device=DEV) < I, 1.0, 0.1) / math.sqrt(I))
    x = _randn(g, M, H)
    # some experts are asked for more often than others
    score = _randn(g, M, E) + 0.5 * _randn(g, E)
    top = torch.topk(score, k, dim=1)
    return dict(case=c, x=x.bfloat16(), ids=top.indices.to(torch.int32), weights=torch.softmax(top.values, 1),
                gate_up=gate_up, down=down, gate_up_packed=_packed(*gate_up), down_packed=_packed(*down),
                out=torch.empty(M, H, dtype=torch.bfloat16, device=DEV),
                workspace=torch.zeros(64 << 20, dtype=torch.uint8, device=DEV))


def prepare(case, seed):
    return {"norm": _prepare_norm, "route": _prepare_route, "experts": _prepare_experts}[case["op"]](case, seed)


# -------------------------------------------------------------- plain forms ---
def _normed(x, w):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()


def _norm_plain(s):
    c = s["case"]
    u = s["y"].float()
    if s["post"] is not None:
        u = _normed(u, s["post"])
    if s["gate"] is not None:
        u = u * (s["gate"].float() if s["index"] is None else s["gate"].float()[s["index"].long()])
    r = c["a"] * s["r"].float() + c["b"] * u
    return r.to(s["r"].dtype), _normed(r, s["pre"]).bfloat16()


def _route_plain(s):
    c = s["case"]
    logits = torch.matmul(s["x"].float(), s["w"].float().t())
    if c["sigmoid"]:                                # selected with the correction: 64 bits, next to a border
        score = 1.0 / (1.0 + torch.exp(-logits.double()))
        key = score + s["bias"].double()
    else:
        score = torch.exp(logits - logits.amax(1, keepdim=True))
        key = logits
    ids = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :c["k"]]
    w = torch.gather(score, 1, ids)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    elif not c["sigmoid"]:
        w = w / score.sum(1, keepdim=True)
    return ids.to(torch.int32), w.float()


def _values(codes, scales):
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    v = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).flatten(-2)
    return (v.unflatten(-1, (-1, 32)) * torch.exp2(scales.float() - 127)[..., None]).flatten(-2)


def _experts_plain(s):
    c = s["case"]
    M, E, k, H, I, tail = c["M"], c["E"], c["k"], c["H"], c["I"], c["tail"]
    ids, x = s["ids"].long(), s["x"].float()
    if M * k <= E:                                  # the experts of every pair of a token and an expert
        which = ids.flatten()
        x = x.repeat_interleave(k, 0)[:, None]                                     # [pairs, 1, H]
        gate_up, down = (_values(q[which], sc[which]) for q, sc in (s["gate_up"], s["down"]))
    else:                                           # all experts for all tokens
        gate_up, down = _values(*s["gate_up"]), _values(*s["down"])
        x = x[None].expand(E, M, H)
    y = torch.matmul(x, gate_up.transpose(1, 2))
    h = y[..., :I] / (1.0 + torch.exp(-y[..., :I])) * y[..., I:]
    h = torch.cat([h, h[..., I - tail:]], -1) if tail else h
    y = torch.matmul(h, down.transpose(1, 2))
    if M * k <= E:
        return (y.view(M, k, H) * s["weights"][..., None]).sum(1).bfloat16()
    share = torch.where(ids[None] == torch.arange(E, device=DEV)[:, None, None], s["weights"][None], 0.0).sum(2)
    return (y * share[..., None]).sum(0).bfloat16()


# ------------------------------------------------------------------ one pass ---
def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if not own:
        return {"norm": _norm_plain, "route": _route_plain, "experts": _experts_plain}[op](s)
    from paper_2609_22106_amd import prq
    if op == "norm":
        h, r = prq.prq_block_norm(s["y"], s["r"], s["pre"], post_weight=s["post"], gate=s["gate"], gate_index=s["index"],
                                  eps=EPS, residual_scale=c["a"], block_scale=c["b"], out=s["h"], residual_out=s["r_out"])
        return r, h
    if op == "route":
        return prq.prq_moe_route(s["x"], s["w"], c["k"], scoring="sigmoid" if c["sigmoid"] else "softmax", bias=s["bias"],
                                 renormalize=c["renorm"], ids=s["ids"], weights=s["weights"], workspace=s["workspace"])
    gate_up = prq.PackedWeight(*s["gate_up_packed"], c["E"], 2 * c["I"], c["H"])
    down = prq.PackedWeight(*s["down_packed"], c["E"], c["H"], c["I"] + c["tail"])
    return prq.prq_moe_layer(s["x"], s["ids"], s["weights"], gate_up, down, k_tail=c["tail"], out=s["out"],
                             workspace=s["workspace"])


def _used(c):
    """Experts that a batch reaches when each token takes k of E at random, at least."""
    return min(c["E"], max(c["k"], round(c["E"] * (1 - (1 - c["k"] / c["E"]) ** c["M"]) * 0.9)))


def work(case):
    c, M, H = case, case["M"], case["H"]
    if c["op"] == "norm":
        each = (4 if c["y32"] else 2) + 2 * (4 if c["r32"] else 2) + 2
        return {"bytes": M * H * each + 2 * H * (1 + c["post"] + c["gates"]) + (4 * M if c["gates"] > 1 else 0),
                "flops": M * H * (7 + 4 * c["post"] + (c["gates"] > 0))}
    E, k = c["E"], c["k"]
    if c["op"] == "route":
        return {"bytes": 2 * H * (M + E) + 8 * M * k + (4 * E if c["sigmoid"] else 0), "flops": 2 * M * H * E}
    each = 2 * c["I"] * H + H * (c["I"] + c["tail"])
    return {"bytes": _used(c) * each * 17 // 32 + M * (4 * H + 8 * k), "flops": 2 * M * k * each}


# --------------------------------------------------------------- in 64 bits ---
def _exact_norm(s):
    c = s["case"]

    def norm(v, w):
        return v / torch.sqrt(v.pow(2).sum(-1, keepdim=True) / c["H"] + EPS) * w.double()

    u = s["y"].double()
    u = u if s["post"] is None else norm(u, s["post"])
    if s["gate"] is not None:
        row = torch.zeros(c["M"], dtype=torch.int64, device=DEV) if s["index"] is None else s["index"].long()
        u = u * torch.index_select(s["gate"].double(), 0, row)
    r = s["r"].double() * c["a"] + u * c["b"]
    return r, norm(r, s["pre"])


def _exact_route(s):
    c = s["case"]
    logits = s["x"].double() @ s["w"].double().t()
    score = torch.sigmoid(logits) if c["sigmoid"] else torch.softmax(logits, 1)
    key = (score + s["bias"].double() if c["sigmoid"] else logits).clone()
    rows = torch.arange(c["M"], device=DEV)
    ids = []
    for _ in range(c["k"]):                         # the largest that is left, the lowest index among equals
        best = (key == key.amax(1, keepdim=True)).to(torch.int8).argmax(1)
        key[rows, best] = -math.inf
        ids.append(best)
    ids = torch.stack(ids, 1)
    w = score[rows[:, None], ids]
    return ids, w / w.sum(1, keepdim=True) if c["renorm"] else w


def _exact_values(codes, scales):
    n = torch.stack([codes % 16, codes // 16], -1).flatten(-2).double()
    sign, n = 1 - 2 * (n >= 8).double(), n % 8
    size = torch.where(n < 2, n / 2, (1 + n % 2 / 2) * torch.pow(2.0, torch.floor(n / 2) - 1))
    return sign * size * torch.pow(2.0, scales.double() - 127).repeat_interleave(32, -1)


def _exact_experts(s):
    c = s["case"]
    I, tail = c["I"], c["tail"]
    y = torch.zeros(c["M"], c["H"], dtype=torch.float64, device=DEV)
    for e in sorted(set(s["ids"].flatten().tolist())):
        token, slot = torch.nonzero(s["ids"] == e, as_tuple=True)
        both = s["x"][token].double() @ _exact_values(s["gate_up"][0][e], s["gate_up"][1][e]).t()
        h = torch.nn.functional.silu(both[:, :I]) * both[:, I:]
        w = _exact_values(s["down"][0][e], s["down"][1][e])
        out = h @ w[:, :I].t() + h[:, I - tail:] @ w[:, I:].t()
        y.index_add_(0, token, out * s["weights"][token, slot].double()[:, None])
    return y


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "route": _exact_route, "experts": _exact_experts}[case["op"]](s)
