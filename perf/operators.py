"""Performance cases of the attention block's operators around the MXFP4 linears on one MI355X.

Three operators, each through the public calls of ``paper_2609_22106_amd.prq``:

* ``rope``: ``prq_qk_norm_rope`` -- RMS norm of every query and key head, rotation by position,
  bf16 queries out, keys and values into the paged cache;
* ``attend``: ``prq_tree_attention`` -- the tokens of each request (one, or a tree of drafted
  ones) over that request's pages of the cache;
* ``adapt``: ``prq_lora`` -- the low-rank adapters of many requests beside a shared projection.

``run`` computes the plain form, elementary torch operations in 32 bits, or with ``own`` set the
calls above.  Layouts:

* projections (q, k, v, Y) row-major [M, features], float32 as the GEMM writes them, or bf16;
* ``table`` float32 [positions, rot / 2, 2]: cosine and sine of every position and pair;
* cache: K and V bf16 [pages, kv heads, page size, D]; a slot is page * page size + offset;
* adapters: A bf16 [sum of ranks, K] (adapter a's rows from ``rank_offsets[a]``), B bf16 flat,
  adapter a's [N, rank] from element N * ``rank_offsets[a]``; rows sorted by segment.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
THETA = 1e6
WORKSPACE = 128 << 20                         # what a serving loop keeps for the attention's partial sums
# (query heads, kv heads, head size): the q and k/v projections this repository benchmarks (4096 and
# 1024 wide), and generic others: three query heads a key head, one key head, one query head a key head
HEADS = ((32, 8, 128), (24, 8, 64), (16, 4, 128), (8, 1, 128), (12, 12, 64))
# (out features, in features) of the decoder linears, and a generic odd pair
LINEARS = ((4096, 2560), (1024, 2560), (2560, 4096), (9728, 2560), (2560, 9728), (1936, 5216))


def listed():
    return [
        # one sequence decoding: one token's 32 + 8 + 8 heads after the projections
        dict(name="rope 1 row", op="rope", M=1, Hq=32, Hk=8, D=128, rot=128, inter=False, norm=True, bf16=False, page=64),
        # an odd batch decoding, each row into a page of its own request
        dict(name="rope 61 rows", op="rope", M=61, Hq=32, Hk=8, D=128, rot=128, inter=False, norm=True, bf16=False, page=16),
        # a ragged prompt through narrow heads: interleaved pairs, half of the head rotated, bf16 projections
        dict(name="rope ragged 1537 rows", op="rope", M=1537, Hq=24, Hk=8, D=64, rot=32, inter=True, norm=True, bf16=True, page=32),
        # a long prompt
        dict(name="rope 8192 rows", op="rope", M=8192, Hq=32, Hk=8, D=128, rot=128, inter=False, norm=True, bf16=False, page=64),
        # one sequence decoding over 4 k tokens: few rows, one long axis
        dict(name="attend 1 token over 4097", op="attend", B=1, nodes=1, kv=4097, Hq=32, Hk=8, D=128, page=64),
        # a batch of 32 sequences decoding after prompts of up to 2 k tokens
        dict(name="attend 32 sequences", op="attend", B=32, nodes=1, kv=2176, Hq=32, Hk=8, D=128, page=64),
        # six requests verifying trees of up to 13 drafted tokens, three query heads a key head
        dict(name="attend trees of 13", op="attend", B=6, nodes=13, kv=8211, Hq=24, Hk=8, D=64, page=16),
        # long contexts with wide trees: the largest
        dict(name="attend trees of 64 long", op="attend", B=8, nodes=64, kv=32768, Hq=32, Hk=8, D=128, page=64),
        # one request's adapter beside the q projection of one token
        dict(name="adapt 1 row", op="adapt", M=1, N=4096, K=2560, segments=1, adapters=8, rank=16),
        # 64 requests decoding, 24 adapters of ranks up to 64, beside the down-projection
        dict(name="adapt 64 requests", op="adapt", M=64, N=2560, K=9728, segments=64, adapters=24, rank=64),
        # five ragged prompts beside the k projection
        dict(name="adapt 5 prompts 1537 rows", op="adapt", M=1537, N=1024, K=2560, segments=5, adapters=8, rank=32),
        # four long prompts beside the widest projection: the output is most of the bytes
        dict(name="adapt 4 prompts 8192 rows", op="adapt", M=8192, N=9728, K=2560, segments=4, adapters=8, rank=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rope", "attend", "adapt"))
    Hq, Hk, D = rng.choice(HEADS)
    page = rng.choice((16, 32, 64, 128))
    if op == "rope":
        return dict(op=op, M=_log_int(rng, 1, 8192), Hq=Hq, Hk=Hk, D=D, rot=rng.choice((D, D, D // 2)),
                    inter=rng.random() < 0.3, norm=rng.random() < 0.8, bf16=rng.random() < 0.3, page=page)
    if op == "attend":
        B = _log_int(rng, 1, 64)
        nodes = _log_int(rng, 1, 64)
        return dict(op=op, B=B, nodes=nodes, kv=_log_int(rng, 64, min(32768, (8 << 15) // B)), Hq=Hq, Hk=Hk, D=D,
                    page=page)
    N, K = rng.choice(LINEARS)
    M = _log_int(rng, 1, min(8192, 8192 * 9728 // N))
    segments = _log_int(rng, 1, min(M, 64))
    adapters = _log_int(rng, 1, 32)
    return dict(op=op, M=M, N=N, K=K, segments=segments, adapters=adapters, rank=rng.choice((8, 16, 32, 64)))


# ------------------------------------------------------------------- inputs ---
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * seed + stream)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _positions(c):
    """Rows of a table that holds every position of the case: a prompt starts at 0, a decode batch is spread."""
    return max(4096, c["M"])


def _row_positions(c, r):
    n = _positions(c)
    return [r.randrange(n) for _ in range(c["M"])] if c["M"] <= 64 else list(range(c["M"]))


def _lengths(c):
    """Drafted tokens and cached tokens of every request: the first one full, the others ragged, from the case alone."""
    r = random.Random(7919 * c["B"] + 31 * c["nodes"] + c["kv"])
    n = [c["nodes"]] + [r.randint((c["nodes"] + 1) // 2, c["nodes"]) for _ in range(c["B"] - 1)]
    kv = [c["kv"]] + [r.randint((c["kv"] + 1) // 2, c["kv"]) for _ in range(c["B"] - 1)]
    return n, [max(0, L - m) for L, m in zip(kv, n)]


def _segments(c):
    """Offsets of the rows' segments, the adapter of each (one in nine has none) and every adapter's rank."""
    r = random.Random(104729 * c["M"] + 17 * c["segments"] + c["rank"])
    cuts = sorted(r.sample(range(1, c["M"]), c["segments"] - 1)) if c["segments"] > 1 else []
    of = [-1 if i % 9 == 8 else r.randrange(c["adapters"]) for i in range(c["segments"])]
    ranks = [c["rank"] if a % 2 == 0 else max(8, c["rank"] // (2 << (a % 3))) for a in range(c["adapters"])]
    return [0] + cuts + [c["M"]], of, ranks


def _prepare_rope(c, seed):
    g, r = _gen(seed, 1), random.Random(seed)
    M, Hq, Hk, D, rot = c["M"], c["Hq"], c["Hk"], c["D"], c["rot"]
    dtype = torch.bfloat16 if c["bf16"] else torch.float32
    n = _positions(c)
    angle = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] * \
        THETA ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    pages = (M + c["page"] - 1) // c["page"] + 3 if M > 64 else M + 3
    order = list(range(pages))
    r.shuffle(order)
    if M > 64:                                     # a prompt fills its pages in order
        slots = [order[i // c["page"]] * c["page"] + i % c["page"] for i in range(M)]
    else:                                          # a decoding row goes into its own request's page
        slots = [order[i] * c["page"] + r.randrange(c["page"]) for i in range(M)]
    return dict(case=c, q=(1.5 * _randn(g, M, Hq * D)).to(dtype), k=(1.5 * _randn(g, M, Hk * D)).to(dtype),
                v=_randn(g, M, Hk * D).to(dtype),
                wq=(1 + 0.2 * _randn(g, D)).bfloat16() if c["norm"] else None,
                wk=(1 + 0.2 * _randn(g, D)).bfloat16() if c["norm"] else None,
                table=torch.stack([torch.cos(angle), torch.sin(angle)], -1).float(),
                pos=_int32(_row_positions(c, r)), slots=torch.tensor(slots, dtype=torch.int64, device=DEV),
                K=_randn(g, pages, Hk, c["page"], D).bfloat16(), V=_randn(g, pages, Hk, c["page"], D).bfloat16())


def _tree(r, n):
    """[n, n]: node i sees itself and its ancestors; a node's parent is an earlier one, or the last cached token."""
    see = np.zeros((n, n), dtype=bool)
    for i in range(n):
        parent = r.randrange(-1, i) if r.random() < 0.5 else i - 1
        if parent >= 0:
            see[i] = see[parent]
        see[i, i] = True
    return see


def _prepare_attend(c, seed):
    g, r = _gen(seed, 2), random.Random(seed)
    B, Hq, Hk, D, page = c["B"], c["Hq"], c["Hk"], c["D"], c["page"]
    n, cached = _lengths(c)
    M = sum(n)
    width = (c["kv"] + page - 1) // page
    used = [(a + b + page - 1) // page for a, b in zip(n, cached)]
    order = list(range(sum(used) + 3))
    r.shuffle(order)
    pages, at = np.zeros((B, width), np.int32), 0
    for b in range(B):
        pages[b, :used[b]] = order[at:at + used[b]]
        at += used[b]
    see = np.zeros((M, c["nodes"]), dtype=bool)
    row = 0
    for b in range(B):
        see[row:row + n[b], :n[b]] = _tree(r, n[b])
        row += n[b]
    K = _randn(g, len(order), Hk, page, D)
    return dict(case=c, q=(2 * _randn(g, M, Hq, D)).bfloat16(), K=K.bfloat16(),
                V=_randn(g, len(order), Hk, page, D).bfloat16(), pages=torch.from_numpy(pages).to(DEV),
                cached=_int32(cached), offsets=_int32(np.concatenate([[0], np.cumsum(n)]).tolist()),
                see=torch.from_numpy(see).to(DEV), scale=1.0 / math.sqrt(D),
                out=torch.empty(M, Hq, D, dtype=torch.bfloat16, device=DEV), lse=torch.empty(M, Hq, device=DEV),
                workspace=torch.zeros(WORKSPACE, dtype=torch.uint8, device=DEV))


def _prepare_adapt(c, seed):
    g = _gen(seed, 3)
    M, N, K = c["M"], c["N"], c["K"]
    offsets, of, ranks = _segments(c)
    R = sum(ranks)
    x = _randn(g, M, K)
    x[:, torch.randperm(K, generator=g, device=DEV)[:max(1, K // 200)]] *= 30.0     # outlier channels
    return dict(case=c, x=x.bfloat16(), A=(0.02 * _randn(g, R, K)).bfloat16(), B=(0.02 * _randn(g, N * R)).bfloat16(),
                rank_offsets=_int32([0] + list(np.cumsum(ranks).tolist())), max_rank=max(ranks),
                scales=0.5 + torch.rand(c["adapters"], generator=g, device=DEV),
                offsets=_int32(offsets), of=_int32(of), Y=_randn(g, M, N), out=torch.empty(M, N, device=DEV))


def prepare(case, seed):
    return {"rope": _prepare_rope, "attend": _prepare_attend, "adapt": _prepare_adapt}[case["op"]](case, seed)


# -------------------------------------------------------------- plain forms ---
def _rotated(x, w, table, rot, inter):
    """x [M, H, D] float32, normed per head where w is given, then its first `rot` dims rotated."""
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    c, s = table[:, None, :, 0], table[:, None, :, 1]
    one, two = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    y1, y2 = one * c - two * s, two * c + one * s
    y = torch.stack([y1, y2], -1).flatten(-2) if inter else torch.cat([y1, y2], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _rope_plain(s):
    c = s["case"]
    M, D = c["M"], c["D"]
    table = s["table"][s["pos"].long()]
    q = _rotated(s["q"].float().view(M, c["Hq"], D), s["wq"], table, c["rot"], c["inter"]).bfloat16()
    k = _rotated(s["k"].float().view(M, c["Hk"], D), s["wk"], table, c["rot"], c["inter"]).bfloat16()
    page, at = s["slots"] // c["page"], s["slots"] % c["page"]
    s["K"][page, :, at] = k
    s["V"][page, :, at] = s["v"].float().view(M, c["Hk"], D).bfloat16()
    return q, s["K"], s["V"]


def _attend_plain(s):
    c = s["case"]
    B, Hq, Hk, D, page, T = c["B"], c["Hq"], c["Hk"], c["D"], c["page"], c["nodes"]
    G, M = Hq // Hk, s["q"].shape[0]
    pages, first = s["pages"].long(), s["offsets"][:-1].long()
    n, cached = s["offsets"][1:].long() - first, s["cached"].long()
    L = pages.shape[1] * page
    k = s["K"][pages].transpose(1, 2).reshape(B, Hk, L, D).float()
    v = s["V"][pages].transpose(1, 2).reshape(B, Hk, L, D).float()
    node = torch.arange(T, device=DEV)
    row = (first[:, None] + node).clamp(max=M - 1)                                        # [B, T]
    q = s["q"][row].float().view(B, T, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, T * G, D)
    drafted = torch.arange(L, device=DEV)[None] - cached[:, None]                         # [B, L]
    seen = torch.gather(s["see"][row], 2, drafted.clamp(0, T - 1)[:, None].expand(B, T, L))
    seen = (seen & (drafted >= 0)[:, None] & (drafted < n[:, None])[:, None]) | (drafted < 0)[:, None]
    seen = seen[:, None, :, None].expand(B, 1, T, G, L).reshape(B, 1, T * G, L)
    score = torch.where(seen, torch.matmul(q, k.transpose(2, 3)) * s["scale"], -math.inf)
    most = score.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(score - torch.where(most == -math.inf, 0.0, most)), 0.0)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    lse = (most + torch.log(total)).view(B, Hk, T, G).permute(0, 2, 1, 3).reshape(B, T, Hq)
    o = o.view(B, Hk, T, G, D).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D)
    rows = torch.arange(M, device=DEV)
    b = (rows[:, None] >= s["offsets"][1:]).sum(1)
    at = rows - first[b]
    return o[b, at].bfloat16(), lse[b, at]


def _adapt_plain(s):
    c = s["case"]
    M, N = c["M"], c["N"]
    off = s["rank_offsets"].long()
    R = s["A"].shape[0]
    col = torch.arange(R, device=DEV)
    adapter = (col[:, None] >= off[1:]).sum(1)                                            # of every rank row
    of_row = s["of"][(torch.arange(M, device=DEV)[:, None] >= s["offsets"][1:]).sum(1)]
    t = torch.matmul(s["x"].float(), s["A"].float().t()) * s["scales"][adapter]
    t = torch.where(of_row[:, None] == adapter, t, 0.0)
    rank = (off[1:] - off[:-1])[adapter]
    at = N * off[adapter] + torch.arange(N, device=DEV)[:, None] * rank + (col - off[adapter])
    return s["Y"] + torch.matmul(t, s["B"][at].float().t())


# ------------------------------------------------------------------ one pass ---
def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"rope": _rope_plain, "attend": _attend_plain, "adapt": _adapt_plain}[op](s)
    from paper_2609_22106_amd import prq
    if op == "rope":
        cache = prq.PagedKV(s["K"], s["V"])
        q = prq.prq_qk_norm_rope(s["q"], s["k"], s["v"], s["pos"], s["table"], cache, s["slots"], q_weight=s["wq"],
                                 k_weight=s["wk"], eps=EPS, interleaved=s["case"]["inter"])
        return q, s["K"], s["V"]
    if op == "attend":
        c = s["case"]
        return prq.prq_tree_attention(s["q"], prq.PagedKV(s["K"], s["V"]), s["pages"], s["cached"], s["offsets"],
                                      s["scale"], tree_mask=s["see"], max_kv_len=c["kv"], out=s["out"], lse=s["lse"],
                                      workspace=s["workspace"])
    adapters = prq.LoraAdapters(s["A"], s["B"], s["rank_offsets"], s["scales"], s["max_rank"])
    return prq.prq_lora(s["x"], adapters, s["offsets"], s["of"], s["Y"], out=s["out"])


def work(case):
    c = case
    if c["op"] == "rope":
        heads, e = c["Hq"] + 2 * c["Hk"], 2 if c["bf16"] else 4
        rows = min(c["M"], _positions(c))
        turned = c["M"] * (c["Hq"] + c["Hk"])
        return {"bytes": c["M"] * (heads * c["D"] * (e + 2) + 4 + 8) + rows * c["rot"] * 4 + (4 * c["D"] if c["norm"] else 0),
                "flops": turned * (3 * c["rot"] + (4 * c["D"] if c["norm"] else 0))}
    if c["op"] == "attend":
        n, cached = _lengths(c)
        M, keys = sum(n), sum(n) + sum(cached)
        pairs = sum(a * (b + 1) for a, b in zip(n, cached))      # a node sees the cached tokens and itself at least
        return {"bytes": keys * c["Hk"] * c["D"] * 4 + M * c["Hq"] * (c["D"] * 4 + 4) + M * c["nodes"] + 4 * keys // c["page"],
                "flops": 4 * c["D"] * c["Hq"] * pairs}
    offsets, of, ranks = _segments(c)
    M, N, K = c["M"], c["N"], c["K"]
    rows = [(b - a, i) for a, b, i in zip(offsets, offsets[1:], of) if i >= 0]
    used = sum(ranks[i] for i in {i for _, i in rows})
    return {"bytes": sum(m for m, _ in rows) * K * 2 + M * N * 8 + used * (K + N) * 2,
            "flops": 2 * (K + N) * sum(m * ranks[i] for m, i in rows)}


# --------------------------------------------------------------- in 64 bits ---
def _exact_rope(s):
    c = s["case"]
    M, D, rot = c["M"], c["D"], c["rot"]
    t = s["table"].double()[s["pos"].long()]
    turn = torch.complex(t[..., 0].contiguous(), t[..., 1].contiguous())[:, None]         # [M, 1, rot / 2]

    def head(x, w):
        x = x.double().reshape(M, -1, D)
        if w is not None:
            x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + EPS) * w.double()
        i = torch.arange(rot // 2, device=DEV)
        a, b = (2 * i, 2 * i + 1) if c["inter"] else (i, i + rot // 2)
        z = torch.complex(x[..., a].contiguous(), x[..., b].contiguous()) * turn
        y = x.clone()
        y[..., a], y[..., b] = z.real, z.imag
        return y

    K, V = s["K"].double(), s["V"].double()
    page, at = torch.div(s["slots"], c["page"], rounding_mode="floor"), s["slots"].remainder(c["page"])
    K[page, :, at] = head(s["k"], s["wk"])
    V[page, :, at] = s["v"].double().reshape(M, -1, D)
    return head(s["q"], s["wq"]), K, V


def _exact_attend(s):
    c = s["case"]
    G, D, page = c["Hq"] // c["Hk"], c["D"], c["page"]
    n, cached = _lengths(c)
    out, lse, row = [], [], 0
    for b in range(c["B"]):
        P, m = cached[b], n[b]
        keys = torch.arange(P + m, device=DEV)
        held = s["pages"][b].long()[keys // page]
        k, v = s["K"][held, :, keys % page].double(), s["V"][held, :, keys % page].double()     # [L, Hk, D]
        hide = torch.zeros(m, P + m, dtype=torch.float64, device=DEV)
        hide[:, P:] = torch.where(s["see"][row:row + m, :m], 0.0, -math.inf)
        os, ls = [], []
        for h in range(c["Hq"]):
            score = s["q"][row:row + m, h].double() @ k[:, h // G].t() * s["scale"] + hide
            os.append(torch.softmax(score, -1) @ v[:, h // G])
            ls.append(torch.logsumexp(score, -1))
        out.append(torch.stack(os, 1))
        lse.append(torch.stack(ls, 1))
        row += m
    return torch.cat(out), torch.cat(lse)


def _exact_adapt(s):
    c = s["case"]
    offsets, of, ranks = _segments(c)
    first = [sum(ranks[:a]) for a in range(len(ranks))]
    y = s["Y"].double()
    for lo, hi, a in zip(offsets, offsets[1:], of):
        if a < 0:
            continue
        A = s["A"][first[a]:first[a] + ranks[a]].double()
        B = s["B"][c["N"] * first[a]:c["N"] * (first[a] + ranks[a])].double().view(c["N"], ranks[a])
        y[lo:hi] += s["scales"][a].double() * (s["x"][lo:hi].double() @ A.t() @ B.t())
    return y


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "attend": _exact_attend, "adapt": _exact_adapt}[case["op"]](s)
