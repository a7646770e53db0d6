"""Which kernels the calls of a mixture-of-experts half layer take at given sizes (the library's own rules, by
way of libprq_probe.so; no GPU)."""
import ctypes

CUS = 256                                                     # of an MI355X


def _plan(name, n, *sizes):
    from paper_2609_22106_amd import build, prq               # noqa: F401  (prq loads torch first)
    out = (ctypes.c_int32 * n)()
    assert getattr(ctypes.CDLL(build.PROBE_LIB), name)(*sizes, out) == 0
    return tuple(out)


def norm(M, H, y_bf16, r_bf16, residual=True, h=True):
    """Lanes a row, quadruples a lane, past the last cache."""
    return _plan("prq_probe_norm_plan", 3, M, H, int(y_bf16), int(r_bf16), int(residual), int(h))


def route(M, E, H):
    """Groups of 32 experts a workgroup (0: 16 tokens and 16 experts), groups of a block apart."""
    return _plan("prq_probe_route_plan", 2, M, E, H, CUS)


def layer(M, k, E, H, I, k_tail, N):
    """Slots, by expert, waves a tile, tiles a workgroup, workgroups along the experts, tokens an item."""
    return _plan("prq_probe_layer_plan", 6, M, k, E, H, I, k_tail, N, CUS)
