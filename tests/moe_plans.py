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


# (rows, width, y in bf16, residual in bf16) and the plan: every form, at the ends of its range.
NORM_FORMS = [
    (61, 1024, 0, 1, (256, 1, 0)), (5, 520, 1, 0, (256, 1, 0)), (1023, 1016, 0, 0, (256, 1, 0)), (2, 1000, 1, 1, (256, 1, 0)),
    (7, 4096, 1, 1, (256, 4, 0)), (900, 3080, 0, 0, (256, 4, 0)), (3, 3584, 1, 0, (256, 4, 0)), (1100, 4088, 0, 1, (256, 4, 0)),
    (9, 1032, 0, 0, (256, 2, 0)), (1030, 2048, 1, 0, (256, 2, 0)), (4, 8192, 0, 1, (256, 8, 0)), (3, 8200, 1, 1, (256, 16, 0)),
    (1024, 1032, 0, 0, (128, 3, 0)), (1025, 1024, 1, 1, (128, 2, 0)), (6, 512, 1, 0, (64, 2, 0)), (4097, 264, 0, 1, (64, 2, 0)),
    (3, 256, 0, 1, (64, 1, 0)), (4099, 8, 1, 0, (64, 1, 0)), (5, 2056, 1, 1, (256, 3, 0)), (1027, 2560, 0, 0, (256, 3, 0))]
# The same of what is more than the last cache holds.
NORM_PAST_THE_CACHE = [
    (80001, 256, 0, 0, (64, 1, 1)), (60003, 504, 0, 1, (64, 2, 1)), (30001, 1024, 0, 0, (128, 2, 1)),
    (20003, 1056, 0, 0, (128, 3, 1)), (18001, 2048, 1, 1, (256, 2, 1)), (8192, 2560, 0, 0, (256, 3, 1)),
    (6003, 4096, 1, 0, (256, 4, 1)), (2801, 8192, 0, 0, (256, 8, 1)), (2003, 16384, 0, 1, (256, 16, 1))]

# (tokens, experts, chosen, width) of the router and the plan: last blocks of 32 with few tokens and with many, widths
# within a chunk of H, at its end and past it.
ROUTE_FORMS = [
    (8200, 16, 4, 40, (1, 0)), (4200, 32, 32, 24, (1, 0)), (4129, 20, 3, 1056, (1, 0)), (8193, 1, 1, 520, (1, 0)),
    (2800, 40, 5, 328, (2, 0)), (2053, 60, 4, 136, (2, 0)), (2080, 64, 6, 1032, (2, 0)), (2753, 33, 32, 256, (2, 0)),
    (1700, 70, 5, 72, (4, 0)), (1400, 96, 8, 264, (4, 0)), (1029, 128, 8, 520, (4, 0)), (1900, 130, 7, 64, (4, 0)),
    (1029, 250, 8, 1024, (4, 0)), (1100, 256, 32, 40, (4, 0)), (5470, 300, 4, 16, (4, 0)), (4100, 512, 3, 24, (4, 0)),
    (1000, 300, 8, 136, (4, 1)), (1033, 512, 16, 2056, (4, 1)), (900, 400, 4, 8, (4, 1)), (1025, 257, 2, 640, (4, 1)),
    (1, 128, 8, 2048, (0, 0)), (61, 64, 6, 264, (0, 0)), (1100, 16, 4, 72, (0, 0)), (1100, 1000, 9, 72, (0, 0))]
# One of each for the inputs that are the same in all of them.
ROUTE_KINDS = [(8200, 16), (2800, 40), (1400, 96), (1029, 250), (4100, 512), (1000, 300), (40, 300)]

# (tokens, experts, experts a token, hidden, intermediate, tail, output width) of the experts' call and of the plan: by
# expert, waves a tile, tiles a workgroup, workgroups along the experts, tokens an item.
LAYER_FORMS = [
    # two waves a tile: up to 16 tokens, more than 16 of an expert over several pieces of H, wide
    (12, 128, 8, 1184, 256, 32, 32, (0, 2, 2, 8, 8)), (64, 8, 4, 2144, 1024, 0, 64, (1, 2, 2, 5, 16)),
    (20, 2, 2, 1056, 4096, 0, 32, (1, 2, 2, 5, 16)), (64, 8, 4, 1056, 1024, 32, 48, (1, 2, 1, 6, 16)),
    # one: the same
    (16, 64, 6, 1056, 1408, 0, 48, (1, 1, 1, 8, 8)), (64, 12, 4, 544, 1408, 64, 48, (1, 1, 1, 8, 16)),
    (64, 8, 4, 1184, 2816, 0, 32, (1, 1, 2, 8, 16)), (33, 512, 2, 160, 352, 64, 64, (0, 1, 2, 8, 8)),
    (64, 130, 2, 96, 544, 32, 48, (0, 1, 1, 8, 8)),
    # four: the same
    (9, 16, 4, 2080, 96, 32, 64, (1, 4, 2, 1, 8)), (20, 16, 4, 2080, 96, 32, 48, (1, 4, 1, 1, 16)),
    (64, 3, 2, 2112, 64, 0, 96, (1, 4, 2, 1, 16)), (8, 3, 2, 1056, 1408, 0, 64, (1, 4, 2, 2, 8)),
    # more workgroups than CUs of the second launch, an output of odd tiles
    (64, 4, 1, 32, 96, 96, 8224, (1, 4, 2, 1, 16)), (40, 16, 5, 544, 160, 0, 8208, (1, 4, 1, 1, 16))]
# More than 64 items to a workgroup of the second launch.
LAYER_WINDOWS = [
    (64, 256, 8, 64, 32, 0, 7168, (1, 2, 2, 1, 8)), (64, 300, 8, 32, 32, 32, 4112, (1, 2, 1, 1, 8)),
    (64, 400, 32, 32, 32, 0, 4112, (1, 2, 1, 1, 16)), (64, 200, 30, 64, 32, 0, 7200, (1, 2, 2, 1, 16)),
    (64, 4096, 32, 64, 32, 0, 16, (0, 1, 1, 8, 8))]
