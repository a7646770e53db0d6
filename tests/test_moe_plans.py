"""The kernels that the calls of a mixture-of-experts half layer take, by size (no GPU): every kernel that
is built is one that a call takes."""
import re
import shutil
import subprocess

import pytest

from tests import moe_plans


def _built(kernel):
    """Template arguments of every instance of a kernel in the library."""
    from paper_2609_22106_amd import build
    if not shutil.which("nm"):
        pytest.skip("no nm")
    names = subprocess.run(["nm", "-C", build.LIB], capture_output=True, text=True, check=True).stdout
    found = re.findall(r"__device_stub__" + kernel + r"<([^>]*)>\(", names)
    assert found and len(found) == len(set(found))
    return {tuple(s.strip() for s in f.split(",")) for f in found}


def _text(*values):
    return tuple(str(v).lower() if isinstance(v, bool) else str(v) for v in values)


def test_every_norm_kernel_is_taken():
    taken = set()
    rows = [1, 7, 1023, 1024, 1 << 14, 1 << 17, 1 << 20, (1 << 24) - 1]
    for H in [8, 256, 264, 512, 520, 1024, 1032, 1536, 1544, 2048, 2056, 2560, 3080, 4096, 4104, 8192, 8200, 16384]:
        for M in rows:
            for y in (False, True):
                for r in (False, True):
                    lanes, quads, once = moe_plans.norm(M, H, y, r)
                    assert lanes * quads * 4 >= H and (quads == 1 or quads > 4 or lanes * (quads - 1) * 4 < H)
                    kind = ("float", "unsigned short")
                    taken.add(_text(kind[y], kind[r], lanes, quads, bool(once)))
    assert _built("block_norm_kernel") == taken


def test_norm_sizes_reach_the_forms_that_they_name():
    cases = moe_plans.NORM_FORMS + moe_plans.NORM_PAST_THE_CACHE
    for M, H, y, r, plan in cases:
        assert moe_plans.norm(M, H, y, r) == plan, (M, H)
    reached = {plan for *_, plan in cases}
    for H in range(8, 16385, 40):
        for M in (1, 1023, 1024, 1 << 20):
            assert moe_plans.norm(M, H, 0, 0) in reached, (M, H)


def test_every_router_kernel_is_taken_and_the_sizes_reach_them():
    reached = set()
    for M, E, k, H, plan in moe_plans.ROUTE_FORMS:
        assert moe_plans.route(M, E, H) == plan, (M, E)
        reached.add(plan)
    assert reached == {moe_plans.route(M, E, H) for M, E in moe_plans.ROUTE_KINDS for H in (8, 64)}
    assert reached == {moe_plans.route(M, E, 64) for E in range(1, 1025, 3)
                       for M in (1, 100, 1000, 2000, 3000, 5000, 10000, 1 << 20)}
    for bias in (False, True):
        assert {f for f in _built("route_many_kernel") if f[1] == _text(bias)[0]} == \
            {_text(groups, bias, bool(split)) for groups, split in reached if groups}
    assert _built("route_few_kernel") == {("false",), ("true",)}


def test_every_kernel_of_the_experts_is_taken_and_the_sizes_reach_them():
    up, down = set(), set()
    for M, E, k, H, I, tail, N, plan in moe_plans.LAYER_FORMS + moe_plans.LAYER_WINDOWS:
        slots, by_expert, parts, tiles, splits, item = moe_plans.layer(M, k, E, H, I, tail, N)
        assert (by_expert, parts, tiles, splits, item) == plan, (M, E)
        assert slots == min(E, M * k) and by_expert == (slots == E)
        up.add((parts, M > 16, H > 1024))
        down.add((tiles, item, splits > 1))
    assert up >= {(parts, many, True) for parts in (1, 2, 4) for many in (False, True)}
    assert down >= {(tiles, item, True) for tiles in (1, 2) for item in (8, 16)}
    assert {int(f[1]) for f in _built("moe_up_kernel")} == {parts for parts, *_ in up}
    assert {(int(f[0]), 8 if f[3] == "true" else 16) for f in _built("moe_down_kernel")} == {d[:2] for d in down}
    # the experts that random choices name, an item each at least, over the workgroups along them
    for M, E, k, H, I, tail, N, (*_, splits, _) in moe_plans.LAYER_WINDOWS:
        assert 0.8 * E * (1 - (1 - k / E) ** M) / splits > 64, (M, E)
