"""The group norm's plans on the host (no GPU): every shape gets one, and it
covers the shape."""
import pytest

from tests._norm_paths import TYPES, backward_cases, forward_cases
from tests._plans import compiled, plans


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return compiled(str(tmp_path_factory.mktemp("plan")))



GROUPS = [(C, G) for C in [1, 2, 3, 5, 7, 8, 9, 12, 16, 24, 33, 40, 56, 64, 72, 96, 120, 132, 256, 264, 512, 1000, 1024, 2048, 2600]
          for G in range(1, C + 1) if C % G == 0]


@pytest.mark.parametrize("tx,ty", TYPES)
@pytest.mark.parametrize("backward", [False, True])
def test_every_shape_has_a_plan_that_covers_it(program, tx, ty, backward):
    """Groups of one channel and more, with every width of a vector."""
    shapes = [(B, P, C, G, C + extra, 0, tx, ty, backward) for C, G in GROUPS for extra in (0, 1, 8)
              for B, P in ((1, 1), (2, 64), (300, 100), (200, 2000), (1, 70001))]
    most = {1: 32, 4: 8, 8: 8}                              # pixels a thread holds in registers
    for (B, P, C, G, *_), p in zip(shapes, plans(program, shapes)):
        if p.way == "stream":
            continue
        what = (B, P, C, G, p)
        assert p.L * p.V * p.slabs == C and p.groups * (C // G) == p.L * p.V, what
        assert 1 <= p.L * p.rows <= 256 and 1 <= p.cluster <= 8 and p.cluster * p.ppc >= P, what
        assert p.smem <= 100 * 1024 and (p.V > 1 or p.smem == 0), what
        if not backward:
            assert p.per == C // G // (p.V // p.GPT) >= 1 and p.GPT in (1, 2, 4), what
        if p.way == "held":
            assert p.cluster == 1 and P <= p.rows * most[p.V], what
        if p.way == "shared":
            assert -(-p.ppc // p.rows) * 256 * p.V * (4 if tx == "f" else 2) <= p.smem, what


def test_chunks_only_in_the_forward(program):
    assert plans(program, [(2, 252003, 96, 8, 160, 0, "b", "b", False)])[0].way == "chunks"
    assert plans(program, [(2, 252003, 96, 8, 160, 0, "b", "b", True)])[0].way == "stream"


def test_the_shapes_of_the_gpu_tests_take_the_kernels_they_name(program):
    """A rule tuned anew may not leave a kernel without a case."""
    fwd, bwd = forward_cases(), backward_cases()
    for (case, way, V, GPT), p in zip(fwd, plans(program, [(*c[0][:8], False) for c in fwd])):
        assert (p.way, p.V) == (way.split("_")[0], V) and GPT in (None, p.GPT), (case, p)
        assert way not in ("reread", "reread_cluster") or (p.cluster > 1) == (way == "reread_cluster"), (case, p)
    for (case, way, V), p in zip(bwd, plans(program, [(*c[0][:8], True) for c in bwd])):
        assert (p.way, p.V) == (way.split("_")[0], V), (case, p)
        assert way not in ("reread", "reread_cluster") or (p.cluster > 1) == (way == "reread_cluster"), (case, p)


@pytest.mark.parametrize("backward", [False, True])
def test_no_kernel_is_left_out(program, backward):
    """Whatever plans the shapes of these tests get, a GPU case has each combination of kernel, vector, groups among its
    channels and types."""
    named = {(c[0][6], c[0][7], c[1].split("_")[0], *c[2:]) for c in (backward_cases() if backward else forward_cases())}
    named = {n[:4] + (None,) if n[2] == "stream" or backward else n for n in named}
    for tx, ty in TYPES:
        shapes = [(B, P, C, G, C, 0, tx, ty, backward) for C, G in GROUPS for B, P in ((1, 1), (300, 100), (700, 300), (2, 30000))]
        for s, p in zip(shapes, plans(program, shapes)):
            if p.way == "stream":
                assert any(n[2] == "stream" and n[3] == p.V for n in named), (s, p)
            else:
                assert (tx, ty, p.way, p.V, None if backward else p.GPT) in named, (s, p)
