"""The packed join at the widest rows of values one by one, whose heads meet in shared memory: every shape that the forward takes, the reverse pass takes."""
import pytest

from oracle import join as O
from tests import test_gpu_join as J
from tests import test_gpu_join_packed as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 2730, 2, 3), (1, 2673, 2, 3), (1, 1170, 3, 7), (1, 1638, 2, 5), (1, 8191, 2, 1)])
def test_widest_rows(io, shape):
    x, d = J._make(*shape, io, "silu", True, seed=3)
    r = P.Run(x, io, "silu")
    xo, n = O.forward(**x, kind="silu", **J.EPS)
    J.check(r.fwd(), {"x_out": xo, "n": n})
    J.check(r.bwd(d), O.backward(**P.kept(x), kind="silu", **J.EPS, **d, terms=True))
