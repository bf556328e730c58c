"""Attention over a cache in 4 bits where the numbers are not a unit normal's: scores far from zero, values of very different sizes."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_kvq import Layer, _i32, _i64, _rows, api  # noqa: F401  (api is a fixture)

pytestmark = pytest.mark.gpu

SHAPES = [(1, 0), (8, 0), (10, 0), (4, 2), (24, 0), (40, 0), (20, 3)]      # 1, 8, 10, 12, 24, 40 and 80 rows


def _put(x, b, k=None, v=None, at=0):
    """Rows [n][H][d] (on the CPU, in 32 bits) into sequence b's slots from `at` on; ones where K or V is not given."""
    one = torch.ones((k if k is not None else v).shape)
    k, v = ((one if t is None else t).to(torch.bfloat16).cuda()[None, None] for t in (k, v))
    x.api.ss_kvq_write(k, v, x.cache, _i64([x.starts[b]]), _i32([at]), None, None, None, None)


def _normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("nodes,gamma", SHAPES)
def test_first_scores_far_below_zero(api, d, nodes, gamma):
    """Cached keys whose scores are some 200 below zero: the first that a row sees.  The keys behind the prefix are as far below in
    the first round, so that all weigh, and near zero in the second."""
    H, lens = 3, [1, 40, 700]
    x = Layer(api, 3, H, d, lens, [nodes] * 3, gamma, seed=5 + d)
    for b, n in enumerate(lens):
        _put(x, b, -(_normal((n, H, d), b).abs() * 0.2 + 10.0), _normal((n, H, d), 10 + b))
    for t in (x.q_main, x.q_spec):
        if t is not None:
            t.copy_((t.float().abs() * 0.1 + 20.0 * d ** -0.5).to(torch.bfloat16))
    for far in (True, False):
        for t in (x.k_tree, x.k_spec):
            if t is not None:
                t.copy_((t.float().abs() * 0.2 + 10.0 if far else t.float().abs() * 0.2) * -1.0)
        x.fresh()
        x.run()
        x.check()
