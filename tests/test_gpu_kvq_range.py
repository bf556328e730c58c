"""Attention over a cache in 4 bits where the numbers are not a unit normal's: scores far from zero, values of very different sizes."""
import pytest

torch = pytest.importorskip("torch")

import kvq_util as U
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


def _check_lse(x, b):
    """Log-sum-exps of sequence b, which do not depend on the values."""
    keys, _ = U.cache_values(x.cache, 0, "cuda")
    n, g, held = x.nodes[b], x.gamma, slice(x.starts[b], x.starts[b] + x.lens[b])
    spec = (lambda t: t[b, :n] if g else None)
    none = [torch.zeros_like(t) if t is not None else None for t in (keys[held], x.v_tree[b, :n], spec(x.v_spec))]
    _, lse, _, tol = U.attention(x.parents[b], g, x.scale, x.q_main[b, :n], spec(x.q_spec), keys[held], none[0], x.k_tree[b, :n], none[1],
                                 spec(x.k_spec), none[2])
    got = torch.cat([x.lse_main[b, :n].double()] + ([x.lse_spec[b, :n].double().flatten(0, 1)] if g else []))
    assert ((got - lse).abs() <= tol).all()


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


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("nodes,gamma", SHAPES)
def test_values_without_a_number_leave_the_log_sum_exps(api, d, nodes, gamma):
    """A sequence's cached values are all NaN (their keys are not): so are its outputs, while its log-sum-exps, of scores of some 200
    above or below zero, are numbers; another sequence's outputs are untouched by it."""
    H, lens = 3, [33, 600]
    for bad, sign in ((0, 1.0), (1, -1.0), (0, -1.0)):
        x = Layer(api, 2, H, d, lens, [nodes] * 2, gamma, seed=7 + d)
        _put(x, bad, sign * (_normal((lens[bad], H, d), 1).abs() * 0.2 + 10.0), torch.full((lens[bad], H, d), float("nan")))
        for t in (x.q_main, x.q_spec):
            if t is not None:
                t.copy_((t.float().abs() * 0.1 + 20.0 * d ** -0.5).to(torch.bfloat16))
        for t in (x.k_tree, x.k_spec):
            if t is not None:
                t.copy_((sign * (t.float().abs() * 0.2 + 10.0)).to(torch.bfloat16))
        x.run()
        x.check([1 - bad])
        for o in (x.o_main, x.o_spec):
            assert o is None or torch.isnan(o[bad]).all()
        _check_lse(x, bad)


# log2 of the sizes of the cached values: of the first keys, of those from key 100 on; of the nodes' and streams' values
SIZES = {"cached large": (112, 112, 0), "later ones large": (0, 20, 0), "later ones small": (0, -20, 3), "cached tiny": (-100, -100, 0),
         "both large": (89, 89, 89), "behind the prefix large": (0, 0, 89), "behind the prefix tiny": (10, 12, -70), "all tiny": (-110, -112, -110)}


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("nodes,gamma", SHAPES)
@pytest.mark.parametrize("sizes", list(SIZES))
def test_values_of_very_different_sizes(api, d, nodes, gamma, sizes):
    H, lens = 3, [20, 133, 900]
    first, later, behind = SIZES[sizes]
    x = Layer(api, 3, H, d, lens, [nodes] * 3, gamma, seed=11 + d)
    for b, n in enumerate(lens):
        v = _normal((n, H, d), b)
        v[:100] *= 2.0 ** first
        v[100:] *= 2.0 ** later
        _put(x, b, _normal((n, H, d), 20 + b), v)
    for t in (x.v_tree, x.v_spec):
        if t is not None:
            t.copy_((t.float() * 2.0 ** behind).to(torch.bfloat16))
    x.run()
    x.check()


def test_starts_at_the_ends_of_64_bits(api):
    """A start whose sum with the length or the number of rows passes 2^63 is one outside the slab, for all three calls; the sequences
    beside it are dealt with."""
    H, d, far = 2, 64, [2 ** 63 - 1, 2 ** 63 - 30, -2 ** 63, -2 ** 63 + 7]
    for nodes in (3, 30):
        x = Layer(api, 5, H, d, [40, 50, 60, 70, 80], [nodes] * 5, 0, seed=3)
        x.kv_start = _i64(far + x.starts[4:])
        ws = x.workspace()
        api.ss_msa_attention_kvq(x.params(ws))
        assert api.ss_status(ws) == api.SS_ERR_CAPACITY
        x.check([4])
        assert (x.o_main[:4] == 77.0).all() and (x.lse_main[:4] == 77.0).all()
    cache = api.empty_kvq_cache(1, 60, H, d)
    k, v = _rows((1, 5, 6, H, d), 1), _rows((1, 5, 6, H, d), 2)
    lens, out, status = _i32([40, 29, 0, 0, 3]), _i32([0] * 5), api.workspace(256)
    api.ss_kvq_write(k, v, cache, _i64(far + [10]), lens, None, None, None, out, status)
    assert out.tolist() == [40, 29, 0, 0, 9] and api.ss_status(status) == api.SS_ERR_CAPACITY
    assert (cache.tensors[1][0] != 0).any(1).nonzero().flatten().tolist() == list(range(13, 19))
    back = torch.full((1, 5, 6, H, d), 9.0, dtype=torch.bfloat16, device="cuda")
    other = torch.full_like(back, 9.0)
    api.ss_kvq_read(cache, back, other, _i64(far + [13]), _i32([40, 2 ** 31 - 1, -2 ** 31, -8, 0]))
    assert (back[:, :4] == 9.0).all() and (other[:, :4] == 9.0).all()
    step = (k[:, 4].double().amax(-1).clamp(min=0) - k[:, 4].double().amin(-1).clamp(max=0)) / 15 * (1 + 2.0 ** -7)
    assert ((back[:, 4].double() - k[:, 4].double()).abs() <= (step * (1 + 16 * 2.0 ** -8))[..., None]).all()


def _leaning(case, n, H, d, seed):
    """Queries' lean, and keys [n][H][d], of models whose queries and keys are not centred."""
    k = _normal((n, H, d), seed)
    if case == "one channel":                                  # a key channel far larger than the others, queries with a mean
        k[..., 7] = 60.0 * (1.0 - 2.0 * (torch.arange(H) % 2))
        return 4.0, k
    if case == "two channels":
        k[..., 3], k[..., d - 2] = 45.0, -30.0
        return -3.0, k
    if case == "keys with a mean":
        return 2.0, 0.1 * k + 5.0
    k[:, :, 11] += 20.0                                        # "both in one channel"
    return None, k


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("nodes,gamma", SHAPES)
@pytest.mark.parametrize("case", ["one channel", "two channels", "keys with a mean", "both in one channel"])
def test_queries_and_keys_that_are_not_centred(api, d, nodes, gamma, case):
    """Scores are sums of q s (c - z), whose size bounds their error (see attention()): large sums of q alone, or of codes, must not
    enter them.  Log-sum-exps show it."""
    H, lens = 4, [40, 700]
    x = Layer(api, 2, H, d, lens, [nodes] * 2, gamma, seed=17 + d)
    for b, n in enumerate(lens):
        lean, k = _leaning(case, n, H, d, 30 + b)
        _put(x, b, k, _normal((n, H, d), 40 + b))
    for t in (x.q_main, x.q_spec):
        if t is not None and lean is not None:
            t.copy_((t.float() + lean).to(torch.bfloat16))
        elif t is not None:
            t[..., 11] += 50.0
    x.run()
    x.check()


def _single_scores(api, d, rows, case):
    """A row that sees one cached key, its own and the root's lying far below, has that key's score as its log-sum-exp.  Its bound is that
    of attention() for this key alone: (d + 16) 2^-23 sum |q| |k| scale for the products, and what exp and log lose."""
    B, H = 32, 8
    cache = api.empty_kvq_cache(1, 4 * B, H, d)
    lean, k = _leaning(case, B, H, d, 50)
    k = k.to(torch.bfloat16).cuda()[None, :, None]             # [1][B][1][H][d]
    q = _normal((B, rows, H, d), 60)
    if lean is None:
        q[..., 11] += 50.0
    q = (q + (lean or 0.0)).to(torch.bfloat16).cuda()
    start, length = _i64([4 * b for b in range(B)]), _i32([1] * B)
    api.ss_kvq_write(k, k, cache, start, _i32([0] * B), None, None, None, None)
    below = (-200.0 * torch.sign(q.float())).to(torch.bfloat16)
    lse = torch.zeros((B, rows, H), device="cuda")
    kw = dict(q_main=q, o_main=torch.zeros_like(q), k_tree=below, v_tree=below, cache=cache, kv_start=start, kv_len=length, gamma=0, sm_scale=d ** -0.5,
              trees=api.trees_to_device([api.ss_tree_build([-1] + [0] * (rows - 1), 0)] * B), lse_main=lse)
    ws = api.workspace(api.ss_msa_attention_kvq_workspace_bytes(api.make_kvq_attn_params(**kw)))
    api.ss_msa_attention_kvq(api.make_kvq_attn_params(workspace=ws, **kw))
    assert api.ss_status(ws) == 0
    keys = U.cache_values(cache, 0, "cuda")[0][::4]
    score = torch.einsum("brhd,bhd->brh", q.double(), keys) * d ** -0.5
    size = torch.einsum("brhd,bhd->brh", q.double().abs(), keys.abs()) * d ** -0.5
    assert (score > -100.0).all()
    bound = (d + 16) * 2.0 ** -23 * size + 2.0 ** -20 + 65 * 2.0 ** -24 + 2.0 ** -22 * score.abs() + 2.0 ** -20
    err = (lse.double() - score).abs()
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("rows", [24, 64])
@pytest.mark.parametrize("case", ["one channel", "two channels", "keys with a mean", "both in one channel"])
def test_single_scores_of_blocks_that_are_not_centred(api, d, rows, case):
    _single_scores(api, d, rows, case)


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("rows", [1, 8, 12])
@pytest.mark.parametrize("case", ["one channel", "two channels", "keys with a mean", "both in one channel"])
def test_single_scores_of_few_rows_that_are_not_centred(api, d, rows, case):
    _single_scores(api, d, rows, case)


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("nodes,gamma", SHAPES)
@pytest.mark.parametrize("q_scale,k_scale", [(2.0 ** -10, 1.0), (300.0, 1.0), (1.0, 10.0), (2.0 ** -100, 2.0 ** 90), (2.0 ** 100, 2.0 ** -97)])
def test_queries_and_keys_of_other_sizes(api, d, nodes, gamma, q_scale, k_scale):
    """Queries enter the few-rows kernel under a power of two of their own; scores from nothing to hundreds."""
    x = Layer(api, 2, 3, d, [50, 700], [nodes] * 2, gamma, seed=19 + d, q_scale=q_scale, k_scale=k_scale)
    for t in (x.k_tree, x.k_spec):
        if t is not None and k_scale != 1.0:
            t.copy_((t.float() * k_scale).to(torch.bfloat16))
    x.run()
    x.check()


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("nodes,gamma", [s for s in SHAPES if s[0] > 1])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_keys_that_a_row_does_not_see_may_hold_anything(api, d, nodes, gamma, what):
    """The last node's key, which only its own rows see, and the last stream's key of the first node are not numbers: the other rows'
    outputs are what they are without."""
    x = Layer(api, 2, 3, d, [0, 300], [nodes] * 2, gamma, seed=23 + d)
    x.run()
    x.check()
    want = [None if t is None else t.clone() for t in (x.o_main, x.lse_main, x.o_spec, x.lse_spec)]
    x.k_tree[:, nodes - 1] = what
    if gamma:
        x.k_spec[:, 0, gamma - 1] = what
    x.fresh()
    x.run()
    last = nodes - 1
    for t, w in zip((x.o_main, x.lse_main), want[:2]):
        assert torch.equal(t[:, :last], w[:, :last])
        assert not torch.isfinite(t[:, last]).any()
    if gamma:
        for t, w in zip((x.o_spec, x.lse_spec), want[2:]):
            assert torch.equal(t[:, 1:last], w[:, 1:last]) and torch.equal(t[:, 0, :gamma - 1], w[:, 0, :gamma - 1])
            assert not torch.isfinite(t[:, last]).any() and not torch.isfinite(t[:, 0, gamma - 1]).any()
