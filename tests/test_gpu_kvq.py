"""The cache in 4 bits on the GPU: rows written (bit by bit against exact fractions), rows read back, attention over the codes."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kvq_util as U
from paper_2402_11131_b200 import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2402_11131_b200 import api, build
    build.build()
    return api


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _i64(x):
    return torch.tensor(x, dtype=torch.int64, device="cuda")


def _rows(shape, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16).cuda()


def _edge_rows(d):
    """Rows at which the quantiser can go wrong, [n][d]."""
    g = torch.Generator().manual_seed(d)
    base = torch.randn((24, d), generator=g)
    base[0] = 0.0
    base[1] = base[1].abs() + 1.0                        # one sign only: the zero point is 0
    base[2] = -base[2].abs() - 1.0                       # .. is 15
    base[3] = torch.linspace(-7.5, 7.5, d)               # quotients in the middle between two codes
    base[4] = torch.arange(d) % 16 * 0.5 - 3.75
    base[5] *= 1e-38                                     # scales at the floor and subnormal values
    base[6] *= 1e-36
    base[7] *= 1e37
    base[8] = 3.3895313892515355e38                      # the largest bf16
    base[8, ::2] *= -1
    base[9] = 0.0
    base[9, d // 2] = 5.0                                # a single value
    base[10, 0] = 3e4                                    # an outlier
    base[11, 3] = float("inf")
    base[12, d - 1] = float("nan")
    base[13, 7] = -float("inf")
    base[14] = 1.0                                       # constants
    base[15] = -0.0
    base[16] = torch.where(torch.arange(d) % 2 == 0, 15.0, 0.0)
    base[17] = torch.where(torch.arange(d) % 3 == 0, 7.5, torch.where(torch.arange(d) % 3 == 1, -7.5, 0.5))
    base[18] = torch.where(torch.arange(d) % 2 == 0, 1.0, -2.0 ** -30)
    base[19] = torch.where(torch.arange(d) % 2 == 0, -15.0, 2.0 ** -60)
    x = base.to(torch.bfloat16)
    x[20] = torch.from_numpy(np.arange(1, d + 1, dtype=np.int16)).view(torch.bfloat16)       # the smallest patterns
    return x


@pytest.mark.parametrize("d", [64, 80, 128])
def test_write_is_the_definition_bit_by_bit_and_read_gives_its_values(api, d):
    edge = _edge_rows(d)
    rows = torch.cat((edge, _rows((200, d), 5).cpu(), _rows((100, d), 6, 37.0).cpu()))
    n, H = 108, 3
    x = rows[:n * H].reshape(1, 1, n, H, d).cuda()
    y = rows.flip(0)[:n * H].reshape(1, 1, n, H, d).contiguous().cuda()
    cache = api.empty_kvq_cache(1, n + 9, H, d)
    for t in cache.tensors:
        t.fill_(0x5A)
    out = _i32([-1])
    api.ss_kvq_write(x, y, cache, _i64([2]), _i32([3]), None, None, None, out)
    assert out.tolist() == [n + 3]
    back = [torch.full((1, 1, n, H, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    api.ss_kvq_read(cache, back[0], back[1], _i64([2]), _i32([3]), None)
    for src, codes, params, got in ((x, *cache.tensors[:2], back[0]), (y, *cache.tensors[2:], back[1])):
        bits, codes, params = U.bits_of(src).reshape(n, H, d), codes[0].cpu().numpy(), params[0].cpu().numpy()
        assert (codes[:5] == 0x5A).all() and (codes[n + 5:] == 0x5A).all() and (params[:5] == 0x5A).all() and (params[n + 5:] == 0x5A).all()
        for r in range(n):
            for h in range(H):
                c, s, z = U.quantise_row(bits[r, h])
                assert params[5 + r, h] == (s | z << 16), (r, h)
                assert (codes[5 + r, h] == U.pack_row(c)).all(), (r, h)
        want = torch.from_numpy(U.unpack(codes[5:n + 5], params[5:n + 5])).to(torch.bfloat16)
        g = got.cpu()[0, 0]
        assert torch.equal(torch.isnan(g), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(g), torch.nan_to_num(want))
        # a value is off by half a step, by a whole one where its code was clamped
        ok = torch.isfinite(want).all(-1)
        step = torch.from_numpy(U.from_bits((params[5:n + 5] & 0xFFFF).astype(np.uint16)))[..., None]
        off = (torch.from_numpy(U.unpack(codes[5:n + 5], params[5:n + 5])) - src.cpu()[0, 0].double()).abs()
        assert (off[ok] <= step.expand_as(off)[ok] * 1.0000001).all()


@pytest.mark.parametrize("d,layers,order", [(128, 3, "slots"), (64, 2, "heads"), (80, 2, "slots"), (80, 1, "heads")])
def test_write_ragged_runs_paths_and_strides(api, d, layers, order):
    """Ragged runs into slabs of either order, from rows with strides, with and without a path; what is not written stays."""
    B, H, R = 4, 5, 17
    starts, lens, counts = [0, 40, 70, 110], [3, 0, 12, 7], [17, 0, 5, 1]
    slots = 140
    if order == "heads":
        codes = [torch.full((layers, H, slots, d // 2), 0x11, dtype=torch.uint8, device="cuda").transpose(1, 2) for _ in "kv"]
        params = [torch.full((layers, slots, H), 0x22, dtype=torch.int32, device="cuda") for _ in "kv"]
    else:
        codes = [torch.full((layers, slots, H, d // 2), 0x11, dtype=torch.uint8, device="cuda") for _ in "kv"]
        params = [torch.full((layers, H, slots), 0x22, dtype=torch.int32, device="cuda").transpose(1, 2) for _ in "kv"]
    cache = api.make_kvq_cache(codes[0], params[0], codes[1], params[1])
    qkv = _rows((layers, B, R, 3, H, d), 3)                      # rows as a fused projection leaves them
    k, v = qkv[:, :, :, 1], qkv[:, :, :, 2]
    rng = np.random.default_rng(d)
    for path in (None, [sorted(rng.choice(R, max(n, 1), replace=False).tolist()) for n in counts]):
        before = [t.cpu().clone() for t in cache.tensors]
        pt = None if path is None else _i32([p + [-1] * (api.SS_PATH_STRIDE - len(p)) for p in path])
        out = _i32([-5] * B)
        api.ss_kvq_write(k, v, cache, _i64(starts), _i32(lens), _i32(counts), pt, None, out)
        assert out.tolist() == [a + b for a, b in zip(lens, counts)]
        after = [t.cpu() for t in cache.tensors]
        for i, src in ((0, k), (2, v)):
            want_c, want_p = before[i].numpy().copy(), before[i + 1].numpy().copy()
            for layer in range(layers):
                for b in range(B):
                    for r in range(counts[b]):
                        bits = U.bits_of(src[layer, b, r if path is None else path[b][r]])
                        for h in range(H):
                            c, s, z = U.quantise_row(bits[h])
                            want_c[layer, starts[b] + lens[b] + r, h] = U.pack_row(c)
                            want_p[layer, starts[b] + lens[b] + r, h] = s | z << 16
            assert (after[i].numpy() == want_c).all() and (after[i + 1].numpy() == want_p).all()
        lens = [a + 1 for a in lens]


def test_write_lengths_in_place_and_sequences_that_do_not_fit(api):
    d, H, R = 64, 2, 6
    cache = api.empty_kvq_cache(1, 40, H, d)
    k, v = _rows((1, 5, R, H, d), 1), _rows((1, 5, R, H, d), 2)
    lens = _i32([4, 4, 2, -1, 0])
    ws = api.workspace(256)
    # over its capacity; behind the slab; fits exactly; a negative length; nothing to write
    api.ss_kvq_write(k, v, cache, _i64([0, 33, 20, 30, 39]), lens, _i32([6, 4, 6, 2, -3]), None, _i32([9, 99, 8, 99, 99]), lens, ws)
    assert lens.tolist() == [4, 4, 8, -1, 0]
    assert api.ss_status(ws) == api.SS_ERR_CAPACITY
    assert api.ss_status(ws) == 0
    used = (cache.tensors[1][0] != 0).any(1).nonzero().flatten().tolist()
    assert used == list(range(22, 28))
    # more rows asked for than there are: all there are; path entries outside the rows are left out
    lens = _i32([0] * 5)
    out = _i32([0] * 5)
    api.ss_kvq_write(k, v, cache, _i64([0, 6, 12, 18, 24]), lens, _i32([99] * 5), None, None, out)
    assert out.tolist() == [R] * 5
    for t in cache.tensors:
        t.zero_()
    path = _i32([[2, R, -1, 5] + [0] * 60] * 5)
    api.ss_kvq_write(k, v, cache, _i64([0, 6, 12, 18, 24]), lens, _i32([4, 0, 0, 0, 0]), path, None, None)
    assert (cache.tensors[1][0] != 0).any(1).nonzero().flatten().tolist() == [0, 3]
    # no rows at all
    api.ss_kvq_write(k[:, :, :0], v[:, :, :0], cache, _i64([0] * 5), _i32([1, 2, 3, 4, 5]), None, None, None, out)
    assert out.tolist() == [1, 2, 3, 4, 5]


@pytest.mark.parametrize("d,H", [(64, 3), (80, 5), (128, 13)])
def test_write_and_read_of_long_runs(api, d, H):
    """Runs of many steps of a CTA, beside short ones, and a head count that no CTA's warps divide."""
    B, layers, M = 3, 2, 2900
    cache = api.empty_kvq_cache(layers, 6000, H, d)
    starts, n_rows = _i64([0, 2950, 3100]), _i32([M, 1, 2603])
    k, v = _rows((layers, B, M, H, d), d), _rows((layers, B, M, H, d), d + 1)
    out = _i32([0] * B)
    api.ss_kvq_write(k, v, cache, starts, _i32([0, 0, 0]), n_rows, None, None, out)
    assert out.tolist() == n_rows.tolist()
    back = [torch.full_like(k, 7.0) for _ in "kv"]
    api.ss_kvq_read(cache, back[0], back[1], starts, None, n_rows)
    for b, n in enumerate(n_rows.tolist()):
        for x, got in ((k, back[0]), (v, back[1])):
            # within half a step of the value's own scale where nothing was clamped, a step anywhere; the value is rounded to bf16 once
            want = x[:, b, :n].double()
            s = (want.amax(-1).clamp(min=0) - want.amin(-1).clamp(max=0)) / 15 * (1 + 2.0 ** -7)
            err = (got[:, b, :n].double() - want).abs()
            assert (err <= (s * (1 + 16 * 2.0 ** -8))[..., None]).all()
            assert (got[:, b, n:] == 7.0).all()
    # the same rows one call per sequence give the same cache
    other = api.empty_kvq_cache(layers, 6000, H, d)
    for b, n in enumerate(n_rows.tolist()):
        for at in range(0, n, 701):
            m = min(701, n - at)
            api.ss_kvq_write(k[:, b:b + 1, at:at + m], v[:, b:b + 1, at:at + m], other, starts[b:b + 1], _i32([at]), None, None, None, None)
    for a, c in zip(cache.tensors, other.tensors):
        assert torch.equal(a, c)


def test_read_leaves_what_is_not_asked_for(api):
    d, H = 80, 3
    cache = api.empty_kvq_cache(2, 50, H, d)
    k, v = _rows((2, 1, 50, H, d), 1), _rows((2, 1, 50, H, d), 2)
    api.ss_kvq_write(k, v, cache, _i64([0]), _i32([0]), None, None, None, None)
    kv, vv = zip(*(U.cache_values(cache, layer) for layer in range(2)))
    back = [torch.full((2, 3, 12, H, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    api.ss_kvq_read(cache, back[0], back[1], _i64([0, 10, 45]), _i32([3, -12, 0]), _i32([5, 12, 99]))
    for got, ref in ((back[0].cpu(), kv), (back[1].cpu(), vv)):
        want = torch.full((2, 3, 12, H, d), 9.0, dtype=torch.bfloat16)
        for layer in range(2):
            want[layer, 0, :5] = ref[layer][3:8].to(torch.bfloat16)
            want[layer, 1, 2:] = ref[layer][:10].to(torch.bfloat16)       # (slots -2 and -1 are outside the slab)
            want[layer, 2, :5] = ref[layer][45:].to(torch.bfloat16)       # (as are those from 50 on)
        assert torch.equal(got, want)


class Layer:
    """Inputs of one layer of attention over a cache in 4 bits."""

    def __init__(self, api, B, H, d, lens, nodes, gamma, seed=0, order="slots", lse=True, q_scale=1.0, k_scale=1.0, kind="uniform_parent",
                 slack=0, scale=None):
        rng = np.random.default_rng(seed)
        self.api, self.B, self.H, self.d, self.lens, self.nodes, self.gamma = api, B, H, d, lens, nodes, gamma
        T = max(nodes)
        caps = [n + 5 for n in lens]
        self.starts = [int(x) + 2 for x in np.cumsum([0] + caps[:-1])]
        slots = sum(caps) + 4 + slack
        if order == "heads":
            codes = [torch.zeros((1, H, slots, d // 2), dtype=torch.uint8, device="cuda").transpose(1, 2) for _ in "kv"]
            params = [torch.zeros((1, slots, H), dtype=torch.int32, device="cuda") for _ in "kv"]
            self.cache = api.make_kvq_cache(codes[0], params[0], codes[1], params[1])
        else:
            self.cache = api.empty_kvq_cache(1, slots, H, d)
        for i, t in enumerate(self.cache.tensors):          # slots that nothing owns hold anything: here NaN scales
            t.fill_(0x7FFF if i % 2 else 0xA7)
        for b in range(B):
            if lens[b]:
                k = _rows((1, 1, lens[b], H, d), 1000 * seed + b, k_scale)
                v = _rows((1, 1, lens[b], H, d), 2000 * seed + b + 500)
                api.ss_kvq_write(k, v, self.cache, _i64([self.starts[b]]), _i32([0]), None, None, None, None)
        self.parents = [W.draw_tree(rng, n, 6, kind) if n else None for n in nodes]
        one = api.ss_tree_build([-1], 0)
        descs = [api.ss_tree_build(p, gamma) if p is not None else api.TreeDesc() for p in self.parents]
        assert one.n_nodes == 1
        self.trees = api.trees_to_device(descs)
        self.kv_len, self.kv_start = _i32(lens), _i64(self.starts)
        self.q_main, self.k_tree, self.v_tree = (_rows((B, T, H, d), seed + i, q_scale if i == 11 else 1.0) for i in (11, 12, 13))
        self.q_spec, self.k_spec, self.v_spec = (_rows((B, T, gamma, H, d), seed + i, q_scale if i == 14 else 1.0) if gamma else None
                                                 for i in (14, 15, 16))
        self.scale = d ** -0.5 if scale is None else scale
        self.with_lse = lse
        self.fresh()

    def fresh(self):
        B, T, H, d, g = self.B, max(self.nodes), self.H, self.d, self.gamma
        self.o_main = torch.full((B, T, H, d), 77.0, dtype=torch.bfloat16, device="cuda")
        self.o_spec = torch.full((B, T, g, H, d), 77.0, dtype=torch.bfloat16, device="cuda") if g else None
        self.lse_main = torch.full((B, T, H), 77.0, device="cuda") if self.with_lse else None
        self.lse_spec = torch.full((B, T, g, H), 77.0, device="cuda") if self.with_lse and g else None

    def params(self, ws, **kw):
        return self.api.make_kvq_attn_params(**dict(dict(
            q_main=self.q_main, o_main=self.o_main, k_tree=self.k_tree, v_tree=self.v_tree, cache=self.cache, kv_start=self.kv_start,
            kv_len=self.kv_len, trees=self.trees, gamma=self.gamma, sm_scale=self.scale, q_spec=self.q_spec, k_spec=self.k_spec,
            v_spec=self.v_spec, o_spec=self.o_spec, lse_main=self.lse_main, lse_spec=self.lse_spec, workspace=ws), **kw))

    def workspace(self):
        return self.api.workspace(self.api.ss_msa_attention_kvq_workspace_bytes(self.params(None)))

    def run(self, ws=None, **kw):
        ws = self.workspace() if ws is None else ws
        self.api.ss_msa_attention_kvq(self.params(ws, **kw))
        assert self.api.ss_status(ws) == 0
        return ws

    def check(self, seqs=None):
        kv, vv = U.cache_values(self.cache, 0, "cuda")
        vs = U.value_scales(self.cache, 0, "cuda")
        T, g = max(self.nodes), self.gamma
        for b in range(self.B) if seqs is None else seqs:
            n, s0, L = self.nodes[b], self.starts[b], self.lens[b]
            if n:
                spec = [t[b, :n] if g else None for t in (self.q_spec, self.k_spec, self.v_spec)] if g else [None] * 3
                o, lse, o_tol, lse_tol = U.attention(self.parents[b], g, self.scale, self.q_main[b, :n], spec[0], kv[s0:s0 + L], vv[s0:s0 + L],
                                                     self.k_tree[b, :n], self.v_tree[b, :n], spec[1], spec[2], vs[s0:s0 + L])
                got = [self.o_main[b, :n].double()] + ([self.o_spec[b, :n].double().flatten(0, 1)] if g else [])
                err = (torch.cat(got) - o).abs()
                assert torch.isfinite(err).all(), b
                assert (err <= o_tol).all(), (b, float((err / o_tol).max()))
                if self.with_lse:
                    got = [self.lse_main[b, :n].double()] + ([self.lse_spec[b, :n].double().flatten(0, 1)] if g else [])
                    err = (torch.cat(got) - lse).abs()
                    assert (err <= lse_tol).all(), (b, float((err / lse_tol).max()))
            # rows of nodes that the tree does not have are left as they were
            for t in (self.o_main, self.o_spec, self.lse_main, self.lse_spec):
                if t is not None:
                    assert (t[b, n:] == 77.0).all()


LENGTHS = [0, 1, 2, 15, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 511, 700]


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("nodes,gamma", [(1, 0), (1, 4), (5, 0), (8, 0), (9, 0), (16, 0), (17, 1), (33, 0), (64, 0), (27, 2), (64, 4), (32, 3)])
def test_attention_over_lengths_and_trees(api, d, nodes, gamma):
    """One batch with every length from none to several tiles; trees of other sizes beside the largest one."""
    B = len(LENGTHS)
    counts = [nodes if b % 3 else max(1, nodes - b) for b in range(B)]
    x = Layer(api, B, 3, d, LENGTHS, counts, gamma, seed=d + nodes)
    x.run()
    x.check()


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("nodes,gamma", [(17, 0), (20, 0), (32, 0), (8, 2), (6, 4), (11, 1), (5, 3)])
def test_attention_of_blocks_of_up_to_32_rows(api, d, nodes, gamma):
    B = len(LENGTHS)
    counts = [nodes if b % 3 else max(1, nodes - b) for b in range(B)]
    x = Layer(api, B, 3, d, LENGTHS, counts, gamma, seed=2 * d + nodes)
    x.run()
    x.check()


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("rows", [1, 7, 8, 9, 16, 17, 19, 32, 33, 50, 64])
@pytest.mark.parametrize("length", [5, 112, 900])
def test_attention_writes_its_rows_and_nothing_else(api, d, rows, length):
    """One sequence (whole heads, and heads in pieces), odd heads; what lies around the outputs is left as it was."""
    x = Layer(api, 1, 5, d, [length], [rows], 0, seed=rows + length)
    room = torch.full((x.o_main.numel() + 2048,), 77.0, dtype=torch.bfloat16, device="cuda")
    room_lse = torch.full((x.lse_main.numel() + 2048,), 77.0, device="cuda")
    x.o_main = room[1024:-1024].view(x.o_main.shape)
    x.lse_main = room_lse[1024:-1024].view(x.lse_main.shape)
    x.run()
    x.check()
    for t in (room, room_lse):
        assert (t[:1024] == 77.0).all() and (t[-1024:] == 77.0).all()


@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("H,length,nodes,gamma,order", [(32, 2048, 1, 0, "slots"), (1, 5000, 4, 0, "heads"), (2, 3001, 64, 0, "slots"),
                                                        (7, 1000, 40, 1, "heads"), (32, 517, 16, 3, "slots"), (40, 100, 64, 4, "heads"),
                                                        (148, 33, 2, 0, "slots"), (1, 1, 1, 0, "slots"), (1, 0, 1, 0, "heads")])
def test_attention_of_one_sequence(api, d, H, length, nodes, gamma, order):
    x = Layer(api, 1, H, d, [length], [nodes], gamma, seed=nodes + H, order=order)
    x.run()
    x.check()


@pytest.mark.parametrize("nodes,gamma", [(1, 0), (12, 0), (40, 0), (64, 2)])
def test_attention_of_a_ragged_batch(api, nodes, gamma):
    """Many sequences of very different lengths: pieces that end inside heads, whole heads between them; a workspace reused."""
    rng = np.random.default_rng(nodes)
    lens = [int(n) for n in rng.integers(0, 900, 70)]
    lens[3], lens[40] = 7000, 0
    x = Layer(api, 70, 2, 128, lens, [nodes] * 70, gamma, seed=nodes, kind="uniform_parent")
    ws = x.run()
    x.check()
    first = [t.clone() for t in (x.o_main, x.lse_main)]
    for _ in range(3):                                   # the workspace is left ready, and results do not depend on arrival
        x.fresh()
        x.run(ws)
        assert torch.equal(x.o_main, first[0]) and torch.equal(x.lse_main, first[1])


@pytest.mark.parametrize("nodes,gamma", [(1, 0), (10, 0), (50, 0), (40, 3)])
def test_attention_scores_that_grow_along_the_keys_or_lie_far_apart(api, nodes, gamma):
    """References that later keys exceed by far, weights that underflow, and a first tile that outweighs all others."""
    for grow in (1, -1):
        x = Layer(api, 2, 4, 128, [1500, 333], [nodes, nodes], gamma, seed=3, q_scale=1.0)
        for b in range(2):
            L = x.lens[b]
            ramp = torch.linspace(*((0.01, 12.0) if grow > 0 else (12.0, 0.01)), L).reshape(1, 1, L, 1, 1)
            k = (_rows((1, 1, L, 4, 128), 5 + b).cpu().float() * ramp).to(torch.bfloat16).cuda()
            v = _rows((1, 1, L, 4, 128), 9 + b)
            api.ss_kvq_write(k, v, x.cache, _i64([x.starts[b]]), _i32([0]), None, None, None, None)
        x.run()
        x.check()


def test_attention_scale_of_zero_and_negative_scales(api):
    for scale in (0.0, -0.3, 1e-30):
        x = Layer(api, 2, 3, 64, [77, 300], [12, 3], 1, seed=8, scale=scale)
        x.run()
        x.check()


def test_attention_skips_sequences_that_cannot_be_run(api):
    x = Layer(api, 5, 3, 64, [50, 60, 70, 80, 40], [4, 4, 0, 4, 4], 1, seed=4)
    ws = x.workspace()
    # over its capacity; behind the slab; no nodes; the others are run
    x.kv_start = _i64([x.starts[0], 10 ** 9] + x.starts[2:])
    cap = _i32([49, 10 ** 9, 99, 80, 40])
    api.ss_msa_attention_kvq(x.params(ws, kv_capacity=cap))
    assert api.ss_status(ws) == api.SS_ERR_CAPACITY
    x.check([3, 4])
    for t in (x.o_main, x.o_spec, x.lse_main, x.lse_spec):
        assert (t[:3] == 77.0).all()
    api.ss_msa_attention_kvq(x.params(ws, kv_len=_i32([-4] * 5)))
    assert api.ss_status(ws) == api.SS_ERR_CAPACITY


@pytest.mark.parametrize("nodes", [3, 30])
def test_attention_skips_lengths_at_the_end_of_32_bits(api, nodes):
    """Lengths from 2^31 - 2^16 on are refused on the device, whatever the slab is said to hold; the sequences beside them run."""
    x = Layer(api, 3, 2, 64, [40, 70, 100], [nodes] * 3, 0, seed=3)
    ws = x.workspace()
    p = x.params(ws)
    p.cache.total_slots = 1 << 33                            # (a length that is refused reads nothing)
    x.kv_len[1] = 2 ** 31 - 1
    api.ss_msa_attention_kvq(p)
    assert api.ss_status(ws) == api.SS_ERR_CAPACITY
    x.check([0, 2])
    assert (x.o_main[1] == 77.0).all() and (x.lse_main[1] == 77.0).all()


def test_two_calls_at_once(api):
    """Calls on two streams, each with a workspace of its own, and a path with the same node twice."""
    xs = [Layer(api, 4, 4, 128, [900, 30, 2000, 500], [n] * 4, 0, seed=40 + n) for n in (7, 40)]
    spaces, streams = [x.workspace() for x in xs], [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, ws, s in zip(xs, spaces, streams):
            api.ss_msa_attention_kvq(x.params(ws), s)
    torch.cuda.synchronize()
    for x, ws in zip(xs, spaces):
        assert api.ss_status(ws) == 0
        x.check()
    cache = api.empty_kvq_cache(1, 16, 2, 64)
    k = _rows((1, 1, 5, 2, 64), 3)
    path = torch.full((1, api.SS_PATH_STRIDE), -1, dtype=torch.int32, device="cuda")
    path[0, :4] = torch.tensor([0, 3, 3, 1])
    back = torch.zeros((1, 1, 4, 2, 64), dtype=torch.bfloat16, device="cuda")
    api.ss_kvq_write(k, k, cache, _i64([2]), _i32([0]), _i32([4]), path, None, None)
    api.ss_kvq_read(cache, back, torch.empty_like(back), _i64([2]), None, None)
    assert torch.equal(back[:, :, 1], back[:, :, 2]) and not torch.equal(back[:, :, 0], back[:, :, 1])


def test_attention_a_row_that_was_not_finite_stays_within_its_head(api):
    """A value that is not finite makes its head's row NaN, and with it the outputs that see it; other heads and sequences do not."""
    x = Layer(api, 2, 3, 128, [100, 90], [6, 6], 0, seed=6)
    k = _rows((1, 1, 1, 3, 128), 1)
    k[0, 0, 0, 1, 5] = float("nan")
    api.ss_kvq_write(k, k, x.cache, _i64([x.starts[0]]), _i32([44]), None, None, None, None)
    x.run()
    assert torch.isnan(x.o_main[0, :, 1]).all()
    assert torch.isfinite(x.o_main[0, :, 0]).all() and torch.isfinite(x.o_main[0, :, 2]).all()
    x.check([1])


def test_attention_beyond_32_bit_offsets(api):
    """A slab of more than 2^32 bytes of codes: the sequence lies at its end."""
    H, d = 32, 128
    slots = (1 << 32) // (H * d // 2) + 700
    try:
        x = Layer(api, 1, H, d, [300], [5], 0, seed=2, slack=slots)
    except torch.OutOfMemoryError:
        pytest.skip("no room for a slab of 4 GiB")
    kc, kp, vc, vp = x.cache.tensors
    at, s0 = slots - 320, x.starts[0]
    for t in (kc, kp, vc, vp):
        t[0, at:at + 300].copy_(t[0, s0:s0 + 300].clone())
        t[0, s0:s0 + 300].fill_(0x7FFF if t.dtype == torch.int32 else 0x5A)
    back = [torch.zeros((1, 1, 300, H, d), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    api.ss_kvq_read(x.cache, back[0], back[1], _i64([at]), None, None)
    x.kv_start = _i64([at])
    x.run()
    k = U.unpack(kc[0, at:at + 300].cpu().numpy(), kp[0, at:at + 300].cpu().numpy())
    v = U.unpack(vc[0, at:at + 300].cpu().numpy(), vp[0, at:at + 300].cpu().numpy())
    assert torch.equal(back[0][0, 0].cpu(), torch.from_numpy(k).to(torch.bfloat16))
    o, _, tol, _ = U.attention(x.parents[0], 0, x.scale, x.q_main[0].cpu(), None, torch.from_numpy(k), torch.from_numpy(v), x.k_tree[0].cpu(),
                               x.v_tree[0].cpu(), None, None, U.value_scales(x.cache, 0)[at:at + 300])
    assert ((x.o_main[0].cpu().double() - o).abs() <= tol).all()


def test_calls_of_other_shapes_share_a_workspace(api):
    """Grids, partial rows and kernels of different sizes in turn on one workspace, eagerly and as two captured graphs."""
    xs = [Layer(api, 1, 1, 64, [150], [2], 0, seed=31), Layer(api, 2, 8, 128, [3000, 900], [40, 40], 0, seed=32),
          Layer(api, 1, 2, 80, [700], [64], 1, seed=33), Layer(api, 1, 32, 128, [2000], [1], 0, seed=34),
          Layer(api, 3, 2, 128, [400, 33, 5000], [14, 14, 14], 0, seed=35), Layer(api, 1, 1, 128, [90], [30], 0, seed=36)]
    ws = max((x.workspace() for x in xs), key=lambda w: w.numel())
    for order in ([0, 1, 2, 3, 4, 5], [5, 3, 1, 0, 4, 2], [1, 5, 0, 4, 3, 2]):
        for i in order:
            xs[i].fresh()
            xs[i].run(ws)
        for x in xs:
            x.check()
    params = [x.params(ws) for x in xs]
    graphs = []
    for part in (params[:3], params[3:]):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            for p in part:
                api.ss_msa_attention_kvq(p)
    for _ in range(3):
        for x in xs:                                          # (in place: the graphs hold these tensors)
            for t in (x.o_main, x.o_spec, x.lse_main, x.lse_spec):
                if t is not None:
                    t.fill_(77.0)
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for x in xs:
            x.check()
    assert api.ss_status(ws) == 0


def test_captured_calls_and_another_stream(api):
    """Write, attention and read in a graph on a side stream, replayed with other contents of the same buffers."""
    x = Layer(api, 3, 4, 128, [40, 300, 129], [9, 9, 9], 2, seed=12)
    ws = x.workspace()
    p = x.params(ws)
    rows = [_rows((1, 3, 4, 4, 128), 21 + i) for i in range(2)]
    lens, out = _i32(x.lens), _i32([0] * 3)
    starts = _i64(x.starts)
    back = [torch.zeros((1, 3, 4, 4, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv"]

    def step():
        api.ss_kvq_write(rows[0], rows[1], x.cache, starts, lens, None, None, None, out)
        api.ss_msa_attention_kvq(p)
        api.ss_kvq_read(x.cache, back[0], back[1], starts, lens, None)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (50, 60):
        for i in range(2):
            rows[i].copy_(_rows((1, 3, 4, 4, 128), seed + i))
        x.kv_len.copy_(_i32([n + 4 for n in x.lens]))          # the attention sees the rows that the graph writes
        x.q_main.copy_(_rows(tuple(x.q_main.shape), seed + 5))
        graph.replay()
        torch.cuda.synchronize()
        assert out.tolist() == [n + 4 for n in x.lens]
        kv, vv = U.cache_values(x.cache, 0)
        old, x.lens = x.lens, [n + 4 for n in x.lens]
        x.check()
        x.lens = old
        for b in range(3):
            s0 = x.starts[b] + x.lens[b]
            assert torch.equal(back[0][0, b].cpu(), kv[s0:s0 + 4].to(torch.bfloat16))
            assert torch.equal(back[1][0, b].cpu(), vv[s0:s0 + 4].to(torch.bfloat16))


@pytest.mark.parametrize("d", [64, 128])
def test_a_decode_loop_over_a_cache_in_4_bits(api, d):
    """Prompt, then steps of attention in every layer, verification and the accepted path's rows: lengths never leave the device."""
    B, H, layers, T, V, g = 3, 4, 2, 14, 97, 2
    cache = api.empty_kvq_cache(layers, 400, H, d)
    starts, kv_len = _i64([0, 120, 260]), _i32([0, 0, 0])
    prompt = [_rows((layers, B, 60, H, d), 31 + i) for i in range(2)]
    api.ss_kvq_write(prompt[0], prompt[1], cache, starts, kv_len, _i32([60, 1, 33]), None, None, kv_len)
    assert kv_len.tolist() == [60, 1, 33]
    rng = np.random.default_rng(5)
    vws = api.workspace(api.ss_tree_verify_workspace_bytes(B, T, V))
    ws = None
    for step in range(4):
        parents = [W.draw_tree(rng, T, 4, "topk_growth") for _ in range(B)]
        trees = api.trees_to_device([api.ss_tree_build(p, g) for p in parents])
        tokens = _i32(rng.integers(0, V, (B, T)).tolist())
        logits = torch.from_numpy(rng.standard_normal((B, T, V)).astype(np.float32)).cuda()
        for b in range(B):                                       # some drafts are right
            for c in range(1, T):
                if rng.random() < 0.5:
                    logits[b, parents[b][c], int(tokens[b, c])] = 16.0
        nodes = [_rows((layers, B, T, H, d), 100 * step + 40 + i) for i in range(2)]
        for layer in range(layers):
            q = _rows((B, T, H, d), 7 * step + layer)
            spec = [_rows((B, T, g, H, d), 9 * step + layer + i) for i in range(3)] if layer == layers - 1 else [None] * 3
            gamma = g if layer == layers - 1 else 0
            o, lse = torch.zeros_like(q), torch.zeros((B, T, H), device="cuda")
            os_ = torch.zeros_like(spec[0]) if gamma else None
            kw = dict(q_main=q, o_main=o, k_tree=nodes[0][layer], v_tree=nodes[1][layer], cache=cache, layer=layer, kv_start=starts, kv_len=kv_len,
                      trees=trees, gamma=gamma, sm_scale=d ** -0.5, q_spec=spec[0], k_spec=spec[1], v_spec=spec[2], o_spec=os_, lse_main=lse)
            need = api.ss_msa_attention_kvq_workspace_bytes(api.make_kvq_attn_params(**kw))
            if ws is None or ws.numel() < need:
                ws = api.workspace(need)
            api.ss_msa_attention_kvq(api.make_kvq_attn_params(workspace=ws, **kw))
            assert api.ss_status(ws) == 0
            kv, vv = U.cache_values(cache, layer, "cuda")
            vs = U.value_scales(cache, layer, "cuda")
            for b in range(B):
                s0, L = int(starts[b]), int(kv_len[b])
                ref = U.attention(parents[b], gamma, d ** -0.5, q[b], spec[0][b] if gamma else None, kv[s0:s0 + L], vv[s0:s0 + L], nodes[0][layer, b],
                                  nodes[1][layer, b], spec[1][b] if gamma else None, spec[2][b] if gamma else None, vs[s0:s0 + L])
                got = torch.cat([o[b].double()] + ([os_[b].double().flatten(0, 1)] if gamma else []))
                assert ((got - ref[0]).abs() <= ref[2]).all()
        al, ap, ln, bt = _i32([0] * B), _i32([[0] * 64] * B), _i32([0] * B), _i32([0] * B)
        api.ss_tree_verify(logits, tokens, trees, al, ap, ln, bt, None, vws)
        before = kv_len.tolist()
        api.ss_kvq_write(nodes[0], nodes[1], cache, starts, kv_len, al, ap, None, kv_len)
        assert kv_len.tolist() == [n + m for n, m in zip(before, al.tolist())]
        for b in range(B):
            for i in range(int(al[b])):
                node = int(ap[b, i])
                bits = U.bits_of(nodes[0][layers - 1, b, node])
                for h in range(H):
                    c, s, z = U.quantise_row(bits[h])
                    slot = int(starts[b]) + before[b] + i
                    assert int(cache.tensors[1][layers - 1, slot, h]) == (s | z << 16)
                    assert (cache.tensors[0][layers - 1, slot, h].cpu().numpy() == U.pack_row(c)).all()
