"""Host-side checks of the cache in 4 bits that need no GPU: refusals before any launch, layouts, the reference itself."""
import ctypes as C
from fractions import Fraction

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kvq_util as U
from paper_2402_11131_b200 import api, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.lib()


class _Stream:
    cuda_stream = 0                          # stands for a torch.cuda.Stream where there is no GPU


def _fake_cache(**kw):
    """A cache with plausible pointers that are never dereferenced."""
    c = api.KvqCache()
    c.n_layers, c.n_heads, c.head_dim, c.device = 2, 4, 64, -1
    for f in ("k_codes", "v_codes", "k_params", "v_params"):
        setattr(c, f, 0x10000)
    c.layer_stride, c.slot_stride, c.head_stride = 100 * 128, 128, 32
    c.param_layer_stride, c.param_slot_stride, c.param_head_stride = 400, 1, 100
    c.total_slots = 100
    for k, v in kw.items():
        setattr(c, k, v)
    return c


class _Rows(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("layer_stride", C.c_int64), ("batch_stride", C.c_int64),
                ("row_stride", C.c_int64), ("head_stride", C.c_int64), ("batch", C.c_int32), ("max_rows", C.c_int32)]


def _fake_rows(**kw):
    r = _Rows(0x20000, 0x20000, 256 * 3 * 8, 256 * 8, 256, 64, 3, 8)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


P = C.c_void_p(0x30000)


CACHE_FAULTS = [
    (dict(head_dim=96), api.SS_ERR_UNSUPPORTED), (dict(n_layers=0), api.SS_ERR_INVALID_ARG), (dict(n_heads=0), api.SS_ERR_INVALID_ARG),
    (dict(k_codes=None), api.SS_ERR_INVALID_ARG), (dict(v_codes=None), api.SS_ERR_INVALID_ARG), (dict(k_params=None), api.SS_ERR_INVALID_ARG),
    (dict(v_params=None), api.SS_ERR_INVALID_ARG), (dict(k_codes=0x10008), api.SS_ERR_INVALID_ARG), (dict(v_params=0x10002), api.SS_ERR_INVALID_ARG),
    (dict(slot_stride=136), api.SS_ERR_UNSUPPORTED), (dict(head_stride=40), api.SS_ERR_UNSUPPORTED), (dict(total_slots=-1), api.SS_ERR_INVALID_ARG),
    (dict(device=3), api.SS_ERR_INVALID_ARG)]          # (not the current device: here there is none)


@pytest.mark.parametrize("kw,code", CACHE_FAULTS)
def test_calls_refuse_caches_they_cannot_read(lib, kw, code):
    c, r = _fake_cache(**kw), _fake_rows()
    assert lib.ss_kvq_write(C.byref(r), C.byref(c), P, P, None, None, None, None, None, None) == code
    assert lib.ss_kvq_read(C.byref(c), C.byref(r), P, None, None, None) == code
    assert lib.ss_msa_attention_kvq(C.byref(_fake_params(cache=c)), None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), api.SS_ERR_INVALID_ARG), (dict(v=None), api.SS_ERR_INVALID_ARG), (dict(k=0x20008), api.SS_ERR_INVALID_ARG),
    (dict(batch=0), api.SS_ERR_INVALID_ARG), (dict(batch=65536), api.SS_ERR_INVALID_ARG), (dict(max_rows=-1), api.SS_ERR_INVALID_ARG),
    (dict(row_stride=252), api.SS_ERR_UNSUPPORTED), (dict(head_stride=68), api.SS_ERR_UNSUPPORTED),
    (dict(layer_stride=4), api.SS_ERR_UNSUPPORTED), (dict(batch_stride=2), api.SS_ERR_UNSUPPORTED)])
def test_calls_refuse_rows_they_cannot_read(lib, kw, code):
    c, r = _fake_cache(), _fake_rows(**kw)
    assert lib.ss_kvq_write(C.byref(r), C.byref(c), P, P, None, None, None, None, None, None) == code
    assert lib.ss_kvq_read(C.byref(c), C.byref(r), P, None, None, None) == code


def test_calls_refuse_sizes_beyond_their_index_arithmetic(lib):
    for c, r, code in ((_fake_cache(n_heads=65536), _fake_rows(), api.SS_ERR_UNSUPPORTED),
                       (_fake_cache(), _fake_rows(max_rows=(1 << 30) + 1), api.SS_ERR_INVALID_ARG)):
        assert lib.ss_kvq_write(C.byref(r), C.byref(c), P, P, None, None, None, None, None, None) == code
        assert lib.ss_kvq_read(C.byref(c), C.byref(r), P, None, None, None) == code
    assert lib.ss_msa_attention_kvq(C.byref(_fake_params(cache=_fake_cache(n_heads=65536))), None) == api.SS_ERR_UNSUPPORTED
    # lengths updated in place are one CTA's work
    c, r = _fake_cache(), _fake_rows(batch=1025)
    assert lib.ss_kvq_write(C.byref(r), C.byref(c), P, P, None, None, None, P, None, None) == api.SS_ERR_UNSUPPORTED


def test_write_and_read_refuse_missing_arguments(lib):
    c, r = _fake_cache(), _fake_rows()
    bad = api.SS_ERR_INVALID_ARG
    assert lib.ss_kvq_write(None, C.byref(c), P, P, None, None, None, None, None, None) == bad
    assert lib.ss_kvq_write(C.byref(r), None, P, P, None, None, None, None, None, None) == bad
    assert lib.ss_kvq_write(C.byref(r), C.byref(c), None, P, None, None, None, None, None, None) == bad
    assert lib.ss_kvq_write(C.byref(r), C.byref(c), P, None, None, None, None, None, None, None) == bad
    assert lib.ss_kvq_read(C.byref(c), C.byref(r), None, None, None, None) == bad
    assert lib.ss_kvq_read(C.byref(c), C.byref(_fake_rows(max_rows=0)), P, None, None, None) == api.SS_OK      # nothing to do


def _fake_params(**kw):
    p = api.KvqAttnParams()
    p.batch, p.gamma, p.max_nodes, p.layer, p.sm_scale = 3, 2, 6, 1, 1.0
    for f in ("q_main", "o_main", "k_tree", "v_tree", "q_spec", "k_spec", "v_spec", "o_spec", "kv_start", "kv_len", "trees", "workspace"):
        setattr(p, f, 0x40000)
    p.cache = _fake_cache()
    p.workspace_bytes = 1 << 40
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), api.SS_ERR_INVALID_ARG), (dict(gamma=-1), api.SS_ERR_INVALID_ARG), (dict(gamma=5), api.SS_ERR_UNSUPPORTED),
    (dict(max_nodes=0), api.SS_ERR_INVALID_ARG), (dict(max_nodes=65), api.SS_ERR_UNSUPPORTED), (dict(layer=2), api.SS_ERR_INVALID_ARG),
    (dict(layer=-1), api.SS_ERR_INVALID_ARG), (dict(q_main=None), api.SS_ERR_INVALID_ARG), (dict(o_main=None), api.SS_ERR_INVALID_ARG),
    (dict(k_tree=None), api.SS_ERR_INVALID_ARG), (dict(v_tree=0x40004), api.SS_ERR_INVALID_ARG), (dict(q_spec=None), api.SS_ERR_INVALID_ARG),
    (dict(o_spec=0x40008), api.SS_ERR_INVALID_ARG), (dict(kv_len=None), api.SS_ERR_INVALID_ARG), (dict(kv_start=None), api.SS_ERR_INVALID_ARG),
    (dict(trees=None), api.SS_ERR_INVALID_ARG), (dict(workspace=None), api.SS_ERR_INVALID_ARG), (dict(sm_scale=float("nan")), api.SS_ERR_INVALID_ARG),
    (dict(sm_scale=float("inf")), api.SS_ERR_INVALID_ARG)])
def test_attention_refuses_bad_arguments_before_any_launch(lib, kw, code):
    assert lib.ss_msa_attention_kvq(C.byref(_fake_params(**kw)), None) == code


def test_attention_workspace(lib):
    need = lib.ss_msa_attention_kvq_workspace_bytes(C.byref(_fake_params()))
    assert need > 256
    assert lib.ss_msa_attention_kvq(C.byref(_fake_params(workspace_bytes=need - 1)), None) == api.SS_ERR_WORKSPACE
    assert lib.ss_msa_attention_kvq(None, None) == api.SS_ERR_INVALID_ARG
    assert lib.ss_msa_attention_kvq_workspace_bytes(C.byref(_fake_params(gamma=9))) == 0
    # the shapes alone decide, not the slab
    assert need == lib.ss_msa_attention_kvq_workspace_bytes(C.byref(_fake_params(cache=_fake_cache(total_slots=10 ** 7))))


def test_binding_refuses_tensors_of_other_sizes(lib):
    cache = api.empty_kvq_cache(2, 10, 3, 64, device="cpu")
    rows = torch.zeros((2, 1, 4, 3, 64), dtype=torch.bfloat16)
    i = torch.zeros(1, dtype=torch.int32)
    for bad in (rows.float(), rows[:1], rows[..., :2, :], rows[..., :32], rows[0], rows.transpose(3, 4).contiguous().transpose(3, 4)):
        with pytest.raises(ValueError):
            api.ss_kvq_write(bad, bad, cache, i, i, stream=_Stream())
        with pytest.raises(ValueError):
            api.ss_kvq_read(cache, bad, bad, i, stream=_Stream())
    with pytest.raises(ValueError):                          # K and V laid out differently
        api.ss_kvq_write(rows, torch.zeros((2, 1, 3, 4, 64), dtype=torch.bfloat16).transpose(2, 3), cache, i, i, stream=_Stream())
    for other in (None, b"\0" * 512, 0):
        with pytest.raises(TypeError):
            api.ss_kvq_write(rows, rows, other, i, i, stream=_Stream())
        with pytest.raises(TypeError):
            api.ss_msa_attention_kvq(other, _Stream())
    for other in (api.CacheLayout(), api.TreeDesc(), C.pointer(cache)):
        with pytest.raises(C.ArgumentError):
            api.ss_kvq_read(other, rows, rows, i, stream=_Stream())
        with pytest.raises(C.ArgumentError):
            api.ss_msa_attention_kvq(other, _Stream())
    codes, params = torch.zeros((1, 4, 2, 32), dtype=torch.uint8), torch.zeros((1, 4, 2), dtype=torch.int32)
    for args in ((codes, params.long(), codes, params), (codes.int(), params, codes, params), (codes, params[:, :3], codes, params[:, :3]),
                 (codes, params, codes[:, :3], params), (codes.transpose(2, 3), params, codes.transpose(2, 3), params)):
        with pytest.raises(ValueError):
            api.make_kvq_cache(*args)
    q = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    ok = dict(q_main=q, o_main=q, k_tree=q, v_tree=q, cache=cache, kv_start=i, kv_len=i, trees=i, gamma=0, sm_scale=1.0)
    api.make_kvq_attn_params(**ok)
    for kw in (dict(q_main=torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)), dict(o_main=q.float()), dict(k_tree=q[:, :1]),
               dict(v_tree=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(gamma=1, q_spec=q), dict(lse_main=q)):
        with pytest.raises(ValueError):
            api.make_kvq_attn_params(**dict(ok, **kw))


def test_binding_refuses_tensors_of_another_device(lib):
    cache = api.empty_kvq_cache(1, 10, 3, 64, device="cpu")
    q, i = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    args = dict(q_main=q, o_main=q, k_tree=q, v_tree=q, cache=cache, kv_start=i, kv_len=i, trees=i, gamma=0, sm_scale=1.0)
    api.make_kvq_attn_params(**args)
    cache.device = 1                                         # as if it lay on the second GPU
    with pytest.raises(ValueError):
        api.make_kvq_attn_params(**args)


def test_struct_sizes_match_the_header(lib):
    assert C.sizeof(api.KvqCache) == 16 + 4 * 8 + 7 * 8
    assert C.sizeof(api.KvqAttnParams) == 24 + 8 * 8 + C.sizeof(api.KvqCache) + 4 * 8 + 3 * 8 + 8


def test_reference_quantiser_by_hand():
    """The reference that the GPU is held to, on rows whose codes can be told by hand."""
    bf = lambda x: U.bits_of(torch.tensor(x, dtype=torch.float32).to(torch.bfloat16))
    c, s, z = U.quantise_row(bf([0.0, 1.0, 2.0, 15.0]))
    assert (list(c), s, z) == ([0, 1, 2, 15], 0x3F80, 0)
    c, s, z = U.quantise_row(bf([-15.0, -1.0, 0.0, -14.5]))
    assert (list(c), s, z) == ([0, 14, 15, 0], 0x3F80, 15)       # -14.5 is in the middle and goes away from zero
    c, s, z = U.quantise_row(bf([0.0, 0.0]))
    assert (list(c), s, z) == ([0, 0], 0x0380, 0)
    c, s, z = U.quantise_row(bf([-7.5, 7.5, 0.5, -0.5]))
    assert (list(c), s, z) == ([0, 15, 9, 7], 0x3F80, 8)         # 8 + 8 is clamped
    assert U.quantise_row(bf([1.0, float("nan")]))[1] == 0x7FFF
    x = np.arange(8, dtype=np.uint8)
    assert list(U.pack_row(x)) == [0x20, 0x64, 0x31, 0x75]
    assert (U.unpack(U.pack_row(x)[None], np.array([0x3F80 | 3 << 16], np.int32))[0] == x - 3.0).all()
    # half a step at most, the scale no more than one bf16 step above a fifteenth of the range
    g = torch.Generator().manual_seed(1)
    for _ in range(20):
        bits = U.bits_of((torch.randn(64, generator=g) * 3).to(torch.bfloat16))
        c, s, z = U.quantise_row(bits)
        v = U.from_bits(bits)
        step = U.from_bits(np.array([s, s - 1], np.uint16))
        assert Fraction(float(step[1])) * 15 < Fraction(float(v.max())) - Fraction(float(v.min())) <= Fraction(float(step[0])) * 15
        off = np.abs((c.astype(float) - z) * step[0] - v)
        assert (off <= step[0] / 2 + (c == 15) * step[0] / 2).all()
