"""Host-side checks of the cache in 4 bits: what its calls refuse before any launch, sizes and tensors at the edge of what they take."""
import ctypes as C
import gc
import weakref

import pytest

torch = pytest.importorskip("torch")

from paper_2402_11131_b200 import api
from test_kvq_host import P, _fake_cache, _fake_params, _fake_rows, lib  # noqa: F401  (lib is a fixture)


def test_calls_refuse_slabs_beyond_their_index_arithmetic(lib):
    c, r = _fake_cache(total_slots=(1 << 48) + 1), _fake_rows()
    assert lib.ss_kvq_write(C.byref(r), C.byref(c), P, P, None, None, None, None, None, None) == api.SS_ERR_INVALID_ARG
    assert lib.ss_kvq_read(C.byref(c), C.byref(r), P, None, None, None) == api.SS_ERR_INVALID_ARG
    assert lib.ss_msa_attention_kvq(C.byref(_fake_params(cache=c)), None) == api.SS_ERR_INVALID_ARG


class _Stream:
    cuda_stream = 0                          # stands for a torch.cuda.Stream where there is no GPU


class _OnGpu:
    """A CPU tensor that says it lies on GPU 0: what the binding sees of a tensor, without one."""

    def __init__(self, t, device=0):
        self._t, self._device = t, device

    def get_device(self):
        return self._device

    def __getattr__(self, name):
        return getattr(self._t, name)


def test_caches_in_host_memory_are_refused_at_every_call(lib):
    cache = api.empty_kvq_cache(2, 10, 4, 64, device="cpu")
    assert cache.device < -1
    c, r = _fake_cache(device=cache.device), _fake_rows()
    assert lib.ss_kvq_write(C.byref(r), C.byref(c), P, P, None, None, None, None, None, None) == api.SS_ERR_INVALID_ARG
    assert lib.ss_kvq_read(C.byref(c), C.byref(r), P, None, None, None) == api.SS_ERR_INVALID_ARG
    assert lib.ss_msa_attention_kvq(C.byref(_fake_params(cache=c)), None) == api.SS_ERR_INVALID_ARG
    # through the binding: host rows, whatever the cache says of itself
    rows, i, l = torch.zeros((2, 1, 3, 4, 64), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int64)
    for device in (cache.device, -1, 0):
        cache.device = device
        with pytest.raises(ValueError):
            api.ss_kvq_write(rows, rows, cache, l, i, stream=_Stream())
        with pytest.raises(ValueError):
            api.ss_kvq_read(cache, rows, rows, l, stream=_Stream())


def test_binding_refuses_whole_numbers_of_other_types_sizes_and_places(lib):
    """kv_start, the lengths and the path reach the kernels as bare pointers: another type or a shorter tensor would be read past its
    end.  (No call here gets as far as a launch, GPU or not: what the binding lets through is a cache that the library refuses.)"""
    B = 3
    cache = api.empty_kvq_cache(2, 10, 4, 64, device="cpu")
    cache.device, cache.total_slots = 0, -1
    rows = _OnGpu(torch.zeros((2, B, 5, 4, 64), dtype=torch.bfloat16))
    good = dict(kv_start=torch.zeros(B, dtype=torch.int64), kv_len_in=torch.zeros(B, dtype=torch.int32), n_rows=torch.zeros(B, dtype=torch.int32),
                path=torch.zeros((B, 64), dtype=torch.int32), kv_capacity=torch.zeros(B, dtype=torch.int32), kv_len_out=torch.zeros(B, dtype=torch.int32),
                status=torch.zeros(256, dtype=torch.uint8))
    good = {k: _OnGpu(t) for k, t in good.items()}
    read = dict(kv_start=good["kv_start"], first=good["kv_len_in"], n_rows=good["n_rows"])

    def write(**kw):
        api.native().kvq_write(rows, rows, cache, *dict(good, **kw).values(), _Stream())

    def back(**kw):
        api.native().kvq_read(cache, rows, rows, *dict(read, **kw).values(), _Stream())

    for call in (write, back):                               # everything in order: the library's own refusal
        with pytest.raises(api.SsError) as e:
            call()
        assert e.value.status == api.SS_ERR_INVALID_ARG
    for call, names in ((write, list(good)[:-1]), (back, list(read))):
        for name in names:
            t = good.get(name, read.get(name))._t
            bad = [_OnGpu(t.to(torch.int32 if t.dtype is torch.int64 else torch.int64)), _OnGpu(t.float()), _OnGpu(t[:B - 1]), _OnGpu(t, 1), t,
                   _OnGpu(torch.stack((t, t), -1)[..., 0])]
            if name == "path":
                bad.append(_OnGpu(t[:, :63].contiguous()))
            for b in bad:
                with pytest.raises(ValueError, match=name):
                    call(**{name: b})
    for b in (good["status"]._t, _OnGpu(good["status"]._t, 1), _OnGpu(good["status"]._t[:3])):
        with pytest.raises(ValueError, match="status"):
            write(status=b)
    for kw in (dict(kv_start=None), dict(kv_len_in=None)):
        with pytest.raises(api.SsError):
            write(**kw)


def test_attention_parameters_refuse_whole_numbers_of_other_types_and_sizes(lib):
    B = 3
    cache = api.empty_kvq_cache(1, 10, 3, 64, device="cpu")
    cache.device = 0
    q = torch.zeros((B, 2, 3, 64), dtype=torch.bfloat16)
    gpu = lambda **kw: {k: _OnGpu(t) if isinstance(t, torch.Tensor) else t for k, t in kw.items()}
    ok = gpu(q_main=q, o_main=q, k_tree=q, v_tree=q, cache=cache, kv_start=torch.zeros(B, dtype=torch.int64), kv_len=torch.zeros(B, dtype=torch.int32),
             kv_capacity=torch.zeros(B, dtype=torch.int32), trees=api.trees_to_device([api.ss_tree_build([-1, 0], 0)] * B, device="cpu"), gamma=0, sm_scale=1.0)
    api.make_kvq_attn_params(**ok)
    for name in ("kv_start", "kv_len", "kv_capacity", "trees"):
        t = ok[name]._t
        bad = [t[:len(t) // 2], torch.stack((t, t), -1)[..., 0]] + ([] if name == "trees" else [t.to(torch.int32 if t.dtype is torch.int64 else torch.int64)])
        for b in bad:
            with pytest.raises(ValueError):
                api.make_kvq_attn_params(**dict(ok, **gpu(**{name: b})))


def test_attention_parameters_keep_the_cache(lib):
    """A cache that only its parameters know is not freed under them."""
    q, i = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int64)
    cache = api.empty_kvq_cache(1, 10, 3, 64, device="cpu")
    parts = [weakref.ref(t) for t in cache.tensors]
    p = api.make_kvq_attn_params(q_main=q, o_main=q, k_tree=q, v_tree=q, cache=cache, kv_start=i, kv_len=i.int(), trees=i, gamma=0, sm_scale=1.0)
    del cache
    gc.collect()
    assert all(r() is not None for r in parts)
    assert p.cache.k_codes == parts[0]().data_ptr()
    del p
    gc.collect()
    assert all(r() is None for r in parts)
