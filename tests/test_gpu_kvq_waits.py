"""Waits of the 4-bit attention's tcgen05 kernel that run out: the call ends, says so, and leaves the stream usable."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_kvq import Layer, api  # noqa: F401  (api is a fixture)

pytestmark = pytest.mark.gpu

# one sequence in pieces, whole heads in turn, streams with more than one block, a ragged batch
CALLS = {"pieces": dict(B=1, H=4, lens=[1500], nodes=40, gamma=0), "whole": dict(B=1, H=500, lens=[200], nodes=20, gamma=0),
         "streams": dict(B=2, H=8, lens=[700, 30], nodes=40, gamma=3), "ragged": dict(B=24, H=8, lens=[100 + 61 * b for b in range(24)], nodes=64, gamma=0)}


def _in_host_memory(api, x):
    """The same cache with its codes in pinned host memory, which the GPU reads in place: a tile's codes take tens of microseconds."""
    kc, kp, vc, vp = x.cache.tensors
    far = api.KvqCache.from_buffer_copy(x.cache)
    far.tensors = (kc.cpu().pin_memory(), kp, vc.cpu().pin_memory(), vp)
    assert far.tensors[0].stride()[1:] == kc.stride()[1:]      # (one layer)
    far.k_codes, far.v_codes = far.tensors[0].data_ptr(), far.tensors[2].data_ptr()
    return far


@pytest.mark.parametrize("name", list(CALLS))
def test_a_call_whose_waits_run_out_ends_and_says_so(api, name):
    c = CALLS[name]
    x = Layer(api, c["B"], c["H"], 128, c["lens"], [c["nodes"]] * c["B"], c["gamma"], seed=9)
    near, x.cache = x.cache, _in_host_memory(api, x)
    ws = x.workspace()
    words = ws.view(torch.int32)
    seen = []
    for _ in range(10):
        words.zero_()
        words[1] = 1                                           # 1024 cycles
        api.ss_msa_attention_kvq(x.params(ws))
        torch.cuda.synchronize()
        seen.append(api.ss_status(ws))
    assert set(seen) <= {0, api.SS_ERR_DEVICE_TIMEOUT}
    assert api.SS_ERR_DEVICE_TIMEOUT in seen
    words.zero_()
    far = x.cache
    for cache in (near, far):                                  # with the default bound, wherever the codes lie
        x.cache = cache
        x.fresh()
        x.run(ws)
        x.cache = near
        x.check([0, x.B - 1])


@pytest.mark.parametrize("name", list(CALLS))
def test_what_a_call_writes_whose_waits_run_out(api, name):
    """Every row is either as it was or what it should be: nothing that a CTA that gave up has left reaches an output, not through the
    partial rows of the CTAs that share its heads either."""
    c = CALLS[name]
    x = Layer(api, c["B"], c["H"], 128, c["lens"], [c["nodes"]] * c["B"], c["gamma"], seed=9)
    ws = x.workspace()
    words = ws.view(torch.int32)
    x.run(ws)
    x.check([0, x.B - 1])
    want = [None if t is None else t.clone() for t in (x.o_main, x.o_spec, x.lse_main, x.lse_spec)]
    x.cache = _in_host_memory(api, x)
    for limit in (1, 8, 16, 32, 64, 128):                      # (longer bounds run out in some CTAs only)
        for _ in range(4):
            x.fresh()
            words.zero_()
            words[1] = limit
            api.ss_msa_attention_kvq(x.params(ws))
            torch.cuda.synchronize()
            assert api.ss_status(ws) in (0, api.SS_ERR_DEVICE_TIMEOUT)
            for t, w in zip((x.o_main, x.o_spec, x.lse_main, x.lse_spec), want):
                if t is not None:
                    assert ((t == w) | (t == 77.0)).all(), (limit, int(((t != w) & (t != 77.0)).sum()))
