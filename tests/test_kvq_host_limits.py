"""Host-side checks of the cache in 4 bits: what its calls refuse before any launch, sizes and tensors at the edge of what they take."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_2402_11131_b200 import api
from test_kvq_host import P, _fake_cache, _fake_params, _fake_rows, lib  # noqa: F401  (lib is a fixture)


def test_calls_refuse_slabs_beyond_their_index_arithmetic(lib):
    c, r = _fake_cache(total_slots=(1 << 48) + 1), _fake_rows()
    assert lib.ss_kvq_write(C.byref(r), C.byref(c), P, P, None, None, None, None, None, None) == api.SS_ERR_INVALID_ARG
    assert lib.ss_kvq_read(C.byref(c), C.byref(r), P, None, None, None) == api.SS_ERR_INVALID_ARG
    assert lib.ss_msa_attention_kvq(C.byref(_fake_params(cache=c)), None) == api.SS_ERR_INVALID_ARG
