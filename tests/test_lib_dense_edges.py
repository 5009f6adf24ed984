"""CPU: what the dense operators refuse at the ends of their ranges, and what their binding makes of it, before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2107_00961_amd as R
from paper_2107_00961_amd import binding as B

P = 256   # an aligned address that nothing reads
ESHAPE = -2


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("op,m,k,n", [(0, (1 << 31) - 1, 8, 1 << 20), (1, (1 << 31) - 1, 1 << 20, 8), (2, 1000, 1 << 20, 1 << 20)])
def test_more_tiles_than_a_launch_takes_are_refused(op, m, k, n, dt):
    """2^24 workgroups of 256 threads are 2^32, which a launch counts modulo 2^32."""
    sh, size, L = B._LinearShape(m, k, n, 0, 0, dt), C.c_int64(), R.lib()
    assert L.resist_linear_workspace_bytes(C.byref(sh), op, C.byref(size)) == ESHAPE
    call = (L.resist_linear_forward, L.resist_linear_dgrad, L.resist_linear_wgrad)[op]
    last = (None, P, P, 1 << 62, None) if op < 2 else (P, P, P, 1 << 62, None)
    assert call(C.byref(sh), P, P, *last) == ESHAPE
    sh.M = 1 << 20 if op < 2 else 0      # as many as the card could hold
    sh.N, sh.K = min(n, 4096), min(k, 4096)
    assert L.resist_linear_workspace_bytes(C.byref(sh), op, C.byref(size)) == 0


def test_rows_farther_apart_than_dense_layers_take_are_copied():
    for far, copied in (((1 << 20) + 16, True), (1 << 20, False)):
        v = torch.zeros(3, far)[:, :40]
        assert (B._matrix(v, "x", far=B._FAR_LINEAR).data_ptr() != v.data_ptr()) == copied
        assert B._ld(B._matrix(v, "x", far=B._FAR_LINEAR)) == (40 if copied else far)
        assert B._matrix(v, "x").data_ptr() == v.data_ptr()                                     # the operators on rows alone take them
        assert B._matrix(v[:1], "x", far=B._FAR_LINEAR).data_ptr() == v.data_ptr()              # one row has no next one


@pytest.mark.parametrize("n", [1 << 31, (1 << 32) + 8])
def test_widths_past_32_bits_are_refused(n):
    """They would reach the library as what is left of them modulo 2^32."""
    wide, tall = torch.empty(4, n, device="meta"), torch.empty(n, 4, device="meta")
    with pytest.raises(R.ResistError, match=f"rows of {n} elements"):
        B._matrix(wide, "x")
    with pytest.raises(R.ResistError, match=f"w: {n} rows"):
        B._weights(tall, torch.empty(4, 4, device="meta"), K=4)
    assert B._matrix(tall, "x").shape == (n, 4)      # rows are counted in 64 bits, and the library's to refuse


def test_first_calls_of_two_threads(monkeypatch):
    """Whoever finds torch in its place finds everything else that the calls need: it is bound last."""
    seen = []

    class Watched(dict):
        def update(self, *a):
            seen.append(B.torch)
            dict.update(self, *a)

    for name, value in (("torch", None), ("_F32", None), ("_INT64", ()), ("_raw_stream", None), ("_device", None), ("_DTYPES", Watched())):
        monkeypatch.setattr(B, name, value)
    B._start()
    assert seen == [None]
    assert B.torch is torch and B._F32 is torch.float32 and B._INT64 and B._raw_stream and B._device and B._DTYPES[torch.bfloat16] == 1
