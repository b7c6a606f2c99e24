"""What csb_spmm_adapters and csb_gated_delta_* refuse (no GPU: by their arguments, with made-up pointers that are never
followed), and what their binding refuses."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2005_05758_b200 import binding
from paper_2005_05758_b200.binding import lib

FAKE, BIG = 4096, 1 << 40
INVALID, SHAPE, DTYPE, UNSUPPORTED = -1, -2, -3, -8


def shape(**changed):
    s = dict(tokens=10, slots=4, sequences=3, k_heads=2, v_heads=4, k_dim=64, v_dim=32, dtype=binding.CSB_F16, ldq=128, ldk=128, ldv=128, ldg=4, ldb=4,
             ldo=128, scale=0.0)
    s.update(changed)
    return binding.csb_delta_shape_t(*s.values())


def forward(s, q=FAKE, k=FAKE, v=FAKE, g=FAKE, beta=FAKE, o=FAKE, state=FAKE, begin=FAKE, ws=FAKE, size=BIG, flags=0):
    return lib.csb_gated_delta_forward(C.byref(s) if s else None, q, k, v, g, beta, o, state, begin, None, None, ws, size, flags, None)


def step(s, q=FAKE, state=FAKE, flags=0):
    return lib.csb_gated_delta_step(C.byref(s) if s else None, q, FAKE, FAKE, FAKE, FAKE, FAKE, state, None, flags, None)


@pytest.mark.parametrize("changed,status", [
    (dict(tokens=-1), INVALID), (dict(sequences=-1), INVALID), (dict(slots=-1), INVALID), (dict(k_heads=0), INVALID), (dict(k_dim=0), INVALID),
    (dict(v_dim=-3), INVALID), (dict(dtype=2), DTYPE), (dict(dtype=9), DTYPE), (dict(k_heads=3), SHAPE), (dict(ldq=127), SHAPE), (dict(ldk=1), SHAPE),
    (dict(ldv=127), SHAPE), (dict(ldo=0), SHAPE), (dict(ldg=3), SHAPE), (dict(ldb=3), SHAPE), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(k_dim=257, ldq=600, ldk=600), UNSUPPORTED), (dict(tokens=1 << 31), UNSUPPORTED),
    (dict(v_dim=70000, ldv=1 << 20, ldo=1 << 20), UNSUPPORTED), (dict(k_heads=1, v_heads=70000, ldv=1 << 24, ldo=1 << 24, ldg=70000, ldb=70000), UNSUPPORTED)])
def test_shapes_that_are_refused(changed, status):
    assert forward(shape(**changed)) == status and lib.csb_last_error()
    if "tokens" not in changed and "sequences" not in changed:
        assert step(shape(tokens=3, **changed)) == status


def test_missing_arguments_and_flags():
    assert forward(None) == INVALID and step(None) == INVALID
    for name in ("q", "k", "v", "g", "beta", "o"):
        assert forward(shape(), **{name: None}) == INVALID, name
    assert forward(shape(), begin=None) == INVALID               # with more than one sequence
    assert forward(shape(), flags=1) == INVALID and forward(shape(), flags=8) == INVALID and step(shape(tokens=3), flags=2) == INVALID
    assert step(shape(tokens=3), state=None) == INVALID and step(shape()) == SHAPE
    assert lib.csb_gated_delta_workspace_bytes(None) == 0
    need = lib.csb_gated_delta_workspace_bytes(C.byref(shape(tokens=5000)))
    assert need > 0 and forward(shape(tokens=5000), size=need - 1) == INVALID and b"workspace" in lib.csb_last_error()
    assert forward(shape(tokens=5000), ws=None) == INVALID
    assert forward(shape(tokens=5000), ws=FAKE + 8) == INVALID and b"aligned" in lib.csb_last_error()
    assert lib.csb_gated_delta_workspace_bytes(C.byref(shape(tokens=8))) == 0      # all short: token by token


def test_nothing_to_do_needs_no_pointers():
    none = dict(q=None, k=None, v=None, g=None, beta=None, o=None, state=None, begin=None, ws=None, size=0)
    assert forward(shape(tokens=0), **none) == 0 and forward(shape(sequences=0), **none) == 0
    assert step(shape(tokens=0, sequences=0), q=None, state=None) == 0


def host_matrix(val_dtype="f16"):
    W, keep = np.ones((8, 12), np.float32), np.ones(6 * 4, np.uint8)
    if val_dtype == "q16":
        return binding.csb_encode_q16(W, 4, 4, keep, keep, 4, -1)
    return binding.csb_encode(W, 4, 4, keep, keep, val_dtype, -1)


def adapters(A, X=FAKE, ldx=12, batch=2, Y=FAKE, ldy=8, dtype=1, count=2, rank=4, down=FAKE, up=FAKE, which=FAKE, ws=FAKE, size=BIG):
    return lib.csb_spmm_adapters(A.handle if A else None, X, ldx, batch, Y, ldy, dtype, count, rank, down, up, which, None, None, ws, size, None)


def test_adapters_that_are_refused():
    A = host_matrix()
    assert adapters(None) == INVALID
    for changed in (dict(batch=-1), dict(count=-1), dict(rank=0), dict(X=None), dict(Y=None), dict(which=None), dict(down=None), dict(up=None), dict(ws=None),
                    dict(size=1), dict(ws=FAKE + 2)):
        assert adapters(A, **changed) == INVALID, changed
    assert adapters(A, dtype=2) == DTYPE and adapters(A, dtype=-1) == DTYPE
    assert adapters(A, ldx=11) == SHAPE and adapters(A, ldy=7) == SHAPE
    assert adapters(A, rank=257) == UNSUPPORTED
    assert adapters(A) == UNSUPPORTED and b"host-only" in lib.csb_last_error()
    assert adapters(A, batch=0, X=None, Y=None, which=None) == 0
    assert lib.csb_adapters_workspace_bytes(A.handle, 2, 4) >= 2 * 16 * 4
    assert lib.csb_adapters_workspace_bytes(A.handle, 0, 4) == 0 and lib.csb_adapters_workspace_bytes(None, 2, 4) == 0
    A.free()


def test_tensors_that_the_binding_refuses():
    A, f = host_matrix(), torch.zeros
    which = f(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="cpu"):
        binding.csb_spmm_adapters(A, f(2, 12), f(2, 8), f(1, 4, 12), f(1, 8, 4), which)
    with pytest.raises(ValueError, match="shape"):
        binding.csb_spmm_adapters(A, f(2, 11), f(2, 8), f(1, 4, 12), f(1, 8, 4), which)
    with pytest.raises(TypeError, match="down"):
        binding.csb_spmm_adapters(A, f(2, 12), f(2, 8), f(1, 4, 12, dtype=torch.float64), f(1, 8, 4), which)
    q = f(5, 2, 16)
    with pytest.raises(TypeError, match="q"):
        binding.csb_gated_delta_step(q.int(), q, q, f(5, 2), f(5, 2), q, f(5, 2, 16, 16))
    with pytest.raises(ValueError, match="cpu"):
        binding.csb_gated_delta_forward(q, q, q, f(5, 2), f(5, 2), q)
    A.free()
