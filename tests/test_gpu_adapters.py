"""The batched product with low-rank adapters on the GPU against the oracle in 64 bits.

Tolerance: an input is taken as two tf32 halves (off by 2^-22 of itself at most), the low-rank values once more; the sums
are fp32 over at most a few thousand terms of either sign, whose partial sums stay far below the sum S of the absolute
values: 2^-19 S covers both by a factor of more than two.  The shared product has its own error, which its tests bound by
1e-5 of its S for the matrices here (values that binary16 holds exactly)."""
import numpy as np
import pytest
import torch

from oracle import adapter_oracle as O
from paper_2005_05758_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def matrix(seed, rows, cols, block=16, dtype="f16", keep=0.5):
    rng = np.random.default_rng(seed)
    nbr, nbc = -(-rows // block), -(-cols // block)
    W = (rng.standard_normal((rows, cols)) * 0.1).astype(np.float16).astype(np.float32)
    rk, ck = ((rng.random(nbr * nbc * block) < keep).astype(np.uint8) for _ in range(2))
    A = binding.csb_encode(W, block, block, rk, ck, dtype)
    mask = (rk.reshape(nbr, nbc, block, 1) * ck.reshape(nbr, nbc, 1, block)).transpose(0, 2, 1, 3).reshape(nbr * block, nbc * block)[:rows, :cols]
    return A, (W * mask).astype(np.float64)


def inputs(seed, rows, cols, batch, count, rank, kind):
    gen = torch.Generator("cuda").manual_seed(seed)
    X = torch.randn((batch, cols), generator=gen, device="cuda")
    down = (torch.randn((count, rank, cols), generator=gen, device="cuda") / np.sqrt(cols)).to(TYPES[kind])
    up = torch.randn((count, rows, rank), generator=gen, device="cuda").to(TYPES[kind])
    which = torch.randint(-1, count + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
    ranks = torch.randint(0, rank + 1, (count,), generator=gen, device="cuda", dtype=torch.int32)
    ranks[0] = rank
    scales = torch.rand((count,), generator=gen, device="cuda") * 2 - 0.5
    return X, down, up, which, ranks, scales


def host(t):
    return None if t is None else t.detach().cpu().double().numpy()


def near(Y, W, X, down, up, which, ranks=None, scales=None):
    add, scale = O.adapters(host(X), host(down), host(up), which.cpu().numpy(), None if ranks is None else ranks.cpu().numpy(), host(scales))
    x = host(X)
    want, tol = x @ W.T + add, 1e-5 * (np.abs(x) @ np.abs(W).T) + 2.0 ** -19 * scale
    worst = np.max(np.abs(host(Y) - want) - tol) if want.size else 0.0
    assert worst <= 0, worst


CASES = [  # rows, cols, batch, adapters, rank, matrix type
    (64, 48, 1, 1, 1, "f16"), (300, 177, 1, 2, 8, "f16"), (512, 192, 5, 3, 12, "f32"), (96, 256, 9, 4, 16, "f16"), (257, 640, 33, 2, 17, "f16"),
    (128, 129, 64, 40, 33, "f16"), (80, 520, 100, 3, 64, "f16"), (48, 64, 20, 2, 100, "f16"), (40, 300, 1100, 5, 9, "f16"), (1030, 72, 3, 1, 256, "f32"),
    (64, 64, 1300, 1, 4, "f16"), (64, 2600, 30, 8, 16, "f16"), (72, 1111, 70, 3, 40, "f16"), (200, 1500, 2, 2, 64, "f32"),
]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,batch,count,rank,dtype", CASES)
def test_matches_the_oracle(rows, cols, batch, count, rank, dtype, kind):
    A, W = matrix(rows + cols, rows, cols, dtype=dtype)
    X, down, up, which, ranks, scales = inputs(batch, rows, cols, batch, count, rank, kind)
    Y = torch.full((batch, rows), float("nan"), device="cuda")
    binding.csb_spmm_adapters(A, X, Y, down, up, which, ranks, scales)
    near(Y, W, X, down, up, which, ranks, scales)
    A.free()


def test_rows_of_wider_tensors_and_no_ranks_or_scales():
    A, W = matrix(1, 100, 96)
    X, down, up, which, _, _ = inputs(2, 100, 96, 12, 3, 20, "f16")
    wide_x, wide_y = torch.zeros((12, 101), device="cuda"), torch.full((12, 107), 5.0, device="cuda")
    wide_x[:, 3:99] = X
    binding.csb_spmm_adapters(A, wide_x[:, 3:99], wide_y[:, 2:102], down, up, which)
    near(wide_y[:, 2:102], W, X, down, up, which)
    assert torch.all(wide_y[:, :2] == 5) and torch.all(wide_y[:, 102:] == 5)
    A.free()


def test_what_is_beyond_a_rank_or_belongs_to_others_is_not_read():
    A, W = matrix(3, 64, 64)
    X, down, up, _, _, scales = inputs(4, 64, 64, 10, 4, 24, "bf16")
    ranks = torch.tensor([24, 5, 0, 16], dtype=torch.int32, device="cuda")
    which = torch.tensor([0, 1, 2, 3, 1, 3, -1, 9, 0, 1], dtype=torch.int32, device="cuda")
    clean = [t.clone() for t in (down, up)]
    for a, r in enumerate(ranks.tolist()):
        down[a, r:], up[a, :, r:] = float("nan"), float("nan")
    Y = torch.empty((10, 64), device="cuda")
    binding.csb_spmm_adapters(A, X, Y, down, up, which, ranks, scales)
    near(Y, W, X, *clean, which, ranks, scales)
    # an adapter of infinities and a request of NaN touch their own rows alone
    down[3], up[3] = float("inf"), float("nan")
    X[1] = float("nan")
    Z = torch.empty((10, 64), device="cuda")
    binding.csb_spmm_adapters(A, X, Z, down, up, which, ranks, scales)
    rest = [0, 2, 4, 6, 7, 8, 9]
    assert torch.equal(Z[rest], Y[rest]) and not torch.isfinite(Z[[1, 3, 5]]).any(1).all()
    A.free()


def test_no_requests_no_adapters_and_plain_rows():
    A, W = matrix(5, 64, 80)
    X, down, up, which, ranks, scales = inputs(6, 64, 80, 16, 2, 8, "f16")
    binding.csb_spmm_adapters(A, X[:0], torch.empty((0, 64), device="cuda"), down, up, which[:0], ranks, scales)
    Y, Z = torch.empty((16, 64), device="cuda"), torch.empty((16, 64), device="cuda")
    binding.csb_spmm_adapters(A, X, Y, down[:0], up[:0], which)
    binding.csb_spmm(A, X, Z)
    assert torch.equal(Y, Z)
    which.fill_(-1)
    binding.csb_spmm_adapters(A, X, Y, down, up, which, ranks, scales)
    assert torch.equal(Y, Z)
    A.free()


def test_inputs_of_any_magnitude():
    # fp32 adapters and inputs far from 1: nothing is held in 16 bits on the adapters' side
    A, W = matrix(7, 64, 64, dtype="f32", keep=0.0)
    X, down, up, which, ranks, scales = inputs(8, 64, 64, 4, 2, 8, "f32")
    for f in (1e-20, 1e20):
        Y = torch.empty((4, 64), device="cuda")
        binding.csb_spmm_adapters(A, X * f, Y, down, up, which, ranks, scales)
        near(Y, W, X * f, down, up, which, ranks, scales)
    A.free()


def test_bits_are_the_same_again_on_another_stream_and_in_a_graph():
    A, W = matrix(9, 200, 128)
    X, down, up, which, ranks, scales = inputs(10, 200, 128, 40, 6, 16, "f16")
    Y, Z, G = (torch.empty((40, 200), device="cuda") for _ in range(3))
    binding.csb_spmm_adapters(A, X, Y, down, up, which, ranks, scales)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    binding.csb_spmm_adapters(A, X, Z, down, up, which, ranks, scales, stream=other)
    other.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.csb_spmm_adapters(A, X, G, down, up, which, ranks, scales)
    G.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(Y, Z) and torch.equal(Y, G)
    near(Y, W, X, down, up, which, ranks, scales)
    A.free()
