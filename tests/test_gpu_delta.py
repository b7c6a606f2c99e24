"""The gated delta rule on the GPU against the token-by-token oracle in 64 bits.

Tolerance: every token rounds each of its sums and products a few times.  The rule does not enlarge errors (decays are at
most 1, and with normalised keys and strengths at most 1 a write does not either), so those of T tokens add up like a
random walk, and those of a sum over k_dim terms as well; operands may be taken as two halves of 11 bits, so a product is off by
2^-22 of itself at most: 2 sqrt(T k_dim) 2^-22 of the largest value of the head.  Outputs of 16 bits are off by half a
step of their type besides."""
import numpy as np
import pytest
import torch

from oracle import delta_oracle as O
from paper_2005_05758_b200 import binding

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def draw(seed, T, Hk, Hv, dk, dv, dtype, slots=0, unit=True, sliced=False):
    """Inputs on the GPU; `sliced`: q, k, v (and the gates) are parts of wider rows."""
    gen = torch.Generator("cuda").manual_seed(seed)
    rows = torch.randn((T, 2 * Hk * dk + Hv * dv), generator=gen, device="cuda")
    if unit:
        keys = rows[:, :2 * Hk * dk].view(T, 2 * Hk, dk)
        keys /= keys.norm(dim=-1, keepdim=True)
    rows = rows.to(TYPES[dtype])
    parts = rows[:, :Hk * dk], rows[:, Hk * dk:2 * Hk * dk], rows[:, 2 * Hk * dk:]
    if not sliced:
        parts = [p.contiguous() for p in parts]
    q, k, v = parts[0].unflatten(1, (Hk, dk)), parts[1].unflatten(1, (Hk, dk)), parts[2].unflatten(1, (Hv, dv))
    gates = torch.empty((T, 2 * Hv), device="cuda")
    gates[:, :Hv] = -torch.exp(torch.rand((T, Hv), generator=gen, device="cuda") * 8 - 7)
    gates[:, Hv:] = torch.sigmoid(torch.randn((T, Hv), generator=gen, device="cuda"))
    g, beta = gates[:, :Hv], gates[:, Hv:]
    if not sliced:
        g, beta = g.contiguous(), beta.contiguous()
    o = torch.full((T, Hv, dv), 7.0, dtype=TYPES[dtype], device="cuda")
    state = torch.randn((slots, Hv, dk, dv), generator=gen, device="cuda") * 0.3 if slots else None
    return dict(q=q, k=k, v=v, g=g, beta=beta, o=o, state=state)


def host(t):
    return None if t is None else t.detach().cpu().double().numpy()


def near(got, want, tokens, k_dim):
    """got [..., rows, columns] of a head against want."""
    want = np.asarray(want)
    eps = {torch.float32: 0.0}.get(got.dtype, torch.finfo(got.dtype).eps / 2)
    have = host(got)
    assert have.shape == want.shape
    assert np.array_equal(np.isfinite(have), np.isfinite(want))
    if not want.size:
        return
    largest = np.max(np.abs(want), axis=(0, -1) if want.ndim == 3 else (-2, -1), keepdims=True)
    tol = 2 * np.sqrt(max(tokens, 1) * k_dim) * 2.0 ** -22 * largest
    tol = tol + (eps * (np.abs(want) + tol) + torch.finfo(got.dtype).tiny if eps else 0)
    worst = np.max(np.abs(have - want) - tol)
    assert worst <= 0, (worst, np.max(np.abs(have - want)))


def check(a, lens, slot=None, fresh=None, normalize=False, scale=None, **more):
    begin = np.concatenate([[0], np.cumsum(lens)])
    args = [host(a[n]) for n in ("q", "k", "v", "g", "beta", "o", "state")]
    want_o, want_S = O.forward(*args, begin, slot, fresh, scale, normalize)
    as_int = lambda v, t: None if v is None else torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
    binding.csb_gated_delta_forward(a["q"], a["k"], a["v"], a["g"], a["beta"], a["o"], a["state"], as_int(begin, torch.int32), as_int(slot, torch.int32),
                                    as_int(fresh, torch.uint8), scale, binding.CSB_FLAG_NORMALIZE if normalize else 0, **more)
    near(a["o"], want_o, max(lens), a["q"].shape[2])
    if want_S is not None:
        near(a["state"].flatten(0, 1), want_S.reshape(-1, *want_S.shape[2:]), max(lens), a["q"].shape[2])


SHAPES = [  # lens, key heads, value heads, k_dim, v_dim
    ([1], 1, 1, 1, 1), ([5, 1, 2], 1, 2, 16, 16), ([31, 32, 33], 2, 2, 64, 64), ([130], 2, 4, 128, 128), ([64, 65, 63, 200], 1, 3, 100, 72),
    ([97], 1, 2, 17, 33), ([40, 260], 2, 2, 256, 64), ([70], 1, 1, 129, 130), ([300], 1, 2, 48, 20), ([1, 1, 1, 1], 4, 4, 32, 8),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens,Hk,Hv,dk,dv", SHAPES)
def test_forward_matches_the_oracle(lens, Hk, Hv, dk, dv, dtype):
    a = draw(sum(lens) + dk, sum(lens), Hk, Hv, dk, dv, dtype, slots=len(lens))
    check(a, lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seed,sequences,longest", [(1, 8, 9), (2, 40, 100), (3, 300, 40), (4, 9, 1), (5, 30, 8)])
def test_requests_that_decode_beside_prompts(seed, sequences, longest, dtype):
    rng = np.random.default_rng(seed)
    lens = rng.choice([0, 1, 1, 1, 2, 7, 8, 9, 31, 32, 33, 64, 100], sequences)
    lens = [int(min(n, longest)) for n in lens]
    lens[-1] = longest
    slot = rng.permutation(sequences + 3)[:sequences].astype(int).tolist()
    slot[2], slot[4] = -1, slot[1]
    a = draw(seed, sum(lens), 1, 2, 64, 40, dtype, slots=sequences + 3)
    check(a, lens, slot=slot, fresh=(rng.random(sequences) < 0.5).astype(int).tolist(), normalize=True)


@pytest.mark.parametrize("lens", [[1] * 200 + [40] + [1] * 100 + [9, 0, 8, 70, 9, 33, 9] + [1] * 60, [33] + [0] * 30 + [9, 9], [2] * 50 + [64], [1] * 12 + [32, 31]])
def test_few_prompts_among_many_tokens(lens):
    a = draw(len(lens), sum(lens), 2, 2, 64, 32, "f16", slots=len(lens))
    check(a, lens)
    need = binding.lib.csb_gated_delta_workspace_bytes(binding.csb_delta_shape_t(1000, 1000, 1000, 16, 32, 128, 128, binding.CSB_BF16, 2048, 2048, 4096, 32, 32, 4096, 0.0))
    assert need < 100 << 20                                      # no record for every sequence


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_slices_of_wider_rows_and_normalisation_and_scale(dtype):
    lens = [50, 3, 129]
    a = draw(5, sum(lens), 2, 4, 64, 48, dtype, slots=5, unit=False, sliced=True)
    check(a, lens, slot=[4, 0, 2], fresh=[0, 1, 0], normalize=True, scale=0.3)


def test_unaligned_rows():
    lens = [45, 90]
    a = draw(6, sum(lens), 2, 2, 64, 64, "f16", slots=2)
    for n in ("q", "k", "v"):                                    # rows that start at odd elements
        wide = torch.zeros((sum(lens), a[n].shape[1] * a[n].shape[2] + 3), dtype=torch.float16, device="cuda")
        wide[:, 1:-2] = a[n].flatten(1)
        a[n] = wide[:, 1:-2].unflatten(1, a[n].shape[1:])
    a["state"] = torch.cat([torch.zeros(1, device="cuda"), a["state"].flatten()])[1:].view(2, 2, 64, 64)
    check(a, lens)


@pytest.mark.parametrize("T", [3, 200])
def test_without_a_pool_and_without_begins(T):
    a = draw(7, T, 1, 2, 64, 64, "f32")
    want, _ = O.forward(*(host(a[n]) for n in ("q", "k", "v", "g", "beta", "o")), None, [0, T])
    binding.csb_gated_delta_forward(a["q"], a["k"], a["v"], a["g"], a["beta"], a["o"])
    near(a["o"], want, T, 64)


@pytest.mark.parametrize("each", [3, 70])
def test_what_a_call_leaves_alone(each):
    # padding slots, one past the pool, one named twice, a sequence without tokens, rows in front of and behind all sequences
    lens, slot = [each, each, 0, each, each, each], [3, -1, 1, 6, 3, 0]
    a = draw(8, sum(lens) + 9, 1, 2, 32, 32, "f32", slots=6)
    begin = np.concatenate([[0], np.cumsum(lens)]) + 4
    args = [host(a[n]) for n in ("q", "k", "v", "g", "beta", "o", "state")]
    want_o, want_S = O.forward(*args, begin, slot)
    before = a["state"].clone()
    binding.csb_gated_delta_forward(a["q"], a["k"], a["v"], a["g"], a["beta"], a["o"], a["state"], torch.tensor(begin, dtype=torch.int32, device="cuda"),
                                    torch.tensor(slot, dtype=torch.int32, device="cuda"))
    near(a["o"], want_o, each, 32)
    near(a["state"].flatten(0, 1), want_S.reshape(-1, 32, 32), each, 32)
    assert torch.equal(a["state"][[1, 2, 4, 5]], before[[1, 2, 4, 5]])
    left = torch.cat([a["o"][:4], a["o"][4 + each:4 + 2 * each], a["o"][4 + 3 * each:4 + 4 * each + each], a["o"][-5:]])
    assert torch.all(left[:4] == 7) and torch.all(left[4:4 + each] == 7) and torch.all(left[-5:] == 7)
    assert torch.all(a["o"][begin[4]:begin[5]] == 7)


def test_nothing_to_do():
    a = draw(9, 0, 1, 1, 16, 16, "f32", slots=2)
    before = a["state"].clone()
    binding.csb_gated_delta_forward(a["q"], a["k"], a["v"], a["g"], a["beta"], a["o"], a["state"], torch.zeros(3, dtype=torch.int32, device="cuda"))
    binding.csb_gated_delta_step(a["q"], a["k"], a["v"], a["g"], a["beta"], a["o"], a["state"])
    assert torch.equal(a["state"], before)
    b = draw(9, 40, 1, 1, 16, 16, "f32")
    binding.csb_gated_delta_forward(b["q"], b["k"], b["v"], b["g"], b["beta"], b["o"], a["state"], torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert torch.all(b["o"] == 7) and torch.equal(a["state"], before)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [6, 150])
def test_gates_at_their_ends(T, dtype):
    a = draw(10, T, 1, 4, 64, 64, dtype, slots=1)
    a["g"][:, 0] = 0.0                                           # nothing is forgotten
    a["g"][:, 1] = -60.0                                         # all is, at every token
    a["g"][T // 2, 2] = -float("inf")                            # all is, once
    a["g"][T // 3, 3] = -3000.0                                  # far below what e^g can hold, then decays next to 1
    a["g"][T // 3 + 1:, 3] = -1e-3
    a["beta"][:, 0] = 1.0
    a["beta"][: T // 2, 1] = 0.0                                 # nothing is written
    check(a, [T])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(64, 48), (128, 33), (200, 20)])
def test_growth_in_some_chunks(dk, dv, dtype):
    a = draw(20, 140, 1, 2, dk, dv, dtype, slots=1)
    a["g"][[5, 40, 41, 90]] = 0.02                               # (the states grow by a few hundredths: no more than the tolerance is for)
    a["beta"][100:] *= -0.1                                      # and writes that take away
    check(a, [140])


def test_a_long_memory():
    a = draw(21, 2500, 1, 1, 128, 16, "f32", slots=1)
    a["g"][:] = -1e-4
    check(a, [2500])


@pytest.mark.parametrize("T", [6, 150])
def test_the_same_key_again_and_zero_keys(T):
    a = draw(11, T, 1, 2, 64, 32, "f32", slots=1)
    a["k"][:] = a["k"][:1].clone()
    a["k"][T // 2] = 0
    a["beta"][:] = 1.0
    check(a, [T])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("scale", [1e-12, 1e12])
def test_values_far_from_one(scale, dtype):
    # magnitudes that 11-bit halves in 16 bits could not hold as they are: of keys and queries, of values and of states
    if dtype == "f16":
        scale = 1e-4 if scale < 1 else 1e3
    a = draw(12, 100, 1, 1, 64, 64, dtype, slots=1, unit=False)
    a["v"].mul_(scale)
    a["state"].mul_(scale)
    a["k"].mul_(1e-3 if scale < 1 else 1e2)
    check(a, [100], normalize=True)


@pytest.mark.parametrize("T,at", [(4, 2), (96, 75), (200, 40)])
@pytest.mark.parametrize("name", ["q", "k", "v", "g", "beta"])
def test_a_nan_reaches_what_it_must_and_nothing_else(name, T, at):
    lens = [T, T, T]
    bad, good = draw(13, 3 * T, 1, 2, 32, 32, "f32", slots=3), draw(13, 3 * T, 1, 2, 32, 32, "f32", slots=3)
    bad[name][T + at].view(-1)[0] = float("nan")
    begin = torch.tensor([0, T, 2 * T, 3 * T], dtype=torch.int32, device="cuda")
    for x in (bad, good):
        binding.csb_gated_delta_forward(x["q"], x["k"], x["v"], x["g"], x["beta"], x["o"], x["state"], begin)
    at += T
    near(bad["o"][:at], host(good["o"][:at]), T, 32)             # what comes before it
    near(bad["o"][2 * T:], host(good["o"][2 * T:]), T, 32)       # the other sequences
    near(bad["state"][[0, 2]].flatten(0, 1), host(good["state"][[0, 2]].flatten(0, 1)), T, 32)
    assert torch.isnan(bad["o"][at]).any()
    if name == "q":
        near(bad["o"][at + 1:2 * T], host(good["o"][at + 1:2 * T]), T, 32)
        near(bad["state"][1], host(good["state"][1]), T, 32)
    else:
        assert torch.isnan(bad["state"][1, 0]).any() and torch.isnan(bad["o"][at + 1, 0]).any()
    if name == "v":                                              # one column of one head
        near(bad["o"][T:2 * T, 1], host(good["o"][T:2 * T, 1]), T, 32)
        near(bad["o"][T:2 * T, :1, 1:], host(good["o"][T:2 * T, :1, 1:]), T, 32)
        near(bad["state"][1, :, :, 1:], host(good["state"][1, :, :, 1:]), T, 32)
    if name in ("g", "beta"):
        near(bad["o"][T:2 * T, 1], host(good["o"][T:2 * T, 1]), T, 32)


def test_nan_behind_the_sequences_is_not_read():
    a = draw(14, 60, 1, 1, 64, 64, "f16", slots=1)
    for n in ("q", "k", "v", "g", "beta"):
        a[n][45:] = float("nan")
    begin = [0, 45]
    want_o, want_S = O.forward(*(host(a[n]) for n in ("q", "k", "v", "g", "beta", "o", "state")), begin)
    binding.csb_gated_delta_forward(a["q"], a["k"], a["v"], a["g"], a["beta"], a["o"], a["state"], torch.tensor(begin, dtype=torch.int32, device="cuda"))
    near(a["o"], want_o, 45, 64)
    near(a["state"][0], want_S[0], 45, 64)


STEPS = [(1, 1, 1, 1, 1), (3, 2, 4, 64, 64), (7, 3, 6, 100, 60), (5, 1, 2, 256, 130), (33, 2, 2, 128, 128), (2, 16, 32, 128, 128), (4, 1, 1, 130, 3)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,Hk,Hv,dk,dv", STEPS)
def test_step_matches_the_oracle(B, Hk, Hv, dk, dv, dtype):
    a = draw(B + dk, B, Hk, Hv, dk, dv, dtype, slots=B + 2, unit=False, sliced=True)
    slot = np.random.default_rng(B).permutation(B + 2)[:B].astype(np.int32)
    if B > 4:
        slot[1], slot[2], slot[4] = -1, B + 2, slot[0]           # padding, past the pool, named twice
    want_o, want_S = O.forward(*(host(a[n]) for n in ("q", "k", "v", "g", "beta", "o", "state")), np.arange(B + 1), slot, normalize=True)
    binding.csb_gated_delta_step(a["q"], a["k"], a["v"], a["g"], a["beta"], a["o"], a["state"], torch.from_numpy(slot).cuda(),
                                 flags=binding.CSB_FLAG_NORMALIZE)
    near(a["o"], want_o, 1, dk)
    near(a["state"].flatten(0, 1), want_S.reshape(-1, dk, dv), 1, dk)


def test_states_past_32_bits_of_elements():
    # a pool of 4200 states of 32 heads of 128 x 128: over 2^31 floats
    n = 4200
    pool = torch.empty((n, 32, 128, 128), device="cuda")
    pool[n - 1].normal_(generator=torch.Generator("cuda").manual_seed(1))
    pool[3].normal_(generator=torch.Generator("cuda").manual_seed(2))
    for T in (1, 40):
        a = draw(15, 2 * T, 16, 32, 128, 128, "bf16")
        slot = torch.tensor([n - 1, 3], dtype=torch.int32, device="cuda")
        want_o, want_S = O.forward(*(host(a[x]) for x in ("q", "k", "v", "g", "beta", "o")), host(pool[[n - 1, 3]]), [0, T, 2 * T])
        if T == 1:
            binding.csb_gated_delta_step(a["q"], a["k"], a["v"], a["g"], a["beta"], a["o"], pool, slot)
        else:
            begin = torch.tensor([0, T, 2 * T], dtype=torch.int32, device="cuda")
            binding.csb_gated_delta_forward(a["q"], a["k"], a["v"], a["g"], a["beta"], a["o"], pool, begin, slot)
        near(a["o"], want_o, T, 128)
        near(pool[[n - 1, 3]].flatten(0, 1), want_S.reshape(-1, 128, 128), T, 128)


def test_a_token_past_32_bits_of_elements():
    H, dv = 40000, 65536
    v, o = torch.zeros((1, H, dv), dtype=torch.float16, device="cuda"), torch.zeros((1, H, dv), dtype=torch.float16, device="cuda")
    v[0, -1], v[0, 0, :5] = 2.0, 3.0
    one, g = torch.ones((1, 1, 1), dtype=torch.float16, device="cuda"), torch.zeros((1, H), device="cuda")
    binding.csb_gated_delta_forward(one, one, v, g, torch.full((1, H), 0.5, device="cuda"), o)
    assert torch.all(o[0, -1] == 1.0) and torch.all(o[0, 0, :5] == 1.5) and torch.all(o[0, 0, 5:] == 0) and torch.all(o[0, -2] == 0)


@pytest.mark.parametrize("lens", [[2, 3], [90, 33]])
def test_bits_are_the_same_again_on_another_stream_and_in_a_graph(lens):
    begin = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")

    def call(x, **more):
        binding.csb_gated_delta_forward(x["q"], x["k"], x["v"], x["g"], x["beta"], x["o"], x["state"], begin, flags=binding.CSB_FLAG_NORMALIZE, **more)
    a, b, c = (draw(16, sum(lens), 2, 4, 128, 64, "bf16", slots=2) for _ in range(3))
    start = a["state"].clone()
    call(a)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    call(b, stream=other)
    other.synchronize()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(c)
    for _ in range(2):
        c["state"].copy_(start)
        c["o"].zero_()
        graph.replay()
    torch.cuda.synchronize()
    for x in (b, c):
        assert torch.equal(x["o"], a["o"]) and torch.equal(x["state"], a["state"])


def test_two_graphs_at_once_have_a_workspace_each():
    graphs, sets, lens = [], [draw(17 + i, 300, 2, 2, 64, 64, "f16", slots=1) for i in range(2)], [300]
    wants = [O.forward(*(host(x[n]) for n in ("q", "k", "v", "g", "beta", "o", "state")), [0, 300]) for x in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for x, st in zip(sets, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            binding.csb_gated_delta_forward(x["q"], x["k"], x["v"], x["g"], x["beta"], x["o"], x["state"])
        graphs.append(graph)
    for graph, st in zip(graphs, streams):
        with torch.cuda.stream(st):
            graph.replay()
    torch.cuda.synchronize()
    for x, (o, S) in zip(sets, wants):
        near(x["o"], o, lens[0], 64)
        near(x["state"][0], S[0], lens[0], 64)


def test_a_prompt_in_pieces_then_token_by_token_is_the_whole_sequence():
    T = 150
    a = draw(18, T, 2, 4, 64, 64, "f32", slots=1)
    want_o, want_S = O.forward(*(host(a[n]) for n in ("q", "k", "v", "g", "beta", "o", "state")), [0, T])
    for lo, hi in ((0, 70), (70, 73), (73, 140)):
        p = {n: a[n][lo:hi] for n in ("q", "k", "v", "g", "beta", "o")}
        binding.csb_gated_delta_forward(*p.values(), a["state"])
    for t in range(140, T):
        p = {n: a[n][t:t + 1] for n in ("q", "k", "v", "g", "beta", "o")}
        binding.csb_gated_delta_step(*p.values(), a["state"])
    near(a["o"], want_o, T, 64)
    near(a["state"][0], want_S[0], T, 64)
