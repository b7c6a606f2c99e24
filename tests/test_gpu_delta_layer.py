"""A recurrent layer of the gated delta rule as a server runs it: pruned projections shared by all requests, an adapter of
each request's own beside them, prompts of different lengths in one call, then token by token from the pool of states.
Against the oracles in 64 bits; every output passes two products and the rule, whose tolerances (see their tests) add up
to far less than the 1e-4 of the largest output that is asked for."""
import numpy as np
import pytest
import torch

from oracle import adapter_oracle, delta_oracle
from paper_2005_05758_b200 import binding

pytestmark = pytest.mark.gpu
D, HK, HV, DK, DV, BLOCK, RANK, COUNT = 96, 2, 4, 64, 32, 16, 8, 3
WIDE = 2 * HK * DK + HV * DV + 2 * HV                            # q, k, v and two gates a value head


class Projection:
    """A pruned matrix with a bank of adapters: on the GPU, and as the oracle has it."""

    def __init__(self, rng, rows, cols):
        W = (rng.standard_normal((rows, cols)) / np.sqrt(cols)).astype(np.float16).astype(np.float32)
        nbr, nbc = -(-rows // BLOCK), -(-cols // BLOCK)
        rk, ck = ((rng.random(nbr * nbc * BLOCK) < 0.7).astype(np.uint8) for _ in range(2))
        mask = (rk.reshape(nbr, nbc, BLOCK, 1) * ck.reshape(nbr, nbc, 1, BLOCK)).transpose(0, 2, 1, 3).reshape(nbr * BLOCK, nbc * BLOCK)
        self.W, self.A = (W * mask[:rows, :cols]).astype(np.float64), binding.csb_encode(W, BLOCK, BLOCK, rk, ck, "f16")
        self.down = torch.from_numpy((rng.standard_normal((COUNT, RANK, cols)) / np.sqrt(cols)).astype(np.float16)).cuda()
        self.up = torch.from_numpy((rng.standard_normal((COUNT, rows, RANK)) * 0.3).astype(np.float16)).cuda()

    def __call__(self, X, which):
        Y = torch.empty((X.shape[0], self.W.shape[0]), device="cuda")
        binding.csb_spmm_adapters(self.A, X, Y, self.down, self.up, which)
        return Y

    def oracle(self, X, which):
        return X @ self.W.T + adapter_oracle.adapters(X, self.down.cpu().double().numpy(), self.up.cpu().double().numpy(), which)[0]


def cut(Y):
    """Queries, keys, values and gates as slices of one projection's rows."""
    a, b, c = HK * DK, 2 * HK * DK, 2 * HK * DK + HV * DV
    return Y[:, :a], Y[:, a:b], Y[:, b:c], Y[:, c:c + HV], Y[:, c + HV:]


def close(got, want):
    assert np.max(np.abs(got.cpu().double().numpy() - want)) <= 1e-4 * np.max(np.abs(want))


@pytest.mark.parametrize("lens", [[5, 2, 1], [40, 3, 129]])
def test_prompts_and_then_tokens(lens):
    rng = np.random.default_rng(sum(lens))
    first, last = Projection(rng, WIDE, D), Projection(rng, D, HV * DV)
    users, slots, steps = np.array([2, -1, 0]), np.array([3, 0, 2]), 3
    pool = torch.full((5, HV, DK, DV), float("nan"), device="cuda")   # what a slot held before is not looked at
    begin = np.concatenate([[0], np.cumsum(lens)])
    states = [np.zeros((HV, DK, DV)) for _ in lens]
    for step in range(1 + steps):
        prompt = step == 0
        x = rng.standard_normal((sum(lens) if prompt else len(lens), D)).astype(np.float32)
        which = np.repeat(users, lens) if prompt else users
        as_int = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        X, W = torch.from_numpy(x).cuda(), as_int(which)
        q, k, v, ga, gb = cut(first(X, W))
        g, beta, o = -torch.nn.functional.softplus(ga), torch.sigmoid(gb), torch.empty((X.shape[0], HV, DV), device="cuda")
        heads = (q.unflatten(1, (HK, DK)), k.unflatten(1, (HK, DK)), v.unflatten(1, (HV, DV)), g, beta, o, pool)
        if prompt:
            binding.csb_gated_delta_forward(*heads, as_int(begin), as_int(slots), torch.ones(3, dtype=torch.uint8, device="cuda"), flags=binding.CSB_FLAG_NORMALIZE)
        else:
            binding.csb_gated_delta_step(*heads, as_int(slots), flags=binding.CSB_FLAG_NORMALIZE)
        Y = last(o.flatten(1), W)
        # the same in 64 bits
        q, k, v, ga, gb = cut(first.oracle(x.astype(np.float64), which))
        q, k = delta_oracle.normalised(q.reshape(-1, HK, DK)), delta_oracle.normalised(k.reshape(-1, HK, DK))
        want = np.zeros((len(x), HV, DV))
        for i in range(len(lens)):
            at = slice(begin[i], begin[i + 1]) if prompt else slice(i, i + 1)
            want[at], states[i] = delta_oracle.sequence(q[at], k[at], v[at].reshape(-1, HV, DV), -np.log1p(np.exp(ga[at])), 1 / (1 + np.exp(-gb[at])), states[i],
                                                        1 / np.sqrt(DK))
        close(o, want)
        close(Y, last.oracle(want.reshape(len(x), -1), which))
        for i, slot in enumerate(slots):
            close(pool[slot], states[i])
    assert torch.isnan(pool[[1, 4]]).all()
    first.A.free()
    last.A.free()
