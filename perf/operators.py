"""What is timed of the operators that serve recurrent language models: work that such a program has them do.

Three kinds of pass:
  adapters  csb_spmm_adapters: the product of an encoded matrix with a batch of requests, each with the low-rank
            adapter of its own (or none) beside the shared matrix
  delta     csb_gated_delta_forward: the gated delta rule over packed sequences of different lengths
  step      csb_gated_delta_step: the gated delta rule for one token of each of many requests, their states in a pool

Weights, adapters and inputs are drawn from the seed on the GPU.  Keys and queries are random directions; decays are
those of a gate exp(-A dt) with A in 0.5 .. 16 a head and dt in 0.001 .. 0.1 a token, so heads forget within one token
to two thousand; write strengths are logistic.  With `own` false the operators are computed from elementary torch
operations in 32 bits (the sums of log-decays in 64).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6             # under the root of the normalisation of queries and keys
CHUNK = 64             # tokens that the plain form takes at a time


def listed():
    return [
        # one frame of a speech model's large layer with a small adapter: the smallest call
        {"name": "adapters_1x4096x1177_r8", "op": "adapters", "rows": 4096, "cols": 1177, "block": 32, "rate": 8.16, "dtype": "f16", "kind": "f16",
         "batch": 1, "count": 1, "rank": 8, "bare": 0.0},
        # a full-precision layer and adapters, a handful of requests
        {"name": "adapters_5x512x192_r12_f32", "op": "adapters", "rows": 512, "cols": 192, "block": 16, "rate": 4.0, "dtype": "f32", "kind": "f32",
         "batch": 5, "count": 3, "rank": 12, "bare": 0.2},
        # decoding for many users at once, adapters of several ranks, some requests without one
        {"name": "adapters_48x8192x4096_r16", "op": "adapters", "rows": 8192, "cols": 4096, "block": 64, "rate": 10.0, "dtype": "f16", "kind": "bf16",
         "batch": 48, "count": 24, "rank": 16, "bare": 0.1},
        # prompts of a few users, a few hundred tokens in one call
        {"name": "adapters_395x4096x2048_r64", "op": "adapters", "rows": 4096, "cols": 2048, "block": 64, "rate": 8.0, "dtype": "f16", "kind": "f16",
         "batch": 395, "count": 4, "rank": 64, "bare": 0.1},
        # three short prompts, full precision (slices of one projection's output), small heads
        {"name": "delta_3x40_4h64_f32", "op": "delta", "lens": "1,37,64", "k_heads": 4, "v_heads": 4, "k_dim": 64, "v_dim": 64, "dtype": "f32",
         "sliced": True, "normalize": True, "carried": False},
        # uneven head sizes in full precision, states carried on from earlier chunks of the prompts
        {"name": "delta_4x375_8h100x72_f32", "op": "delta", "lens": "700,33,511,255", "k_heads": 4, "v_heads": 8, "k_dim": 100, "v_dim": 72,
         "dtype": "f32", "sliced": True, "normalize": False, "carried": True},
        # a serving step that takes prompts of many lengths together, some of them continued
        {"name": "delta_12x470_8x16h128_f16", "op": "delta", "lens": "5,1300,64,127,129,900,31,1,777,1000,256,1057", "k_heads": 8, "v_heads": 16,
         "k_dim": 128, "v_dim": 128, "dtype": "f16", "sliced": True, "normalize": True, "carried": True},
        # one long prompt
        {"name": "delta_1x8192_16x32h128_bf16", "op": "delta", "lens": "8192", "k_heads": 16, "v_heads": 32, "k_dim": 128, "v_dim": 128,
         "dtype": "bf16", "sliced": False, "normalize": True, "carried": False},
        # one token of one request
        {"name": "step_1_16x32h128_bf16", "op": "step", "batch": 1, "k_heads": 16, "v_heads": 32, "k_dim": 128, "v_dim": 128, "dtype": "bf16",
         "normalize": True, "idle": 0.0},
        # a few requests, full precision, uneven head sizes
        {"name": "step_7_3x6h100x60_f32", "op": "step", "batch": 7, "k_heads": 3, "v_heads": 6, "k_dim": 100, "v_dim": 60, "dtype": "f32",
         "normalize": False, "idle": 0.0},
        # an ordinary decoding batch
        {"name": "step_61_16x32h128_bf16", "op": "step", "batch": 61, "k_heads": 16, "v_heads": 32, "k_dim": 128, "v_dim": 128, "dtype": "bf16",
         "normalize": True, "idle": 0.0},
        # a large decoding batch, padded to its captured size
        {"name": "step_256_16x32h128_f16", "op": "step", "batch": 256, "k_heads": 16, "v_heads": 32, "k_dim": 128, "v_dim": 128, "dtype": "f16",
         "normalize": True, "idle": 0.1},
    ]


def _between(rng, lo, hi):
    """A whole number, spread over the logarithm of the range, odd ones among them."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["adapters", "delta", "step"])
    if op == "adapters":
        full = rng.random() < 0.25
        return {"op": op, "rows": _between(rng, 256, 4096), "cols": _between(rng, 128, 4096), "block": rng.choice([16, 32, 64]),
                "rate": round(rng.uniform(4.0, 20.0), 2), "dtype": "f32" if full else "f16", "kind": "f32" if full else rng.choice(["f16", "bf16"]),
                "batch": _between(rng, 1, 16 if full else 300), "count": _between(rng, 1, 24), "rank": _between(rng, 4, 64), "bare": rng.choice([0.0, 0.1, 0.5])}
    k_heads = rng.choice([1, 2, 4, 8, 16])
    heads = {"k_heads": k_heads, "v_heads": k_heads * rng.choice([1, 2]), "k_dim": rng.choice([64, 128, 128, _between(rng, 16, 128)]),
             "v_dim": rng.choice([64, 128, 128, _between(rng, 16, 128)]), "dtype": rng.choice(["bf16", "f16", "f32"]), "normalize": rng.random() < 0.7}
    if op == "step":
        return {"op": op, "batch": _between(rng, 1, 256), **heads, "idle": rng.choice([0.0, 0.1, 0.3])}
    # several sequences up to about five thousand tokens in all, or a longer one
    longest = _between(rng, 1, 1500)
    lens = [_between(rng, 1, longest) for _ in range(_between(rng, 1, 24))] if rng.random() < 0.8 else [_between(rng, 1500, 6000)]
    while sum(lens) > 6000:
        lens.pop()
    return {"op": op, "lens": ",".join(map(str, lens)), **heads, "sliced": rng.random() < 0.5, "carried": rng.random() < 0.5}


def _lens(case):
    return [int(n) for n in case["lens"].split(",")]


def _ranks(case):
    """Every third adapter has the full rank, the others three quarters and half of it."""
    return [max(1, case["rank"] - (a % 3) * (case["rank"] // 4)) for a in range(case["count"])]


def _kept(gen, case):
    """Keep masks of every block's rows and columns: as csb_encode takes them, and the mask of the dense matrix."""
    b, R, C = case["block"], case["rows"], case["cols"]
    nbr, nbc = -(-R // b), -(-C // b)

    def lines():
        want = torch.round(b / math.sqrt(case["rate"]) * (0.7 + 0.6 * torch.rand((nbr * nbc, 1), generator=gen, device="cuda")))
        rank = torch.rand((nbr * nbc, b), generator=gen, device="cuda").argsort(dim=1).argsort(dim=1)
        return (rank < want).to(torch.uint8)
    rows, cols = lines(), lines()
    mask = rows.view(nbr, nbc, b, 1) * cols.view(nbr, nbc, 1, b)
    return rows, cols, mask.permute(0, 2, 1, 3).reshape(nbr * b, nbc * b)[:R, :C]


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    s = {"case": case}

    def randn(*shape, std=1.0):
        return torch.randn(shape, generator=gen, device="cuda") * std

    def rand(*shape):
        return torch.rand(shape, generator=gen, device="cuda")
    if case["op"] == "adapters":
        R, C, n, r, kind = case["rows"], case["cols"], case["count"], case["rank"], TYPES[case["kind"]]
        rows, cols, mask = _kept(gen, case)
        s["W"] = (randn(R, C, std=0.05) * mask).to(TYPES[case["dtype"]]).float()
        if own:                                     # the handle that a program keeps of its pruned weight
            from paper_2005_05758_b200 import binding
            s["A"] = binding.csb_encode(s["W"].cpu().numpy(), case["block"], case["block"], rows.cpu().numpy(), cols.cpu().numpy(), case["dtype"])
        s["down"], s["up"] = randn(n, r, C, std=1 / math.sqrt(C)).to(kind), randn(n, R, r, std=0.1).to(kind)
        s["ranks"] = torch.tensor(_ranks(case), dtype=torch.int32, device="cuda")
        s["scales"] = 0.5 + 2 * rand(n)
        which = (rand(case["batch"]) * n).to(torch.int32).clamp(max=n - 1)
        s["which"] = torch.where(rand(case["batch"]) < case["bare"], torch.full_like(which, -1), which)
        s["X"], s["Y"] = randn(case["batch"], C), torch.empty((case["batch"], R), device="cuda")
        return s
    Hk, Hv, dk, dv, t = case["k_heads"], case["v_heads"], case["k_dim"], case["v_dim"], TYPES[case["dtype"]]
    T = sum(_lens(case)) if case["op"] == "delta" else case["batch"]
    qkv = randn(T, 2 * Hk * dk + Hv * dv)
    if not case["normalize"]:                       # directions that the program has normalised already
        keys = qkv[:, :2 * Hk * dk].view(T, 2 * Hk, dk)
        keys /= keys.norm(dim=-1, keepdim=True)
    qkv = qkv.to(t)
    parts = [qkv[:, :Hk * dk], qkv[:, Hk * dk:2 * Hk * dk], qkv[:, 2 * Hk * dk:]]
    if not case.get("sliced", True):
        parts = [p.contiguous() for p in parts]
    s["q"], s["k"], s["v"] = parts[0].unflatten(1, (Hk, dk)), parts[1].unflatten(1, (Hk, dk)), parts[2].unflatten(1, (Hv, dv))
    s["g"] = -(0.5 + 15.5 * rand(Hv)) * torch.exp(math.log(0.001) + math.log(100.0) * rand(T, Hv))
    s["beta"] = torch.sigmoid(randn(T, Hv))
    s["o"] = torch.zeros((T, Hv, dv), dtype=t, device="cuda")
    n = len(_lens(case)) if case["op"] == "delta" else T
    s["state"] = randn(n + 2, Hv, dk, dv, std=0.2)  # a pool with room for more
    s["slots"] = torch.randperm(n + 2, generator=gen, device="cuda")[:n].to(torch.int32)
    if case["op"] == "step":
        s["slots"] = torch.where(rand(n) < case["idle"], torch.full_like(s["slots"], -1), s["slots"])
    else:
        begin = [0]
        for length in _lens(case):
            begin.append(begin[-1] + length)
        s["begin"] = torch.tensor(begin, dtype=torch.int32, device="cuda")
        s["longest"] = max(_lens(case))
        s["fresh"] = (torch.arange(n, device="cuda") % 3 != 0).to(torch.uint8) if case["carried"] else torch.ones(n, dtype=torch.uint8, device="cuda")
    return s


def _adapters(s):
    """All adapters' products at once, those of other requests masked out."""
    n, r = s["down"].shape[:2]
    which, at = s["which"].long(), torch.arange(n, device="cuda")
    weight = (which[:, None] == at).float() * s["scales"]
    weight = weight[:, :, None] * (torch.arange(r, device="cuda") < s["ranks"][:, None]).float()
    low = s["X"] @ s["down"].float().flatten(0, 1).T * weight.flatten(1)
    return s["X"] @ s["W"].T + low @ s["up"].float().permute(0, 2, 1).flatten(0, 1)


def _queries_keys(s):
    """In 32 bits, normalised where asked, a key head for every value head, queries scaled."""
    each = s["case"]["v_heads"] // s["case"]["k_heads"]
    q, k = s["q"].float(), s["k"].float()
    if s["case"]["normalize"]:
        q, k = (x * torch.rsqrt((x * x).sum(-1, keepdim=True) + EPS) for x in (q, k))
    return (q / math.sqrt(s["case"]["k_dim"])).repeat_interleave(each, dim=1), k.repeat_interleave(each, dim=1)


def _step(s):
    q, k = _queries_keys(s)
    live = s["slots"] >= 0
    slots = torch.where(live, s["slots"], len(s["state"]) - 1).long()
    S = s["state"][slots] * torch.exp(s["g"])[:, :, None, None]
    write = s["beta"][:, :, None] * (s["v"].float() - (k[:, :, None, :] @ S)[:, :, 0])
    S = S + k[:, :, :, None] * write[:, :, None, :]
    o = (q[:, :, None, :] @ S)[:, :, 0]
    s["o"].copy_(torch.where(live[:, None, None], o, s["o"].float()))
    at = torch.arange(len(s["state"]), device="cuda")
    took = (slots[:, None] == at) & live[:, None]   # which request, if any, holds each slot of the pool
    s["state"].copy_(torch.where(took.any(0)[:, None, None, None], S[took.int().argmax(0)], s["state"]))
    return s["o"], s["state"]


def _delta(s):
    """Chunks of tokens: within one the rule is a triangular system, from one to the next the state is carried."""
    begin, pad = s["begin"].long(), -(-s["longest"] // CHUNK) * CHUNK
    at = begin[:-1, None] + torch.arange(pad, device="cuda")
    there = at < begin[1:, None]
    at = torch.where(there, at, 0)

    def cut(x):                                     # [T, H, ...] -> [N, H, chunks, CHUNK, ...], zeros behind the end
        x = x[at] * there.view(*there.shape, *[1] * (x.dim() - 1)).to(x.dtype)
        return x.unflatten(1, (-1, CHUNK)).movedim(3, 1)
    q, k = (cut(x) for x in _queries_keys(s))
    v, beta, g = cut(s["v"].float()), cut(s["beta"]), cut(s["g"].double()).cumsum(-1)
    past = torch.ones((CHUNK, CHUNK), dtype=torch.bool, device="cuda").tril()
    decay = torch.exp((g[..., :, None] - g[..., None, :]).masked_fill(~past, -math.inf)).float()
    from_start, to_end, whole = torch.exp(g).float()[..., None], torch.exp(g[..., -1:] - g).float()[..., None], torch.exp(g[..., -1]).float()
    lower = (-beta[..., None] * (k @ k.mT) * decay).tril(-1)
    eye = torch.eye(CHUNK, device="cuda")
    solve, power, done = eye + lower, lower, 2      # the inverse of 1 - lower, as a product of 1 + lower^(2^i)
    while done < CHUNK:
        power = power @ power
        solve, done = solve + solve @ power, 2 * done
    solve = solve * beta[..., None, :]
    u, w = solve @ v, solve @ (k * from_start)
    inner, q, k = (q @ k.mT) * decay, q * from_start, (k * to_end).mT
    slots = s["slots"].long()
    S = s["state"][slots] * (s["fresh"] == 0).float()[:, None, None, None]
    outs = []
    for c in range(pad // CHUNK):
        new = u[:, :, c] - w[:, :, c] @ S
        outs.append(q[:, :, c] @ S + inner[:, :, c] @ new)
        S = whole[:, :, c, None, None] * S + k[:, :, c] @ new
    s["state"][slots] = S
    o = torch.stack(outs, 2).movedim(1, 3).flatten(1, 2)
    s["o"].copy_(o[there])
    return s["o"], s["state"]


def run(state):
    s = state
    if own:
        from paper_2005_05758_b200 import binding
        flags = binding.CSB_FLAG_NORMALIZE if s["case"].get("normalize") else 0
        if s["case"]["op"] == "adapters":
            binding.csb_spmm_adapters(s["A"], s["X"], s["Y"], s["down"], s["up"], s["which"], s["ranks"], s["scales"])
            return s["Y"]
        if s["case"]["op"] == "step":
            binding.csb_gated_delta_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["o"], s["state"], s["slots"], flags=flags)
        else:
            binding.csb_gated_delta_forward(s["q"], s["k"], s["v"], s["g"], s["beta"], s["o"], s["state"], s["begin"], s["slots"], s["fresh"], flags=flags)
        return s["o"], s["state"]
    return {"adapters": _adapters, "step": _step, "delta": _delta}[s["case"]["op"]](s)


def exact(case, seed):
    """From the definitions, in 64 bits: request by adapter, and token by token."""
    s = prepare(case, seed)
    if case["op"] == "adapters":
        X, Y, ranks = s["X"].double(), s["X"].double() @ s["W"].double().T, _ranks(case)
        for a in range(case["count"]):
            mine = torch.nonzero(s["which"] == a)[:, 0]
            r = ranks[a]
            Y[mine] += float(s["scales"][a]) * torch.einsum("ir,rc,bc->bi", s["up"][a, :, :r].double(), s["down"][a, :r].double(), X[mine])
        return Y
    q, k, v, g, beta = (s[name].double() for name in ("q", "k", "v", "g", "beta"))
    if case["normalize"]:
        q, k = q / (q.square().sum(-1, keepdim=True) + EPS).sqrt(), k / (k.square().sum(-1, keepdim=True) + EPS).sqrt()
    of = torch.arange(case["v_heads"], device="cuda") // (case["v_heads"] // case["k_heads"])
    q, k = q[:, of] * case["k_dim"] ** -0.5, k[:, of]
    o, pool, slots = s["o"].double(), s["state"].double(), s["slots"].tolist()
    if case["op"] == "step":
        runs = [(b, 1, False) for b in range(case["batch"])]
    else:
        runs = [(b, n, f != 0) for b, n, f in zip(s["begin"].tolist(), _lens(case), s["fresh"].tolist())]
    live = [i for i, slot in enumerate(slots) if slot >= 0]
    if not live:
        return o, pool
    first, length = torch.tensor([runs[i][0] for i in live], device="cuda"), torch.tensor([runs[i][1] for i in live])
    S = pool[[slots[i] for i in live]]
    S[[j for j, i in enumerate(live) if runs[i][2]]] = 0
    order = torch.argsort(length, descending=True)  # the sequences that still run stand in front
    first, length, S = first[order.cuda()], length[order], S[order.cuda()]
    count = [int((length > t).sum()) for t in range(int(length[0]))]
    for t, n in enumerate(count):
        at, A = first[:n] + t, S[:n]
        A *= g[at].exp()[:, :, None, None]
        seen = (A * k[at][:, :, :, None]).sum(2)
        A += k[at][:, :, :, None] * (beta[at][:, :, None] * (v[at] - seen))[:, :, None, :]
        o[at] = (A * q[at][:, :, :, None]).sum(2)
    pool[torch.tensor([slots[live[j]] for j in order.tolist()], device="cuda")] = S
    return o, pool


def _tokens_bytes(case, tokens):
    size = 4 if case["dtype"] == "f32" else 2
    return tokens * (size * 2 * (case["k_heads"] * case["k_dim"] + case["v_heads"] * case["v_dim"]) + 8 * case["v_heads"])


def work(case):
    """Inputs read once and outputs written once; the adapters, and states, that a pass is expected to touch."""
    if case["op"] == "adapters":
        R, C, B, n = case["rows"], case["cols"], case["batch"], case["count"]
        ranks, size = _ranks(case), 4 if case["kind"] == "f32" else 2
        touched = 1 - (1 - (1 - case["bare"]) / n) ** B
        values, blocks = R * C / case["rate"], R * C / case["block"] ** 2
        weight = values * (4 if case["dtype"] == "f32" else 2) + blocks * (6 + 2 * case["block"] / math.sqrt(case["rate"]))
        mean = sum(ranks) / n
        return {"bytes": weight + touched * sum(ranks) * (R + C) * size + 4 * B * (R + C), "flops": 2 * values * B + 2 * (1 - case["bare"]) * B * mean * (R + C)}
    cells = case["v_heads"] * case["k_dim"] * case["v_dim"]
    if case["op"] == "step":
        live = case["batch"] * (1 - case["idle"])
        return {"bytes": _tokens_bytes(case, live) + 8 * cells * live, "flops": 7 * cells * live}
    lens = _lens(case)
    states = len(lens) + (len(range(0, len(lens), 3)) if case["carried"] else 0)
    return {"bytes": _tokens_bytes(case, sum(lens)) + 4 * cells * states, "flops": 7 * cells * sum(lens)}
