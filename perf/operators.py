"""Checkpoints of activations in 8 bits and projections with low-rank adapters, as cases that can be timed and compared.

`checkpoint`: a matrix of activations goes into 8 bits (stochastic rounding onto a grid for each group of a row) and comes
back.  `project`: tokens of several requests, each with its own low-rank adapter, pass a shared projection whose weights
are packed codes.  `backward`: that projection's backward pass, adapter gradients from the checkpoints.

A case is a dict: `kind` is the operator, `tokens` the rows, `inputs` and `outputs` the projection's sizes, `bits` of its
codes, `rank` and `adapters` the low-rank part, `requests` how many share the tokens, `spare` rows behind the last
request, which every call leaves as they were.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}


def _checkpoint(name, tokens, inputs, dtype, group):
    return {"name": name, "kind": "checkpoint", "tokens": tokens, "inputs": inputs, "dtype": dtype, "group": group}


def _projection(name, kind, tokens, inputs, outputs, bits, dtype, rank, adapters, requests, spare=0, group=128):
    return {"name": name, "kind": kind, "tokens": tokens, "inputs": inputs, "outputs": outputs, "bits": bits, "dtype": dtype,
            "rank": rank, "adapters": adapters, "requests": requests, "spare": spare, "group": group}


def listed():
    return [
        # A minibatch of the ordinary dense problem (1000 features, rows that end inside a group) between two layers.
        _checkpoint("checkpoint_small", 256, 1000, "fp32", 64),
        # One layer's input of a sequence of odd length.
        _checkpoint("checkpoint_odd", 2047, 4096, "fp16", 128),
        # A large batch's input to a wide layer: what checkpoints are for.
        _checkpoint("checkpoint_large", 16384, 8192, "bf16", 128),
        # One token of one request: a serving step where latency counts.
        _projection("project_token", "project", 1, 4096, 4096, 8, "bf16", 16, 8, 1),
        # A decoding step of 64 requests, one token each, over a widening projection at 4 bits.
        _projection("project_decode", "project", 64, 4096, 14336, 4, "fp16", 16, 32, 64),
        # Ragged prompts on odd sizes, rows behind the last one.
        _projection("project_ragged", "project", 777, 1000, 2049, 6, "bf16", 8, 5, 7, spare=23),
        # Long prompts of 16 requests over a large square projection.
        _projection("project_prompts", "project", 8192, 8192, 8192, 4, "bf16", 32, 16, 16),
        # The forward pass of fine-tuning: few requests, one adapter each, 8-bit codes.
        _projection("project_training", "project", 4096, 4096, 16384, 8, "bf16", 16, 2, 4),
        # The backward pass of a short batch on the ordinary problem's 1000 features.
        _projection("backward_small", "backward", 33, 1000, 1000, 8, "bf16", 8, 2, 3, group=64),
        # The backward pass of an ordinary fine-tuning step in fp16.
        _projection("backward_medium", "backward", 2048, 4096, 4096, 4, "fp16", 64, 4, 8),
        # The backward pass of a large one.
        _projection("backward_large", "backward", 8192, 8192, 8192, 8, "bf16", 16, 4, 8),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["checkpoint", "project", "project", "project", "backward", "backward"])
    dtype, group = rng.choice(["bf16", "bf16", "fp16"]), rng.choice([32, 64, 128, 128, 256])
    inputs, outputs = _log_int(rng, 64, 8192), _log_int(rng, 64, 16384)
    if rng.random() < 0.6:                                        # most sizes round, as layers' are
        inputs, outputs = max(64, inputs // 64 * 64), max(64, outputs // 64 * 64)
    if kind == "checkpoint":
        return {"kind": kind, "tokens": _log_int(rng, 16, 16384), "inputs": inputs, "dtype": rng.choice(["fp32", dtype]), "group": group}
    tokens = _log_int(rng, 1, 4096) if kind == "project" else _log_int(rng, 16, 4096)
    requests = min(tokens, _log_int(rng, 1, 64))
    case = _projection("", kind, tokens, inputs, outputs, rng.choice([2, 3, 4, 4, 4, 5, 6, 8, 8, 8]), dtype, rng.choice([4, 8, 12, 16, 16, 32, 64]),
                       _log_int(rng, 1, 32), requests, spare=rng.choice([0, 0, 5, 64]), group=group)
    del case["name"]
    return case


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _activations(rows, columns, dtype, g):
    """Normal values, some features much larger than the others: what a layer's input looks like."""
    width = torch.exp(0.5 * torch.randn(columns, generator=g, device="cuda"))
    return (torch.randn((rows, columns), generator=g, device="cuda") * width).to(dtype)


def _container(bits):
    return 2 if bits <= 2 else 4 if bits <= 4 else 8


def _weights(case, g):
    """A projection's codes, packed low bits first into rows of a multiple of 16 bytes, and the grid of each output."""
    k, n, bits, cb = case["inputs"], case["outputs"], case["bits"], _container(case["bits"])
    top = (1 << bits) - 1
    codes = (torch.randn((k, n), generator=g, device="cuda") * (top / 7) + top / 2).round().clamp(0, top).to(torch.uint8)
    span = (7 / math.sqrt(k)) * torch.exp(0.2 * torch.randn(n, generator=g, device="cuda"))
    step = span / top
    lo = -0.5 * span + 0.1 * step * torch.randn(n, generator=g, device="cuda")
    per = 8 // cb
    row_bytes = (-(-n // per) + 15) // 16 * 16
    padded = torch.zeros((k, row_bytes * per), dtype=torch.uint8, device="cuda")
    padded[:, :n] = codes
    shifts = torch.arange(per, device="cuda", dtype=torch.uint8) * cb
    plane = (padded.view(k, row_bytes, per) << shifts).sum(2, dtype=torch.uint8)
    return plane, lo, step


def _grid_of(x, group):
    """(rows, groups) minimum and maximum of each group of a row's features."""
    rows, n = x.shape
    groups = -(-n // group)
    at = torch.arange(groups * group, device=x.device).clamp(max=n - 1)           # the last group repeats the row's last feature
    v = x[:, at].view(rows, groups, group)
    return v.amin(2), v.amax(2)


_contexts = []


def _context(binding):
    """The program's one context."""
    if not _contexts:
        _contexts.append(binding.Context("cuda:%d" % torch.cuda.current_device()))
    return _contexts[0]


def prepare(case, seed):
    g, dtype, rows = _generator(seed), DTYPES[case["dtype"]], case["tokens"] + case.get("spare", 0)
    state = {"case": case, "seed": int(seed)}
    if case["kind"] == "checkpoint":
        state["x"] = _activations(rows, case["inputs"], dtype, g)
    else:
        k, n, r, count = case["inputs"], case["outputs"], case["rank"], case["adapters"]
        state["plane"], state["lo"], state["step"] = _weights(case, g)
        state["a"] = (torch.randn((count, r, k), generator=g, device="cuda") / math.sqrt(k)).to(dtype)
        state["b"] = (torch.randn((count, r, n), generator=g, device="cuda") / math.sqrt(r)).to(dtype)
        state["scale"] = 0.25 + torch.rand(count, generator=g, device="cuda")
        draws = np.random.RandomState(int(seed) % (1 << 32))
        cuts = np.sort(draws.choice(np.arange(1, case["tokens"]), case["requests"] - 1, replace=False)) if case["requests"] > 1 else []
        state["starts"] = torch.tensor([0, *cuts, case["tokens"]], dtype=torch.int32, device="cuda")
        which = draws.randint(0, count, case["requests"])
        which[draws.rand(case["requests"]) < 0.1] = -1                            # a request without an adapter now and then
        state["which"] = torch.tensor(which, dtype=torch.int32, device="cuda")
        x = _activations(rows, k, dtype, g)
        if case["kind"] == "project":
            state["x"] = x
            state["y"] = torch.zeros((rows, n), dtype=dtype, device="cuda")
            state["hidden"] = torch.zeros((rows, r), device="cuda")
        else:
            low, high = _grid_of(x.float(), case["group"])
            step = (high - low) / 255
            spread = lambda v: v.repeat_interleave(case["group"], 1)[:, :k]  # noqa: E731
            state["codes"] = torch.zeros((rows, (k + 15) // 16 * 16), dtype=torch.uint8, device="cuda")
            state["codes"][:, :k] = ((x.float() - spread(low)) / spread(step)).round().clamp(0, 255).to(torch.uint8)
            state["grid"] = torch.stack([low, step], 2).contiguous()
            state["dy"] = (0.01 * torch.randn((rows, n), generator=g, device="cuda")).to(dtype)
            state["hidden"] = torch.randn((rows, r), generator=g, device="cuda")
            state["dx"] = torch.zeros((rows, k), dtype=dtype, device="cuda")
    if own:
        from paper_1611_05402_b200 import binding
        state["ctx"] = _context(binding)
        if case["kind"] != "checkpoint":
            state["weights"] = binding.Dataset(state["plane"], state["plane"], case["inputs"], case["outputs"], case["bits"],
                                               binding.LEVELS_UNIFORM, state["lo"], state["step"], None)
            state["adapters"] = binding.Adapters(state["a"], state["b"], state["scale"])
        if case["kind"] == "backward":
            state["checkpoint"] = binding.Checkpoint(state["codes"], state["grid"], rows, case["inputs"], case["group"])
    return state


def _draws(seed, rows, n):
    """16 random bits for each element: Philox4x32-10 of (block of 8 features, row), eight halves of its four words."""
    blocks, mask = -(-n // 8), 0xFFFFFFFF
    c0 = torch.arange(blocks, device="cuda", dtype=torch.int64).expand(rows, blocks)
    c1 = torch.arange(rows, device="cuda", dtype=torch.int64)[:, None].expand(rows, blocks)
    c2, c3 = torch.zeros_like(c0), torch.full_like(c0, 8)
    k0, k1 = seed & mask, (seed >> 32) & mask

    def rounds(left, c0, c1, c2, c3, k0, k1):
        if not left:
            return c0, c1, c2, c3
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57                                 # 64-bit products, their wrapped sign bit masked off
        return rounds(left - 1, ((p1 >> 32) & mask) ^ c1 ^ k0, p1 & mask, ((p0 >> 32) & mask) ^ c3 ^ k1, p0 & mask,
                      (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask)

    words = torch.stack(rounds(10, c0, c1, c2, c3, k0, k1), 2)
    halves = torch.stack([words & 0xFFFF, words >> 16], 3)
    return halves.reshape(rows, blocks * 8)[:, :n]


def _round_trip(x, group, seed, dtype):
    """The checkpoint's values: t = (x - lo) * (255 / (hi - lo)) in 32 bits, up where t's fraction, in 2^-16 rounded up, and the draw reach one."""
    rows, n = x.shape
    v = x.float()
    lo, hi = _grid_of(v, group)
    span, top = hi - lo, torch.full_like(lo, 255)                                 # (a tensor: by a number torch multiplies by its rounded inverse)
    inv, step = torch.where(span > 0, top / span, 0).clamp(max=torch.finfo(torch.float32).max), span / top
    spread = lambda q: q.repeat_interleave(group, 1)[:, :n]  # noqa: E731
    t = ((v - spread(lo)) * spread(inv)).clamp(0, 255)
    code = ((t * 65536).ceil().to(torch.int64) + _draws(seed, rows, n)) >> 16
    return (spread(lo) + code.float() * spread(step)).to(dtype)


def _codes(state):
    """The projection's codes as whole numbers, (inputs, outputs)."""
    cb = _container(state["case"]["bits"])
    shifts = torch.arange(8 // cb, device="cuda", dtype=torch.uint8) * cb
    codes = (state["plane"][:, :, None] >> shifts) & ((1 << cb) - 1)
    return codes.view(state["plane"].shape[0], -1)[:, :state["case"]["outputs"]]


def _shares(state, rows):
    """(rows, adapters): the adapter's scale where a row belongs to it, else 0; and whether the row belongs to a request."""
    t = torch.arange(rows, device="cuda")
    request = torch.searchsorted(state["starts"].long(), t, right=True) - 1
    used = request < len(state["which"])
    adapter = torch.where(used, state["which"].long()[request.clamp(max=len(state["which"]) - 1)], -1)
    one = adapter[:, None] == torch.arange(len(state["scale"]), device="cuda")
    return one, used


def _plain_project(state):
    x, a, b = state["x"].float(), state["a"].float(), state["b"].float()
    count, r, k = a.shape
    one, used = _shares(state, len(x))
    w = state["lo"] + _codes(state).float() * state["step"]
    parts = (x @ a.view(count * r, k).T).view(-1, count, r) * (one * state["scale"])[:, :, None]
    y = (x @ w + parts.reshape(-1, count * r) @ b.view(count * r, -1)).to(state["y"].dtype)
    return {"y": torch.where(used[:, None], y, state["y"]), "hidden": torch.where(used[:, None], parts.sum(1), state["hidden"])}


def _plain_backward(state):
    dy, a, b, k = state["dy"].float(), state["a"].float(), state["b"].float(), state["case"]["inputs"]
    count, r, n = b.shape
    one, used = _shares(state, len(dy))
    dy = torch.where(used[:, None], dy, 0)
    w = state["lo"] + _codes(state).float() * state["step"]
    v = (dy @ b.view(count * r, n).T).view(-1, count, r) * (one * state["scale"])[:, :, None]
    v = v.reshape(-1, count * r)
    dx = (dy @ w.T + v @ a.view(count * r, k)).to(state["dx"].dtype)
    spread = lambda q: q.repeat_interleave(state["case"]["group"], 1)[:, :k]  # noqa: E731
    x = spread(state["grid"][:, :, 0]) + state["codes"][:, :k].float() * spread(state["grid"][:, :, 1])
    h = (state["hidden"][:, None, :] * one[:, :, None]).reshape(-1, count * r)
    return {"dx": torch.where(used[:, None], dx, state["dx"]), "da": (v.T @ x).view(count, r, k), "db": (h.T @ dy).view(count, r, n)}


def run(state):
    case = state["case"]
    if own:
        ctx = state["ctx"]
        if case["kind"] == "checkpoint":
            kept = ctx.zipml_checkpoint_encode(state["x"], group=case["group"], seed=state["seed"])
            return {"x": ctx.zipml_checkpoint_decode(kept, dtype=state["x"].dtype)}
        if case["kind"] == "project":
            ctx.zipml_project(state["weights"], state["x"], adapters=state["adapters"], starts=state["starts"], which=state["which"],
                              out=state["y"], hidden=state["hidden"])
            return {"y": state["y"], "hidden": state["hidden"]}
        dx, da, db = ctx.zipml_project_backward(state["weights"], state["dy"], adapters=state["adapters"], starts=state["starts"],
                                                which=state["which"], hidden=state["hidden"], checkpoint=state["checkpoint"],
                                                out=state["dx"])
        return {"dx": dx, "da": da, "db": db}
    if case["kind"] == "checkpoint":
        return {"x": _round_trip(state["x"], case["group"], state["seed"], state["x"].dtype)}
    return _plain_project(state) if case["kind"] == "project" else _plain_backward(state)


def work(case):
    t, k, e = case["tokens"], case["inputs"], SIZE[case["dtype"]]
    if case["kind"] == "checkpoint":
        return {"bytes": 2 * t * k * (e + 1) + 16 * t * -(-k // case["group"]), "flops": 0}
    n, r, used = case["outputs"], case["rank"], min(case["adapters"], case["requests"])
    weights = k * n * _container(case["bits"]) / 8 + 8 * n
    moved = weights + e * t * (k + n) + e * used * r * (k + n) + 4 * t * r
    if case["kind"] == "project":
        return {"bytes": moved, "flops": 2 * t * k * n + 2 * t * r * (k + n)}
    checkpoint = t * k + 8 * t * -(-k // case["group"])
    return {"bytes": moved + checkpoint + 4 * case["adapters"] * r * (k + n), "flops": 2 * t * k * n + 4 * t * r * (k + n)}


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "checkpoint":
        x, group = state["x"].double(), case["group"]
        rows, n = x.shape
        out = torch.empty_like(x)
        draws = _draws(int(seed), rows, n).double()
        for j in range(0, n, group):
            part = x[:, j:j + group]
            lo, hi = part.min(1, keepdim=True).values, part.max(1, keepdim=True).values
            # which code a value gets is defined by roundings to 32 bits, as the framework's quantizers define it; what the code stands for is not
            span = (hi - lo).float().double()
            inv = torch.where(span > 0, (255 / span).float().double(), 0.0)
            t = ((part - lo).float().double() * inv).float().double()
            code = torch.floor((torch.ceil(t * 65536) + draws[:, j:j + group]) / 65536)
            out[:, j:j + group] = lo + code * ((hi - lo) / 255)
        return {"x": out}
    starts, which = state["starts"].tolist(), state["which"].tolist()
    k, n, cb = case["inputs"], case["outputs"], _container(case["bits"])
    w = torch.empty((k, n), dtype=torch.float64, device="cuda")
    for i in range(8 // cb):                                      # the outputs that lie in the i-th field of their bytes
        at = w[:, i::8 // cb]
        at.copy_((state["plane"][:, :at.shape[1]] >> (i * cb)) & ((1 << cb) - 1))
    w = w * state["step"].double() + state["lo"].double()
    a, b, scale = state["a"].double(), state["b"].double(), state["scale"].double()
    if case["kind"] == "project":
        x, y, hidden = state["x"].double(), state["y"].double(), state["hidden"].double()
        for q, i in enumerate(which):
            rows = slice(starts[q], starts[q + 1])
            y[rows], hidden[rows] = x[rows] @ w, 0
            if i >= 0:
                hidden[rows] = scale[i] * (x[rows] @ a[i].T)
                y[rows] += hidden[rows] @ b[i]
        return {"y": y, "hidden": hidden}
    dy, dx, hidden = state["dy"].double(), state["dx"].double(), state["hidden"].double()
    x = state["codes"][:, :k].double()
    for j in range(0, k, case["group"]):
        x[:, j:j + case["group"]] *= state["grid"][:, j // case["group"], 1:].double()
        x[:, j:j + case["group"]] += state["grid"][:, j // case["group"], :1].double()
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    for q, i in enumerate(which):
        rows = slice(starts[q], starts[q + 1])
        dx[rows] = dy[rows] @ w.T
        if i >= 0:
            v = scale[i] * (dy[rows] @ b[i].T)
            dx[rows] += v @ a[i]
            da[i] += v.T @ x[rows]
            db[i] += hidden[rows].T @ dy[rows]
    return {"dx": dx, "da": da, "db": db}
