"""Low-rank adapters beside a residual-binary layer, their backward pass and the clipping of their gradients, as cases that can be
timed and compared.

A case is a dict of plain values.  ``listed()`` gives the fixed ones, ``draw(rng)`` one more of the same ranges, ``prepare(case, seed)``
what a program holds before the call, ``run(state)`` one pass, ``work(case)`` the bytes and operations that pass cannot do without,
``exact(case, seed)`` its result in 64 bits.  With ``own`` false ``run`` computes the operators in elementary torch operations in
32 bits, with ``own`` true it makes the library's calls.

Kinds of pass:

* ``linear``    one layer whose rows bring adapters of a shared pool: ``y = W x + scale b^T (a x)`` per row;
* ``group``     projections that share their input (q|k|v, gate|up), each with its own adapters;
* ``backward``  the gradients of one adapted layer: of the input (through the frozen layer and the adapters) and of both factors;
* ``train``     forward and backward of one adapted group and the clipping of all its factor gradients;
* ``clip``      the norm over the factor gradients of a whole model and their clipping.

Sign words are uniform, h ~ U(0.5, 1.5), g_1 ~ U(0.01, 0.03), g_k = g_{k-1} U(0.2, 0.5), activations N(0, 1), output gradients
N(0, 0.1^2); the first factors N(0, 1/N), the second N(0, 0.02^2), scale 2 as of alpha = 2 r, varied a little from adapter to adapter.
"""
import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"


def listed():
    return [
        # one request, one token: the 8B-shaped k or v projection, where latency counts
        {"name": "linear_kv_1024x4096_b1", "kind": "linear", "K": 2, "M": "1024", "N": 4096, "rows": 1, "rank": 16, "pool": 8, "used": 1, "bare": 0, "prompts": 0},
        # sixteen sequences decoded together, each with an adapter of its own but two that have none: 8B-shaped q|k|v
        {"name": "group_qkv_8b_b16", "kind": "group", "K": 2, "M": "4096,1024,1024", "N": 4096, "rows": 16, "rank": 16, "pool": 32, "used": 14, "bare": 2, "prompts": 0},
        # a server's decode batch, ten adapters shared by 48 rows: 8B-shaped gate projection
        {"name": "linear_14336x4096_b48", "kind": "linear", "K": 2, "M": "14336", "N": 4096, "rows": 48, "rank": 32, "pool": 16, "used": 10, "bare": 5, "prompts": 0},
        # seven prompts of different lengths beside single tokens: 8B-shaped down projection, rank 64
        {"name": "linear_4096x14336_mixed", "kind": "linear", "K": 2, "M": "4096", "N": 14336, "rows": 1037, "rank": 64, "pool": 8, "used": 6, "bare": 23, "prompts": 7},
        # three paths, 13B-sized input, a row count that is no multiple of anything, an odd rank
        {"name": "linear_5001x13824_k3_b200", "kind": "linear", "K": 3, "M": "5001", "N": 13824, "rows": 200, "rank": 12, "pool": 4, "used": 3, "bare": 9, "prompts": 5},
        # a long prompt: 7B-shaped gate projection
        {"name": "linear_11008x4096_b4096", "kind": "linear", "K": 2, "M": "11008", "N": 4096, "rows": 4096, "rank": 16, "pool": 4, "used": 1, "bare": 0, "prompts": 1},
        # a small fine-tuning step: three jobs' rows in one batch
        {"name": "backward_1024x4096_t77", "kind": "backward", "K": 2, "M": "1024", "N": 4096, "rows": 77, "rank": 8, "pool": 3, "used": 3, "bare": 4, "prompts": 3},
        # one job, 2048 tokens: 7B-shaped o projection
        {"name": "backward_4096x4096_t2048", "kind": "backward", "K": 2, "M": "4096", "N": 4096, "rows": 2048, "rank": 16, "pool": 1, "used": 1, "bare": 0, "prompts": 1},
        # two jobs of rank 64 with padding rows between them: 7B-shaped down projection
        {"name": "backward_4096x11008_t4096", "kind": "backward", "K": 2, "M": "4096", "N": 11008, "rows": 4096, "rank": 64, "pool": 2, "used": 2, "bare": 100, "prompts": 9},
        # everything after one another: 8B-shaped q|k|v, forward, backward, clipping
        {"name": "train_qkv_8b_t512", "kind": "train", "K": 2, "M": "4096,1024,1024", "N": 4096, "rows": 512, "rank": 16, "pool": 1, "used": 1, "bare": 0, "prompts": 1},
        # factor gradients of one 8B-shaped decoder layer, rank 8
        {"name": "clip_8b_1_layer_r8", "kind": "clip", "layers": 1, "d": 4096, "kv": 1024, "ffn": 14336, "rank": 8},
        # factor gradients of a 7B-shaped model of 32 layers, rank 16: 448 tensors
        {"name": "clip_7b_32_layers_r16", "kind": "clip", "layers": 32, "d": 4096, "kv": 4096, "ffn": 11008, "rank": 16},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    costs = [(c["kind"], work(c)) for c in listed()]
    while True:
        kind = rng.choice(("linear",) * 8 + ("group", "group", "backward", "backward", "backward", "train", "clip", "clip"))
        if kind == "clip":
            d = 128 * _log_int(rng, 4, 64)
            case = {"kind": kind, "layers": rng.randint(1, 40), "d": d, "kv": d // rng.choice((1, 4, 8)), "ffn": 32 * int(d * rng.uniform(2.5, 3.6) / 32), "rank": _log_int(rng, 1, 64)}
        else:
            N, used = 32 * _log_int(rng, 16, 512), rng.choice((1, 1, 2, 3, 5, 9, 14))
            if kind == "linear":
                M = [_log_int(rng, 256, 16384)]
                rows = _log_int(rng, *rng.choice(((1, 1), (1, 8), (3, 16), (9, 64), (17, 256), (129, 1024), (513, 4096))))
            elif kind == "group":
                M = [_log_int(rng, 256, 4096) for _ in range(rng.randint(2, 3))]
                rows = _log_int(rng, 1, 16)
            else:
                M = [32 * _log_int(rng, 8, 512) for _ in range(1 if kind == "backward" else rng.randint(2, 3))]
                rows = _log_int(rng, 16, 4096 if kind == "backward" else 512)
                used = min(used, 5)
            used = min(used, rows)
            bare = rng.randint(0, min(rows - used, 1 + rows // 8))
            prompts = 0 if rows < 17 else rng.randint(used, used + 6)
            case = {"kind": kind, "K": rng.choice((1, 2, 2, 2, 3)), "M": ",".join(map(str, M)), "N": N, "rows": rows, "rank": rng.choice((4, 8, 8, 16, 16, 32, 64, rng.randint(1, 128))),
                    "pool": used + rng.choice((0, 0, 2, 8)), "used": used, "bare": bare, "prompts": min(prompts, rows - bare)}
        w = work(case)
        if w["bytes"] <= max(c["bytes"] for k, c in costs if k == kind) and w["flops"] <= max(c["flops"] for k, c in costs if k == kind):
            return case


# ---- making the inputs -----------------------------------------------------------------------------------

def _shapes(case):
    return [(int(m), case["N"]) for m in case["M"].split(",")]


def _clip_sizes(case):
    """Elements of the two factor gradients of every adapted projection: q, k, v, o, gate, up, down of each layer."""
    d, kv, f, r = case["d"], case["kv"], case["ffn"], case["rank"]
    return [r * n for _ in range(case["layers"]) for M, N in ((d, d), (kv, d), (kv, d), (d, d), (f, d), (f, d), (d, f)) for n in (N, M)]


def _ids(case, rng):
    """Which adapter each row brings (-1: none): single tokens in any order, or prompts one behind the other with bare rows between."""
    rows, used, bare, prompts = case["rows"], case["used"], case["bare"], case["prompts"]
    slots = rng.permutation(case["pool"])[:used]
    ids = np.full(rows, -1, dtype=np.int32)
    if prompts == 0:
        at = rng.permutation(rows)[: rows - bare]
        ids[at] = slots[np.arange(rows - bare) % used]
    else:
        keep = np.sort(rng.permutation(rows)[: rows - bare])
        cuts = np.sort(rng.permutation(rows - bare - 1)[: prompts - 1]) + 1 if prompts > 1 else np.empty(0, dtype=np.int64)
        ids[keep] = slots[np.searchsorted(cuts, np.arange(rows - bare), side="right") % used]
    return ids


def _half(gen, shape, std):
    return torch.randn(shape, generator=gen, dtype=torch.float32, device=DEVICE).mul_(std).to(torch.float16)


def _projection(case, gen, rng, M, N):
    K, n, r = case["K"], case["pool"], case["rank"]
    h = rng.uniform(0.5, 1.5, (K, N)).astype(np.float16)
    g = np.empty((K, M), dtype=np.float16)
    g[0] = rng.uniform(0.01, 0.03, M)
    for k in range(1, K):
        g[k] = g[k - 1].astype(np.float64) * rng.uniform(0.2, 0.5, M)
    planes = torch.randint(-(1 << 31), 1 << 31, (K, M, N // 32), generator=gen, dtype=torch.int64, device=DEVICE).to(torch.int32)
    return {"planes": planes, "g": torch.from_numpy(g).to(DEVICE), "h": torch.from_numpy(h).to(DEVICE),
            "a": _half(gen, (n, r, N), N ** -0.5), "b": _half(gen, (n, r, M), 0.02),
            "scale": torch.from_numpy(rng.uniform(1.5, 2.5, n).astype(np.float32)).to(DEVICE)}


def _library(case, state):
    """The handles that a program keeps: packed layers, adapters, buffers of the backward pass."""
    import paper_2602_05367_b200 as rabit
    state["rabit"] = rabit
    if case["kind"] == "clip":
        state["gradients"] = rabit.RabitGradients(state["grads"], state["outs"])
        return
    for P in state["projections"]:
        P["layer"] = rabit.rabit_pack(P["planes"].cpu().numpy().view(np.uint32), P["g"].cpu().numpy(), P["h"].cpu().numpy(), device=DEVICE)
        P["adapters"] = rabit.RabitAdapters(P["a"], P["b"], P["scale"])
        if case["kind"] in ("backward", "train"):
            P["layer_t"] = rabit.rabit_transpose(P["layer"])
            P["adapters_t"] = P["adapters"].transposed()
            P["p"] = torch.empty((case["rows"], case["rank"]), dtype=torch.float32, device=DEVICE)
            P["da"] = torch.empty(P["a"].shape, dtype=torch.float32, device=DEVICE)
            P["db"] = torch.empty(P["b"].shape, dtype=torch.float32, device=DEVICE)
    if case["kind"] == "train":
        state["gradients"] = rabit.RabitGradients([t for P in state["projections"] for t in (P["da"], P["db"])])


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    rng = np.random.default_rng(seed)
    state = {"kind": case["kind"]}
    if case["kind"] == "clip":
        state["grads"] = [torch.randn(n, generator=gen, dtype=torch.float32, device=DEVICE).mul_(1e-3) for n in _clip_sizes(case)]
        state["flat"] = torch.empty(sum(_clip_sizes(case)), dtype=torch.float32, device=DEVICE)   # the optimiser's buffer, tensor behind tensor
        state["outs"] = list(state["flat"].split(_clip_sizes(case)))
        state["max_norm"] = 0.3 * 1e-3 * math.sqrt(sum(_clip_sizes(case)))
    else:
        state["x"] = _half(gen, (case["rows"], case["N"]), 1.0)
        state["ids"] = torch.from_numpy(_ids(case, rng)).to(DEVICE)
        state["projections"] = [_projection(case, gen, rng, M, N) for M, N in _shapes(case)]
        for P in state["projections"]:
            if case["kind"] in ("group", "train"):
                P["y"] = torch.empty((case["rows"], P["g"].shape[1]), dtype=torch.float16, device=DEVICE)
            if case["kind"] in ("backward", "train"):
                P["dy"] = _half(gen, (case["rows"], P["g"].shape[1]), 0.1)
                P["u"] = torch.empty((case["rows"], case["rank"]), dtype=torch.float32, device=DEVICE)
            if case["kind"] == "backward":                    # what the forward pass has left
                picked = torch.nn.functional.one_hot(state["ids"].long() + 1, case["pool"] + 1)[:, 1:, None]
                P["u"] = ((state["x"].double() @ P["a"].double().flatten(0, 1).T).unflatten(1, P["a"].shape[:2]) * picked).sum(1).float()
        if case["kind"] == "train":
            state["max_norm"] = 0.05
    if own:
        _library(case, state)
    return state


# ---- the plain form, in 32 bits --------------------------------------------------------------------------

def _signs(planes):
    """+-1 in fp32 [K][M][N] of the packed words [K][M][N/32], column j in bit j % 32 of word j // 32."""
    bits = (planes.unsqueeze(-1) >> torch.arange(32, device=planes.device, dtype=torch.int32)) & 1
    return (1 - 2 * bits).to(torch.float32).flatten(2)


def _spread(v, ids):
    """[T][n][r] -> the same with every row's entries outside its own adapter zero."""
    hit = ids[:, None] == torch.arange(v.shape[1], device=ids.device, dtype=ids.dtype)
    return torch.where(hit[:, :, None], v, torch.zeros((), dtype=v.dtype, device=v.device))


def _narrow(v, factor, ids):
    """v [T][side] in fp32 through the first of two factors [n][r][side]: [T][n][r], zero outside the row's own adapter."""
    return _spread((v @ factor.float().flatten(0, 1).T).unflatten(1, factor.shape[:2]), ids)


def _widen(low, scale, factor):
    return (low * scale[:, None]).flatten(1) @ factor.float().flatten(0, 1)


def _plain_forward(P, x, ids):
    x, B = x.float(), _signs(P["planes"])
    base = ((x * P["h"].float()[:, None, :]) @ B.transpose(1, 2) * P["g"].float()[:, None, :]).sum(0)
    u = _narrow(x, P["a"], ids)
    return (base + _widen(u, P["scale"], P["b"])).half(), u


def _plain_backward(P, x, u, ids):
    x, dy, B = x.float(), P["dy"].float(), _signs(P["planes"])
    base = ((dy * P["g"].float()[:, None, :]) @ B * P["h"].float()[:, None, :]).sum(0)
    p = _narrow(dy, P["b"], ids)
    dx = (base + _widen(p, P["scale"], P["a"])).half()
    da = ((p * P["scale"][:, None]).flatten(1).T @ x).unflatten(0, P["a"].shape[:2])
    db = ((u * P["scale"][:, None]).flatten(1).T @ dy).unflatten(0, P["b"].shape[:2])
    return dx, da, db


def _plain_clip(grads, outs, max_norm):
    norm = torch.stack([t.double().square().sum() for t in grads]).sum().sqrt()
    factor = torch.clamp(max_norm / (norm + 1e-6), max=1.0).float()
    return [torch.mul(t, factor, out=out) for t, out in zip(grads, outs)], norm.float().reshape(1)


def _plain(state):
    kind, ids = state["kind"], state.get("ids")
    if kind == "clip":
        return {"clipped": state["flat"], "norm": _plain_clip(state["grads"], state["outs"], state["max_norm"])[1]}
    if kind == "linear":
        return _plain_forward(state["projections"][0], state["x"], ids)[0]
    if kind == "group":
        return [_plain_forward(P, state["x"], ids)[0] for P in state["projections"]]
    if kind == "backward":
        P = state["projections"][0]
        return _plain_backward(P, state["x"], _spread(P["u"][:, None, :].expand(-1, P["a"].shape[0], -1), ids), ids)
    forward = [_plain_forward(P, state["x"], ids) for P in state["projections"]]
    backward = [_plain_backward(P, state["x"], u, ids) for P, (_, u) in zip(state["projections"], forward)]
    grads = [t for _, da, db in backward for t in (da, db)]
    clipped, norm = _plain_clip(grads, grads, state["max_norm"])
    return {"y": [y for y, _ in forward], "dx": [dx for dx, _, _ in backward], "clipped": clipped, "norm": norm}


# ---- the library's calls ---------------------------------------------------------------------------------

def _own_backward(rabit, P, x, ids):
    dx = rabit.rabit_linear_adapted(P["layer_t"], P["adapters_t"], P["dy"], ids, u=P["p"])
    rabit.rabit_adapter_gradients(P["adapters"], x, P["u"], P["dy"], P["p"], ids, P["da"], P["db"])
    return dx, P["da"], P["db"]


def _own(state):
    rabit, kind = state["rabit"], state["kind"]
    if kind == "clip":
        norm = rabit.rabit_clip_gradients(state["gradients"], state["max_norm"])
        return {"clipped": state["flat"], "norm": norm}
    ps, x, ids = state["projections"], state["x"], state["ids"]
    if kind == "linear":
        return rabit.rabit_linear_adapted(ps[0]["layer"], ps[0]["adapters"], x, ids)
    if kind == "group":
        return rabit.rabit_linear_group_adapted([P["layer"] for P in ps], [P["adapters"] for P in ps], [x] * len(ps), ids, [P["y"] for P in ps])
    if kind == "backward":
        return _own_backward(rabit, ps[0], x, ids)
    ys = rabit.rabit_linear_group_adapted([P["layer"] for P in ps], [P["adapters"] for P in ps], [x] * len(ps), ids, [P["y"] for P in ps], [P["u"] for P in ps])
    dxs = [_own_backward(rabit, P, x, ids)[0] for P in ps]
    norm = rabit.rabit_clip_gradients(state["gradients"], state["max_norm"])
    return {"y": ys, "dx": dxs, "clipped": [t for P in ps for t in (P["da"], P["db"])], "norm": norm}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -----------------------------------------------------------------------

def work(case):
    if case["kind"] == "clip":
        return {"bytes": 8.0 * sum(_clip_sizes(case)), "flops": 3.0 * sum(_clip_sizes(case))}
    K, T, r, n, used, busy = case["K"], case["rows"], case["rank"], case["pool"], case["used"], case["rows"] - case["bare"]
    total = {"bytes": 4.0 * T, "flops": 0.0}
    if case["kind"] != "backward":
        total["bytes"] += 2.0 * T * case["N"]                  # the input that all projections share
    for M, N in _shapes(case):
        layer = {"bytes": K * M * N / 8 + 2.0 * K * (M + N) + 2.0 * used * r * (M + N), "flops": 2.0 * K * M * N * T + 2.0 * busy * r * (M + N)}
        if case["kind"] in ("linear", "group", "train"):
            total["bytes"] += layer["bytes"] + 2.0 * T * M
            total["flops"] += layer["flops"]
        if case["kind"] in ("backward", "train"):              # dy in, dx out, x and u once more, both gradients out
            total["bytes"] += layer["bytes"] + 2.0 * T * (M + N) + (2.0 * T * N if case["kind"] == "backward" else 0.0) + 4.0 * T * r + 4.0 * n * r * (M + N)
            total["flops"] += layer["flops"] + 2.0 * busy * r * (M + N)
    return total


# ---- the definition in 64 bits ---------------------------------------------------------------------------

def _weight64(P):
    """Eq. 2 as a dense matrix: sum over the paths of g_i h_j, with the sign that bit j % 32 of word j // 32 says."""
    K, M, words = P["planes"].shape
    W = torch.zeros((M, 32 * words), dtype=torch.float64, device=DEVICE)
    weight = torch.tensor([1 << j for j in range(32)], dtype=torch.int64, device=DEVICE)
    for k in range(K):
        minus = ((P["planes"][k].to(torch.int64) & 0xFFFFFFFF)[:, :, None].bitwise_and(weight) != 0).reshape(M, 32 * words)
        magnitude = torch.outer(P["g"][k].double(), P["h"][k].double())
        W += torch.where(minus, -magnitude, magnitude)
    return W


def _adapted64(W, first, second, scale, x, ids):
    """x W^T plus the rows' adapters, adapter by adapter; the low-rank products beside it."""
    y, low = x @ W.T, torch.zeros((x.shape[0], first.shape[1]), dtype=torch.float64, device=DEVICE)
    for i in ids.unique().tolist():
        if i >= 0:
            rows = (ids == i).nonzero()[:, 0]
            low[rows] = x[rows] @ first[i].double().T
            y[rows] += scale[i].double() * (low[rows] @ second[i].double())
    return y, low


def _factors64(first, scale, low, v, ids):
    """Gradient of a factor [n][r][side]: scale times the sum over an adapter's rows of low^T v."""
    out = torch.zeros(first.shape, dtype=torch.float64, device=DEVICE)
    for i in ids.unique().tolist():
        if i >= 0:
            rows = (ids == i).nonzero()[:, 0]
            out[i] = scale[i].double() * (low[rows].T @ v[rows])
    return out


def _clip64(grads, max_norm):
    norm = math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in grads))
    return [t.double() * min(1.0, max_norm / (norm + 1e-6)) for t in grads], torch.tensor([norm], dtype=torch.float64)


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "clip":
        outs, norm = _clip64(state["grads"], state["max_norm"])
        return {"clipped": torch.cat(outs), "norm": norm}
    x, ids, ys, dxs, grads = state["x"].double(), state["ids"], [], [], []
    for P in state["projections"]:
        W = _weight64(P)
        y, u = _adapted64(W, P["a"], P["b"], P["scale"], x, ids)
        ys.append(y)
        if "dy" in P:
            dy = P["dy"].double()
            dx, p = _adapted64(W.T, P["b"], P["a"], P["scale"], dy, ids)
            dxs.append(dx)
            grads += [_factors64(P["a"], P["scale"], p, x, ids), _factors64(P["b"], P["scale"], P["u"].double() if case["kind"] == "backward" else u, dy, ids)]
    if case["kind"] == "linear":
        return ys[0]
    if case["kind"] == "group":
        return ys
    if case["kind"] == "backward":
        return dxs[0], grads[0], grads[1]
    clipped, norm = _clip64(grads, state["max_norm"])
    return {"y": ys, "dx": dxs, "clipped": clipped, "norm": norm}
