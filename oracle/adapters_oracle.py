"""CPU float64 oracle of the low-rank adapters beside a layer, of their gradients and of gradient clipping.  TEST INFRASTRUCTURE ONLY.

Shares no code with the CUDA path.  Row by row, straight from the definition:

    u[t] = A[id_t] x[t],  y[t] = layer(x[t]) + scale[id_t] B[id_t]^T u[t]          (no adapter: u[t] = 0, y[t] = layer(x[t]))
    da[i] = scale[i] sum_{t: id_t = i} p[t] x[t]^T,  db[i] = scale[i] sum_{t: id_t = i} u[t] dy[t]^T
    clipped = g min(1, max_norm / (norm + 1e-6)),  norm = sqrt(sum g^2)

with a [count][rank][N], b [count][rank][M].  The bounds beside them are what fp32 sums in blocks and the roundings to fp16 allow.
"""
import numpy as np

from oracle import rabit_oracle as orc

STEP32 = 2.0 ** -23          # an fp32 addition that truncates is off by less than this, relative to its result


def _sum_steps(n):
    """Additions that one term of an n-term sum passes through when it is summed in blocks: at most 64 within a block, the rest between blocks of 32."""
    return 64 + n / 32


def adapted(planes, g, h, a, b, scale, x, ids):
    """(y, u, bound of y, bound of u) in float64; y before its rounding to fp16."""
    x, a, b, scale = (np.asarray(v, dtype=np.float64) for v in (x, a, b, scale))
    base = orc.linear(planes, g, h, x)
    l1 = orc.l1_bound(g, h, x)[:, None]
    T, (n, r, N) = x.shape[0], a.shape
    y, u, err_u = base.copy(), np.zeros((T, r)), np.zeros((T, r))
    # the layer's own sum in y: fp16, with the tight bound that its parity tests use
    err = 2.0 ** -10 * np.abs(base) + 1e-5 * l1
    for t in range(T):
        i = int(ids[t])
        if not 0 <= i < n:
            continue
        u[t] = a[i] @ x[t]
        err_u[t] = _sum_steps(N) * STEP32 * (np.abs(a[i]) @ np.abs(x[t])) + 1e-37
        y[t] += scale[i] * (u[t] @ b[i])
        # u enters as two fp16 parts of a power of two of its row: with 22 bits, or to 2^-39 of its largest finite entry (the parts' smallest step is
        # 2^-24 where the largest entry is at least 2^14: rounding is off by half of it, 2^-39 of that entry at most); the sum over the rank and the scaling are fp32
        size = np.abs(u[t][np.isfinite(u[t])]).max(initial=0.0)
        err[t] += abs(scale[i]) * ((err_u[t] + 2.0 ** -39 * size + np.abs(u[t]) * (2.0 ** -21 + (2 * r + 4) * STEP32)) @ np.abs(b[i]))
    with np.errstate(invalid="ignore"):
        err += 2.0 ** -11 * (np.abs(y) + err) + 2.0 ** -24                 # the rounding of y, 2^-25 below the normal numbers
    return y, u, err, err_u


def gradients(scale, v, low, ids, count):
    """Gradient of one factor, [count][rank][side], and its bound: v [T][side] and low [T][rank]."""
    v, low, scale = (np.asarray(w, dtype=np.float64) for w in (v, low, scale))
    out, err = np.zeros((count, low.shape[1], v.shape[1])), np.zeros((count, low.shape[1], v.shape[1]))
    for i in range(count):
        rows = np.flatnonzero(np.asarray(ids) == i)
        if rows.size:
            out[i] = scale[i] * (low[rows].T @ v[rows])
            # low enters as two fp16 parts of a power of two of its rank (see adapted): to 2^-39 of that rank's largest entry at worst
            size = np.abs(low[rows]).max(axis=0)
            err[i] = abs(scale[i]) * ((_sum_steps(rows.size) * STEP32 + 2.0 ** -21) * (np.abs(low[rows]).T @ np.abs(v[rows])) + 2.0 ** -39 * np.outer(size, np.abs(v[rows]).sum(axis=0)))
    return out, err + 1e-37


def clip(grads, max_norm):
    """(clipped arrays, norm)."""
    grads = [np.asarray(v, dtype=np.float64) for v in grads]
    norm = float(np.sqrt(sum(float((v * v).sum()) for v in grads)))
    factor = min(1.0, max_norm / (norm + 1e-6))
    return [v * factor for v in grads], norm
