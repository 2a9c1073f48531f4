"""The adapters' oracle against differences and closed forms, and the host-side refusals of the adapter, transposition and clipping calls (CPU)."""
import ctypes

import numpy as np
import pytest

import paper_2602_05367_b200 as rabit
from oracle import adapters_oracle as ao
from oracle import rabit_oracle as orc
from paper_2602_05367_b200 import binding
from synth import make_layer


def _inputs(M=40, N=64, T=7, n=3, r=5, seed=1):
    L = make_layer(M, N, 2, key=(90, seed))
    rng = np.random.default_rng(seed)
    a, b = rng.standard_normal((n, r, N)) / 8, rng.standard_normal((n, r, M)) / 8
    x, ids, scale = rng.standard_normal((T, N)), np.array([0, 2, -1, 0, 3, 2, 0][:T]), rng.uniform(0.5, 2, n)
    return L, a, b, scale, x, ids


def test_rows_without_adapter_are_the_layer_and_the_others_add_a_low_rank_matrix():
    L, a, b, scale, x, ids = _inputs()
    y, u, _, _ = ao.adapted(L.planes, L.g, L.h, a, b, scale, x, ids)
    W = orc.dense_weight(L.planes, L.g, L.h)
    for t, i in enumerate(ids):
        want = W + (scale[i] * b[i].T @ a[i] if 0 <= i < 3 else 0.0)
        assert np.allclose(y[t], want @ x[t], rtol=1e-12, atol=1e-12)
        assert (u[t] == 0).all() == (not 0 <= i < 3)


def test_gradients_are_the_differences_of_the_loss():
    """loss = sum dy * y is linear in x, in a and in b: central differences are exact but for rounding."""
    L, a, b, scale, x, ids = _inputs()
    rng = np.random.default_rng(5)
    dy = rng.standard_normal((x.shape[0], L.M))
    loss = lambda x, a, b: float((dy * ao.adapted(L.planes, L.g, L.h, a, b, scale, x, ids)[0]).sum())  # noqa: E731
    planes_t = np.packbits(orc.unpack_signs(L.planes, L.N).transpose(0, 2, 1)[:, :, :32] < 0, axis=2, bitorder="little")
    assert planes_t.shape == (2, L.N, 4)
    W = orc.dense_weight(L.planes, L.g, L.h)
    _, u, _, _ = ao.adapted(L.planes, L.g, L.h, a, b, scale, x, ids)
    p = np.zeros((x.shape[0], a.shape[1]))
    dx = dy @ W
    for t, i in enumerate(ids):
        if 0 <= i < 3:
            p[t] = b[i] @ dy[t]
            dx[t] += scale[i] * (p[t] @ a[i])
    da, db = ao.gradients(scale, x, p, ids, 3)[0], ao.gradients(scale, dy, u, ids, 3)[0]
    for _ in range(3):
        ex, ea, eb = rng.standard_normal(x.shape), rng.standard_normal(a.shape), rng.standard_normal(b.shape)
        step = 2.0 ** -10
        for got, d in (((dx * ex).sum(), loss(x + step * ex, a, b) - loss(x - step * ex, a, b)), ((da * ea).sum(), loss(x, a + step * ea, b) - loss(x, a - step * ea, b)),
                       ((db * eb).sum(), loss(x, a, b + step * eb) - loss(x, a, b - step * eb))):
            assert abs(got - d / (2 * step)) < 1e-9 * (1 + abs(got))
    assert (da[1] == 0).all() and (db[1] == 0).all()                     # no row names it


def test_clipping_by_the_global_norm():
    outs, norm = ao.clip([np.array([3.0]), np.array([[0.0, 4.0]])], 1.0)
    assert norm == 5.0 and np.allclose(outs[0], 0.6, rtol=1e-6) and np.allclose(outs[1], [[0, 0.8]], rtol=1e-6)
    outs, _ = ao.clip([np.array([3.0, 4.0])], 100.0)
    assert (outs[0] == [3.0, 4.0]).all()


# ---- refusals that need no GPU ---------------------------------------------------------------------------

P = 1 << 20                                                               # an address that is never touched: every call here is refused first


def _struct(**kw):
    v = dict(a=P, b=2 * P, scale=3 * P, count=2, rank=8, n_in=64, n_out=32)
    v.update(kw)
    return binding._AdaptersStruct(*(v[k] for k, _ in binding._AdaptersStruct._fields_))


def _grad_call(struct, **kw):
    v = dict(x=4 * P, u=5 * P, dy=6 * P, p=7 * P, ids=8 * P, da=9 * P, db=10 * P, batch=4)
    v.update(kw)
    return binding.raw_lib().rabit_adapter_gradients(ctypes.byref(struct) if struct is not None else None, v["x"], v["u"], v["dy"], v["p"], v["ids"], v["da"], v["db"],
                                                     v["batch"], 0, None)


@pytest.mark.parametrize("struct,kw,code,word", [
    (None, {}, -1, "null"), ({}, {"x": None}, -1, "null"), ({}, {"da": None}, -1, "null"), ({"a": None}, {}, -1, "null"), ({"count": 0}, {}, -1, "count"),
    ({"rank": 0}, {}, -2, "rank"), ({"rank": 129}, {}, -2, "rank"), ({"n_in": 0}, {}, -1, "positive"), ({"a": P + 8}, {}, -1, "aligned"), ({}, {"batch": 0}, -1, "batch"),
    ({}, {"x": 4 * P + 2}, -1, "aligned"), ({}, {"ids": 8 * P + 1}, -1, "aligned"), ({}, {"db": 9 * P + 1024}, -1, "overlap"), ({}, {"da": 4 * P + 64}, -1, "overlap"),
    ({"scale": 9 * P}, {}, -1, "overlap"),
])
def test_gradient_refusals(struct, kw, code, word):
    assert _grad_call(None if struct is None else _struct(**struct), **kw) == code
    assert word in rabit.last_error()


def test_adapted_refusals_without_a_layer():
    lib, s = binding.raw_lib(), _struct()
    assert lib.rabit_linear_adapted(None, ctypes.byref(s), P, P, P, P, 1, None) == -1 and "null layer" in rabit.last_error()
    assert lib.rabit_linear_adapted(None, None, P, P, P, P, 1, None) == -1 and "adapters" in rabit.last_error()
    assert lib.rabit_linear_group_adapted(None, None, None, None, None, None, 1, 1, None) == -1 and "null array" in rabit.last_error()
    arr = (ctypes.c_void_p * 1)(None)
    assert lib.rabit_linear_group_adapted(arr, arr, arr, P, arr, arr, 0, 1, None) == -1 and "n_layers" in rabit.last_error()
    assert lib.rabit_linear_group_adapted(arr, arr, arr, P, arr, arr, 1, 0, None) == -1 and "batch" in rabit.last_error()
    assert lib.rabit_linear_group_adapted(arr, arr, arr, None, arr, arr, 1, 1, None) == -1 and "ids" in rabit.last_error()
    out = ctypes.c_void_p()
    assert lib.rabit_transpose(None, P, 1 << 30, None, ctypes.byref(out)) == -1 and out.value is None
    assert lib.rabit_transpose(None, P, 1 << 30, None, None) == -1


def _bind(tensors, counts, outs=None, dev_buf=P, dev_bytes=1 << 30):
    n = len(counts)
    c = (ctypes.c_size_t * n)(*counts)
    t = (ctypes.c_void_p * n)(*tensors)
    o = None if outs is None else (ctypes.c_void_p * n)(*outs)
    out = ctypes.c_void_p()
    rc = binding.raw_lib().rabit_gradients_bind(t, o, c, n, dev_buf, dev_bytes, None, ctypes.byref(out))
    assert out.value is None
    return rc


@pytest.mark.parametrize("args,kw,code,word", [
    (([16 * P], [0x10000000000000]), {}, -1, "elements"), (([None], [4]), {}, -1, "null tensor"), (([16 * P + 2], [4]), {}, -1, "misaligned"),
    (([16 * P, 16 * P + 12], [4, 4]), {}, -1, "overlap"), (([16 * P, 32 * P], [4, 4]), {"outs": [48 * P, 32 * P + 4]}, -1, "overlap"),
    (([16 * P, 32 * P], [4, 4]), {"outs": [48 * P, 48 * P]}, -1, "overlap"), (([P + 256], [4]), {}, -1, "overlap"), (([16 * P], [4]), {"dev_bytes": 16}, -3, "need"),
    (([16 * P], [4]), {"dev_buf": P + 8}, -1, "aligned"), (([16 * P], [4]), {"dev_buf": None}, -1, "null"), (([16 * P], [4]), {"outs": [None]}, -1, "null tensor"),
])
def test_gradients_bind_refusals(args, kw, code, word):
    assert _bind(*args, **kw) == code and word in rabit.last_error()


def test_clip_refusals():
    lib = binding.raw_lib()
    assert lib.rabit_clip_gradients(None, 1.0, P, None) == -1
    assert lib.rabit_gradients_free(None) == 0
    assert lib.rabit_gradients_bytes(None, 1) == 0 and lib.rabit_gradients_bytes((ctypes.c_size_t * 1)(5), 0) == 0
    assert lib.rabit_gradients_bytes((ctypes.c_size_t * 2)(0, 5), 2) > 0


def test_more_rows_than_32_bit_places_are_refused():
    lib, s = binding.raw_lib(), _struct()
    for batch in (2 ** 31 - 1, 2 ** 31 - 255):
        assert lib.rabit_linear_adapted(None, ctypes.byref(s), P, P, P, P, batch, None) == -2 and "batch" in rabit.last_error()
