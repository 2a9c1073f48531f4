"""Low-rank adapters beside a layer, the gradients of their factors, the transposed layer and gradient clipping, against the float64 oracle."""
import ctypes

import numpy as np
import pytest

from oracle import adapters_oracle as ao
from oracle import rabit_oracle as orc
from synth import make_layer, make_x

pytestmark = pytest.mark.gpu


def _pool(M, N, n, r, seed):
    rng = np.random.default_rng([7, seed, M, N, n, r])
    a = (rng.standard_normal((n, r, N)) / np.sqrt(N)).astype(np.float16)
    b = (rng.standard_normal((n, r, M)) * 0.1).astype(np.float16)
    return a, b, rng.uniform(0.5, 2.0, n).astype(np.float32)


def _ids(batch, n, kind, seed=0):
    rng = np.random.default_rng([8, batch, n, seed])
    if kind == "one":
        return np.full(batch, n - 1, np.int32)
    if kind == "none":
        return np.full(batch, -1, np.int32)
    if kind == "prompts":
        return np.sort(rng.integers(-1, n, batch)).astype(np.int32)[::-1].copy()
    return rng.choice(np.array([-7, -1, n, n + 5] + 3 * list(range(n)), np.int32), batch).astype(np.int32)   # "mixed": also ids outside the pool


def _cuda(*arrays):
    import torch
    return [torch.from_numpy(np.ascontiguousarray(v)).cuda() for v in arrays]


def _adapters(a, b, scale):
    import paper_2602_05367_b200 as rabit
    return rabit.RabitAdapters(*_cuda(a, b, scale))


def _transposed_planes(L):
    bits = ((L.planes[..., None] >> np.arange(32, dtype=np.uint32)) & 1).astype(np.uint8).reshape(L.K, L.M, L.N).transpose(0, 2, 1)
    return np.ascontiguousarray(np.packbits(np.ascontiguousarray(bits), axis=2, bitorder="little")).view(np.uint32)


def _within(got, want, bound, what):
    got = got.astype(np.float64)
    assert got.shape == want.shape
    off = ~(np.abs(got - want) <= bound)                                    # (a NaN is off)
    if off.any():
        at = tuple(np.argwhere(off)[0])
        raise AssertionError(f"{what}{list(at)}: {got[at]:.8g}, want {want[at]:.8g}, off {abs(got[at] - want[at]):.3g} > {bound[at]:.3g} ({int(off.sum())} of {off.size})")


CASES = [(2, 128, 64, 1, 8, 2, "one"), (1, 33, 32, 2, 1, 1, "one"), (2, 100, 160, 3, 3, 4, "mixed"), (3, 129, 1184, 5, 16, 3, "mixed"), (2, 256, 512, 8, 12, 9, "mixed"),
         (2, 1000, 96, 9, 17, 3, "mixed"), (2, 72, 2080, 16, 64, 16, "mixed"), (2, 520, 1024, 17, 16, 4, "prompts"), (1, 1031, 640, 31, 128, 2, "mixed"), (2, 300, 4096, 33, 8, 40, "mixed"),
         (2, 264, 736, 64, 33, 3, "prompts"), (3, 136, 320, 65, 16, 5, "mixed"), (2, 520, 256, 128, 64, 2, "one"), (2, 97, 288, 130, 5, 7, "mixed"), (2, 640, 1056, 257, 16, 3, "prompts"),
         (2, 200, 544, 515, 100, 2, "prompts"), (1, 64, 8224, 12, 24, 3, "mixed"), (2, 128, 128, 40, 16, 2, "none"), (2, 1032, 64, 300, 128, 5, "mixed"), (2, 96, 160, 2100, 24, 3, "prompts"),
         (1, 40, 416, 600, 70, 4, "mixed"), (1, 264, 96, 2500, 16, 2, "mixed"), (2, 33, 352, 480, 40, 3, "prompts"), (3, 100, 224, 90, 9, 30, "mixed"), (2, 1000, 288, 48, 20, 50, "mixed")]


@pytest.mark.parametrize("K,M,N,batch,r,n,kind", CASES)
def test_adapted_linear(K, M, N, batch, r, n, kind):
    import torch
    import paper_2602_05367_b200 as rabit
    L = make_layer(M, N, K, key=(91, K, M, N))
    a, b, scale = _pool(M, N, n, r, 1)
    x, ids = make_x(batch, N, key=(91, batch, N)), _ids(batch, n, kind)
    layer, A = rabit.rabit_pack(L.planes, L.g, L.h), _adapters(a, b, scale)
    xd, idd = _cuda(x, ids)
    want, want_u, err, err_u = ao.adapted(L.planes, L.g, L.h, a, b, scale, x, ids)
    buf = torch.full((batch + 2, M), 7.0, dtype=torch.float16, device="cuda")           # rows behind the last stay as they were
    ubuf = torch.full((batch + 2, r), 7.0, dtype=torch.float32, device="cuda")
    first = None
    for rep in range(2):
        y = rabit.rabit_linear_adapted(layer, A, xd, idd, buf[:batch], ubuf[:batch])
        torch.cuda.synchronize()
        _within(y.cpu().numpy(), want, err, "y")
        _within(ubuf[:batch].cpu().numpy(), want_u, err_u, "u")
        assert (buf[batch:] == 7.0).all() and (ubuf[batch:] == 7.0).all()
        assert first is None or torch.equal(first, y)                                  # the same bits every time
        first = y.clone()
    y2 = rabit.rabit_linear_adapted(layer, A, xd, idd)
    torch.cuda.synchronize()
    assert torch.equal(y2, first) and layer.status() == 0
    bare = ~((ids >= 0) & (ids < n))
    assert np.array_equal(first.cpu().numpy()[bare], rabit.rabit_linear(layer, xd).cpu().numpy()[bare])   # bit for bit the layer
    layer.free()


@pytest.mark.parametrize("K,M,N,batch,r,n,kind", [
    (2, 20008, 64, 70, 8, 3, "mixed"), (1, 9001, 96, 130, 16, 2, "prompts"), (2, 10504, 32, 200, 24, 3, "prompts"), (1, 9003, 64, 150, 31, 4, "mixed"), (1, 12000, 64, 100, 60, 4, "mixed"),
    (1, 8209, 32, 129, 64, 2, "one"), (2, 8200, 32, 257, 100, 2, "mixed"), (1, 8191, 96, 300, 128, 2, "prompts"), (2, 5008, 288, 513, 12, 9, "mixed"), (1, 4104, 64, 700, 16, 3, "mixed"),
    (1, 2003, 64, 1100, 30, 3, "mixed"), (1, 2000, 160, 1500, 70, 3, "prompts"), (2, 1200, 64, 1030, 110, 2, "prompts"), (1, 520, 64, 2050, 50, 3, "mixed"), (1, 264, 96, 2049, 128, 2, "prompts"),
    (1, 261, 96, 2049, 16, 40, "mixed"), (1, 9000, 64, 600, 16, 3, "none")])
def test_adapted_linear_in_two_launches(K, M, N, batch, r, n, kind):
    """Rows times outputs beyond what one launch behind the layer takes, in all tile heights and ranks."""
    test_adapted_linear(K, M, N, batch, r, n, kind)


@pytest.mark.parametrize("batch", [130, 1025, 2050])
def test_more_rows_of_a_group_and_what_is_not_finite(batch):
    test_adapted_group_with_unlike_ranks_and_a_layer_without(batch)
    test_what_is_not_finite_stays_in_its_rows(batch)


def test_one_flat_row():
    import torch
    import paper_2602_05367_b200 as rabit
    L = make_layer(96, 64, 2, key=(92,))
    a, b, scale = _pool(96, 64, 2, 4, 2)
    x = make_x(1, 64, key=(92, 1))
    layer, A = rabit.rabit_pack(L.planes, L.g, L.h), _adapters(a, b, scale)
    xd, ids = _cuda(x, np.array([1], np.int32))
    y = rabit.rabit_linear_adapted(layer, A, xd[0], ids)
    assert y.shape == (96,)
    want, _, err, _ = ao.adapted(L.planes, L.g, L.h, a, b, scale, x, [1])
    _within(y.cpu().numpy()[None], want, err, "y")
    layer.free()


@pytest.mark.parametrize("batch", [1, 2, 6, 13, 16, 70])
def test_adapted_group_with_unlike_ranks_and_a_layer_without(batch):
    import torch
    import paper_2602_05367_b200 as rabit
    specs = [(520, 16, 3), (128, 3, 5), (200, 0, 0), (136, 64, 3)]
    N, Ls = 544, []
    x = make_x(batch, N, key=(93, batch))
    ids = _ids(batch, 3, "mixed")
    xd, idd = _cuda(x, ids)
    layers, pools, ys, us, wants = [], [], [], [], []
    for i, (M, r, n) in enumerate(specs):
        L = make_layer(M, N, 2, key=(93, i))
        layers.append(rabit.rabit_pack(L.planes, L.g, L.h))
        ys.append(torch.zeros((batch, M), dtype=torch.float16, device="cuda"))
        if r:
            pool = _pool(M, N, n, r, i)
            pools.append(_adapters(*pool))
            us.append(torch.zeros((batch, r), dtype=torch.float32, device="cuda") if i != 1 else None)
            wants.append(ao.adapted(L.planes, L.g, L.h, *pool, x, ids))
        else:
            pools.append(None)
            us.append(None)
            wants.append(ao.adapted(L.planes, L.g, L.h, *_pool(M, N, 1, 1, 0), x, np.full(batch, -1)))
    for give_u in (us, None):
        rabit.rabit_linear_group_adapted(layers, pools, [xd] * 4, idd, ys, give_u)
        torch.cuda.synchronize()
        for y, u, (want, want_u, err, err_u) in zip(ys, us, wants):
            _within(y.cpu().numpy(), want, err, "y")
            if u is not None:
                _within(u.cpu().numpy(), want_u, err_u, "u")
    for layer in layers:
        layer.free()


def test_more_layers_than_a_launch_takes():
    import torch
    import paper_2602_05367_b200 as rabit
    N, batch = 96, 3
    x, ids = make_x(batch, N, key=(94,)), _ids(batch, 2, "one")
    xd, idd = _cuda(x, ids)
    Ls = [make_layer(32 + 8 * i, N, 2, key=(94, i)) for i in range(19)]
    pools = [_pool(L.M, N, 2, 1 + i, i) for i, L in enumerate(Ls)]
    layers = [rabit.rabit_pack(L.planes, L.g, L.h) for L in Ls]
    ys = [torch.zeros((batch, L.M), dtype=torch.float16, device="cuda") for L in Ls]
    rabit.rabit_linear_group_adapted(layers, [_adapters(*p) for p in pools], [xd] * 19, idd, ys)
    torch.cuda.synchronize()
    for L, p, y in zip(Ls, pools, ys):
        want, _, err, _ = ao.adapted(L.planes, L.g, L.h, *p, x, ids)
        _within(y.cpu().numpy(), want, err, "y")
    for layer in layers:
        layer.free()


@pytest.mark.parametrize("batch", [5, 40, 300])
def test_what_is_not_finite_stays_in_its_rows(batch):
    """NaN and infinities in a row of x, in an adapter, in one that no row names: only the rows that they belong to see them."""
    import torch
    import paper_2602_05367_b200 as rabit
    M, N, n, r = 136, 160, 4, 12
    L = make_layer(M, N, 2, key=(95,))
    a, b, scale = _pool(M, N, n, r, 3)
    x, ids = make_x(batch, N, key=(95, batch)), np.array([0, 1, 2, -1, 0] * (batch // 5), np.int32)
    layer = rabit.rabit_pack(L.planes, L.g, L.h)
    want, want_u, err, err_u = ao.adapted(L.planes, L.g, L.h, a, b, scale, x, ids)
    x[3, 5] = np.nan                                                                    # a row without adapter
    x[4, 7] = np.inf
    a[3], b[3] = np.nan, np.inf                                                         # named by no row
    b[1, 2] = -np.inf
    a[2, :, 9] = np.nan
    u = torch.empty((batch, r), dtype=torch.float32, device="cuda")
    y = rabit.rabit_linear_adapted(layer, _adapters(a, b, scale), *_cuda(x, ids), None, u)
    torch.cuda.synchronize()
    y, u = y.cpu().numpy(), u.cpu().numpy()
    clean = ids == 0
    clean[4] = False
    bare = ids == -1
    bare[3] = False
    _within(y[clean | bare], want[clean | bare], err[clean | bare], "y")
    _within(u[clean | bare], want_u[clean | bare], err_u[clean | bare], "u")
    assert (u[3] == 0).all() and not np.isfinite(y[3]).any() and not np.isfinite(y[4]).any()
    _within(u[ids == 1], want_u[ids == 1], err_u[ids == 1], "u")
    assert not np.isfinite(y[ids == 1]).any() and np.isnan(y[ids == 2]).all() and np.isnan(u[ids == 2]).all()
    layer.free()


def test_low_rank_products_of_any_size():
    """u beyond fp16's range, and far below it, beside ordinary ones."""
    import torch
    import paper_2602_05367_b200 as rabit
    M, N, r = 64, 256, 8
    L = make_layer(M, N, 1, key=(96,))
    for batch in (3, 100):
        a, b, scale = _pool(M, N, 1, r, 4)
        x = make_x(batch, N, key=(96, batch))
        a[0, 0], a[0, 1], b[0, 0], b[0, 1] = 6e4 * np.sign(x[0]).astype(np.float16), 1e-7, 6e-8, 1.0
        x[1] *= np.float16(100)
        x[2] *= np.float16(1e-3)
        ids = np.zeros(batch, np.int32)
        layer = rabit.rabit_pack(L.planes, L.g, L.h)
        u = torch.empty((batch, r), dtype=torch.float32, device="cuda")
        y = rabit.rabit_linear_adapted(layer, _adapters(a, b, scale), *_cuda(x, ids), None, u)
        want, want_u, err, err_u = ao.adapted(L.planes, L.g, L.h, a, b, scale, x, ids)
        assert np.abs(want_u).max() > 65504
        _within(u.cpu().numpy(), want_u, err_u, "u")
        _within(y.cpu().numpy(), want, err, "y")
        layer.free()


def test_captured_replayed_and_on_another_stream():
    import torch
    import paper_2602_05367_b200 as rabit
    M, N, n, r = 520, 1056, 3, 16
    L = make_layer(M, N, 2, key=(97,))
    pool = _pool(M, N, n, r, 5)
    layer, A = rabit.rabit_pack(L.planes, L.g, L.h), _adapters(*pool)
    for batch in (2, 11, 200):
        x, ids = make_x(batch, N, key=(97, batch)), _ids(batch, n, "mixed")
        xd, idd = _cuda(x, ids)
        y, u = torch.zeros((batch, M), dtype=torch.float16, device="cuda"), torch.zeros((batch, r), dtype=torch.float32, device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        rabit.rabit_linear_adapted(layer, A, xd, idd, y, None, s.cuda_stream)            # an explicit stream, u from the allocator
        s.synchronize()
        want, want_u, err, err_u = ao.adapted(L.planes, L.g, L.h, *pool, x, ids)
        _within(y.cpu().numpy(), want, err, "y")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            rabit.rabit_linear_adapted(layer, A, xd, idd, y, u)
        for rep in range(3):                                                            # new activations and ids in place
            x2, ids2 = make_x(batch, N, key=(97, batch, rep)), _ids(batch, n, "mixed", rep + 1)
            for t, v in zip((xd, idd), _cuda(x2, ids2)):
                t.copy_(v)
            graph.replay()
            torch.cuda.synchronize()
            want, want_u, err, err_u = ao.adapted(L.planes, L.g, L.h, *pool, x2, ids2)
            _within(y.cpu().numpy(), want, err, "y")
            _within(u.cpu().numpy(), want_u, err_u, "u")
    layer.free()


@pytest.mark.parametrize("variant,batch,r,kind", [(0, 1, 16, "one"), (0, 7, 16, "mixed"), (0, 12, 16, "mixed"), (0, 48, 40, "mixed"), (0, 48, 16, "none"), (0, 200, 16, "none"), (0, 300, 16, "mixed"),
                                                  (0, 1100, 64, "prompts"), (0, 1100, 64, "none"), (1, 70, 16, "mixed"), (2, 12, 16, "mixed"), (3, 12, 16, "mixed"),
                                                  (4, 300, 128, "prompts"), (5, 300, 16, "prompts"), (6, 300, 16, "mixed")])
def test_a_chain_of_calls_without_a_stop_between(variant, batch, r, kind):
    """Each call's y is the next one's x, u is shared, and ids and factors change by copies on the stream: kernels that start while those before them run see all of it."""
    import torch
    import paper_2602_05367_b200 as rabit
    side, n, steps = 512, 3, 6
    L = make_layer(side, side, 2, key=(98,))
    layer = rabit.rabit_pack(L.planes, (L.g.astype(np.float32) / 16).astype(np.float16), L.h)
    if variant:
        layer.set_variant(variant)
    (xd,) = _cuda(make_x(batch, side, key=(98, batch)))
    pools = [_cuda(*_pool(side, side, n, r, 11 + k)) for k in range(2)]
    ids = [_cuda(_ids(batch, n, kind, k))[0] for k in range(2)]
    s, outs = torch.cuda.Stream(), {}
    torch.cuda.synchronize()
    for stop in (True, False):
        A, at = rabit.RabitAdapters(*[t.clone() for t in pools[0]]), ids[0].clone()
        ys = [torch.zeros((batch, side), dtype=torch.float16, device="cuda") for _ in range(steps)]
        u, us = torch.zeros((batch, r), device="cuda"), torch.zeros((steps, batch, r), device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for k in range(steps):
                if k == 3:                                                              # calls 0-2 and 3-5 follow one another without anything between but the calls
                    at.copy_(ids[1])
                    for t, v in zip((A.a, A.b, A.scale), pools[1]):
                        t.copy_(v)
                rabit.rabit_linear_adapted(layer, A, ys[k - 1] if k else xd, at, ys[k], u if k % 3 != 2 else us[k])
                if stop:
                    s.synchronize()
        torch.cuda.synchronize()
        outs[stop] = [t.cpu().numpy() for t in ys] + [us.cpu().numpy(), u.cpu().numpy()]
    assert all(np.isfinite(v).all() for v in outs[True][:steps]) and (outs[True][0] != 0).any()   # (rows without adapter shrink from call to call)
    for k, (a, b) in enumerate(zip(outs[True], outs[False])):
        assert np.array_equal(a, b), k
    layer.free()



@pytest.mark.parametrize("batch,r,kind", [(5, 16, "mixed"), (40, 16, "mixed"), (40, 16, "none"), (1100, 64, "prompts"), (1100, 16, "none")])
def test_a_captured_chain_of_calls(batch, r, kind):
    """The same kernels beside one another in a replayed graph: bit for bit the calls one by one."""
    import torch
    import paper_2602_05367_b200 as rabit
    side, n, steps = 512, 3, 4
    L = make_layer(side, side, 2, key=(98,))
    layer, A = rabit.rabit_pack(L.planes, (L.g.astype(np.float32) / 16).astype(np.float16), L.h), _adapters(*_pool(side, side, n, r, 13))
    xd, idd = _cuda(make_x(batch, side, key=(99, batch)), _ids(batch, n, kind))
    ys = [torch.zeros((batch, side), dtype=torch.float16, device="cuda") for _ in range(steps)]
    u, s, graph = torch.zeros((batch, r), device="cuda"), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        for k in range(steps):
            rabit.rabit_linear_adapted(layer, A, ys[k - 1] if k else xd, idd, ys[k], u)
    for rep in range(3):
        x = _cuda(make_x(batch, side, key=(99, batch, rep)))[0]
        want = [x]
        for k in range(steps):
            want.append(rabit.rabit_linear_adapted(layer, A, want[-1], idd))
            torch.cuda.synchronize()
        xd.copy_(x)
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ys, want[1:]))
    layer.free()


def test_offsets_beyond_32_bits():
    """A pool of 4.4 GB whose last adapter is named, and its gradient of 8.8 GB."""
    import torch
    import paper_2602_05367_b200 as rabit
    M, N, r, n = 64, 8192, 64, 4200
    L = make_layer(M, N, 1, key=(102,))
    a, b, _ = _pool(M, N, 1, r, 30)
    big, out = torch.zeros((n, r, N), dtype=torch.float16, device="cuda"), torch.zeros((n, r, M), dtype=torch.float16, device="cuda")
    big[-1], out[-1] = _cuda(a[0], b[0])
    scale = torch.full((n,), 1.5, device="cuda")
    A, layer = rabit.RabitAdapters(big, out, scale), rabit.rabit_pack(L.planes, L.g, L.h)
    for batch in (3, 70, 300):
        x = make_x(batch, N, key=(102, batch))
        ids = np.full(batch, n - 1, np.int32)
        u = torch.empty((batch, r), dtype=torch.float32, device="cuda")
        y = rabit.rabit_linear_adapted(layer, A, *_cuda(x, ids), None, u)
        want, want_u, err, err_u = ao.adapted(L.planes, L.g, L.h, a, b, [1.5], x, np.zeros(batch, np.int32))
        _within(y.cpu().numpy(), want, err, "y")
        _within(u.cpu().numpy(), want_u, err_u, "u")
    rng = np.random.default_rng(31)
    dy, p = rng.standard_normal((batch, M)).astype(np.float16), rng.standard_normal((batch, r)).astype(np.float32)
    da, db = rabit.rabit_adapter_gradients(A, *_cuda(x, u.cpu().numpy(), dy, p, ids))
    _within(da[-1].cpu().numpy()[None], *ao.gradients([1.5], x, p, np.zeros(batch, np.int32), 1), "da")
    _within(db[-1].cpu().numpy()[None], *ao.gradients([1.5], dy, u.cpu().numpy(), np.zeros(batch, np.int32), 1), "db")
    assert not da[:-1].any() and not db[:-1].any()
    layer.free()


def test_infinite_x_beside_a_rank_that_is_no_multiple():
    """One rank, one infinity: y is infinite where the factors are not zero, not NaN."""
    import torch
    import paper_2602_05367_b200 as rabit
    M, N = 64, 96
    L = make_layer(M, N, 1, key=(103,))
    L.planes[:] = 0
    a, b, scale = np.ones((1, 1, N), np.float16), np.ones((1, 1, M), np.float16), np.ones(1, np.float32)
    layer = rabit.rabit_pack(L.planes, L.g, L.h)
    for batch in (1, 100, 400):
        x = np.abs(make_x(batch, N, key=(103, batch)))
        x[0, 0] = np.inf
        u = torch.empty((batch, 1), dtype=torch.float32, device="cuda")
        y = rabit.rabit_linear_adapted(layer, _adapters(a, b, scale), *_cuda(x, np.zeros(batch, np.int32)), None, u)
        base = rabit.rabit_linear(layer, *_cuda(x))
        torch.cuda.synchronize()
        assert torch.isinf(u[0]).all() and (u[1:] < 1e5).all()
        assert torch.isfinite(y[1:]).all() and not torch.isfinite(y[0]).any()
        assert torch.equal(torch.isnan(y[0]), torch.isnan(base[0]))
    layer.free()


def test_adapted_refusals():
    import torch
    import paper_2602_05367_b200 as rabit
    from paper_2602_05367_b200 import binding
    M, N, n, r, batch = 64, 96, 2, 4, 3
    L = make_layer(M, N, 2, key=(98,))
    layer, A = rabit.rabit_pack(L.planes, L.g, L.h), _adapters(*_pool(M, N, n, r, 6))
    xd, idd = _cuda(make_x(batch, N, key=(98,)), np.zeros(batch, np.int32))
    for bad in (dict(x=xd.float()), dict(x=xd[:, :64]), dict(ids=idd.long()), dict(ids=idd[:2]), dict(ids=idd.cpu()), dict(y=torch.empty((batch, N), dtype=torch.float16, device="cuda")),
                dict(u=torch.empty((batch, r), dtype=torch.float16, device="cuda")), dict(u=torch.empty((batch, r + 1), dtype=torch.float32, device="cuda"))):
        kw = dict(dict(x=xd, ids=idd, y=None, u=None), **bad)
        with pytest.raises(ValueError):
            rabit.rabit_linear_adapted(layer, A, kw["x"], kw["ids"], kw["y"], kw["u"])
    for a, b, s in ((A.a.float(), A.b, A.scale), (A.a, A.b[:1], A.scale), (A.a, A.b, A.scale[:1]), (A.a.cpu(), A.b, A.scale), (A.a.transpose(1, 2), A.b, A.scale), (A.a, A.b, A.scale.half())):
        with pytest.raises(ValueError):
            rabit.RabitAdapters(a, b, s)
    other = _adapters(*_pool(M + 8, N, n, r, 6))
    with pytest.raises(rabit.RabitError, match="beside a layer"):
        rabit.rabit_linear_adapted(layer, other, xd, idd)
    wide = rabit.RabitAdapters(torch.zeros((1, 129, N), dtype=torch.float16, device="cuda"), torch.zeros((1, 129, M), dtype=torch.float16, device="cuda"), A.scale[:1])
    with pytest.raises(rabit.RabitError, match="rank"):
        rabit.rabit_linear_adapted(layer, wide, xd, torch.zeros_like(idd))
    lib, vp = binding.raw_lib(), ctypes.c_void_p
    y, u = torch.zeros((batch, M), dtype=torch.float16, device="cuda"), torch.zeros((batch, r), dtype=torch.float32, device="cuda")
    def call(x=xd.data_ptr(), ids=idd.data_ptr(), y=y.data_ptr(), u=u.data_ptr(), batch=batch):
        return lib.rabit_linear_adapted(layer.handle, vp(A._addr), vp(x), vp(ids), vp(y), vp(u), batch, None)
    assert call() == 0
    assert call(batch=0) == -1
    for kw in (dict(u=None), dict(u=u.data_ptr() + 4), dict(ids=None), dict(ids=idd.data_ptr() + 2), dict(y=A.a.data_ptr()), dict(u=A.b.data_ptr()), dict(u=xd.data_ptr()), dict(u=y.data_ptr()),
               dict(y=u.data_ptr()), dict(y=xd.data_ptr()), dict(x=xd.data_ptr() + 2), dict(y=y.data_ptr() + 2)):
        assert call(**kw) == -1, kw
    torch.cuda.synchronize()
    layer.free()
    with pytest.raises(rabit.RabitError):
        rabit.rabit_linear_adapted(layer, A, xd, idd)


@pytest.mark.parametrize("K,M,N", [(1, 32, 32), (2, 96, 160), (3, 160, 640), (2, 1024, 96), (2, 288, 2080), (1, 32, 1000 * 32), (2, 4096, 1024)])
def test_transposed_layer_is_the_pack_of_the_transposed_planes(K, M, N):
    import torch
    import paper_2602_05367_b200 as rabit
    L = make_layer(M, N, K, key=(99, K, M, N))
    planes_t = _transposed_planes(L)
    layer = rabit.rabit_pack(L.planes, L.g, L.h)
    turned = rabit.rabit_transpose(layer)
    assert (turned.K, turned.M, turned.N) == (K, N, M)
    assert np.array_equal(turned.dev_buf.cpu().numpy(), rabit.pack_host(planes_t, L.h, L.g))
    dy = make_x(2, M, key=(99, M))
    got = rabit.rabit_linear(turned, *_cuda(dy)).cpu().numpy().astype(np.float64)
    assert (np.abs(got - dy.astype(np.float64) @ orc.dense_weight(L.planes, L.g, L.h)).max(axis=1) <= orc.tolerance(L.h, L.g, dy)).all()
    again = rabit.rabit_transpose(turned)
    assert torch.equal(again.dev_buf, layer.dev_buf)
    for v in (layer, turned, again):
        v.free()


def test_transpose_refusals():
    import torch
    import paper_2602_05367_b200 as rabit
    from paper_2602_05367_b200 import binding
    L = make_layer(40, 64, 2, key=(100,))
    layer = rabit.rabit_pack(L.planes, L.g, L.h)
    with pytest.raises(rabit.RabitError, match="multiple of 32"):
        rabit.rabit_transpose(layer)
    layer.free()
    L = make_layer(64, 96, 2, key=(100,))
    layer = rabit.rabit_pack(L.planes, L.g, L.h)
    lib, out, vp = binding.raw_lib(), ctypes.c_void_p(), ctypes.c_void_p
    size = rabit.packed_bytes(2, 96, 64)
    buf = torch.zeros(size + 256, dtype=torch.uint8, device="cuda")
    assert lib.rabit_transpose(layer.handle, vp(buf.data_ptr()), size - 1, None, ctypes.byref(out)) == -3
    assert lib.rabit_transpose(layer.handle, vp(buf.data_ptr() + 16), size, None, ctypes.byref(out)) == -1
    assert lib.rabit_transpose(layer.handle, vp(layer.dev_buf.data_ptr()), size, None, ctypes.byref(out)) == -1
    host = torch.zeros(size + 256, dtype=torch.uint8)
    assert lib.rabit_transpose(layer.handle, vp((host.data_ptr() + 255) // 256 * 256), size, None, ctypes.byref(out)) == -1
    s = torch.cuda.Stream()
    x = torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=s):
        x.add_(1)
        assert lib.rabit_transpose(layer.handle, vp(buf.data_ptr()), size, vp(s.cuda_stream), ctypes.byref(out)) == -1 and "captured" in rabit.last_error()
    torch.cuda.synchronize()
    assert out.value is None
    layer.free()


GRADIENT_CASES = [(32, 64, 1, 1, 1, "one"), (64, 32, 3, 8, 2, "mixed"), (1000, 96, 17, 16, 3, "mixed"), (33, 104, 40, 5, 4, "mixed"), (264, 640, 64, 33, 2, "prompts"),
                  (128, 1056, 77, 64, 3, "mixed"), (136, 320, 300, 128, 2, "prompts"), (256, 520, 1000, 16, 1, "one"), (96, 64, 2500, 12, 5, "prompts"), (72, 200, 513, 17, 9, "mixed"), (64, 64, 20, 16, 2, "none"), (64, 96, 9000, 8, 1, "one"), (40, 72, 9000, 40, 3, "mixed"),
                  (36, 44, 700, 7, 60, "mixed")]


@pytest.mark.parametrize("M,N,batch,r,n,kind", GRADIENT_CASES)
def test_factor_gradients(M, N, batch, r, n, kind):
    import torch
    import paper_2602_05367_b200 as rabit
    rng = np.random.default_rng([9, M, N, batch, r])
    a, b, scale = _pool(M, N, n, r, 7)
    x, dy = rng.standard_normal((batch, N)).astype(np.float16), (0.1 * rng.standard_normal((batch, M))).astype(np.float16)
    u, p = rng.standard_normal((batch, r)).astype(np.float32), (0.1 * rng.standard_normal((batch, r))).astype(np.float32)
    ids = _ids(batch, n, kind)
    bare = ~((ids >= 0) & (ids < n))
    want = ao.gradients(scale, x, p, ids, n), ao.gradients(scale, dy, u, ids, n)
    x[bare], dy[bare], u[bare], p[bare] = np.nan, np.inf, np.nan, -np.inf                 # rows without adapter: whatever they hold
    A = _adapters(a, b, scale)
    args = _cuda(x, u, dy, p, ids)
    guard = [torch.full((n * r * side + 64,), 3.0, dtype=torch.float32, device="cuda") for side in (N, M)]
    da, db = (g[:n * r * side].view(n, r, side) for g, side in zip(guard, (N, M)))
    rabit.rabit_adapter_gradients(A, *args, da, db)
    torch.cuda.synchronize()
    for got, (w, err), g in zip((da, db), want, guard):
        _within(got.cpu().numpy(), w, err, "gradient")
        assert (g[-64:] == 3.0).all()
    first = da.clone(), db.clone()
    da2, db2 = rabit.rabit_adapter_gradients(A, *args)
    assert torch.equal(da2, first[0]) and torch.equal(db2, first[1])                     # the same bits every time
    rabit.rabit_adapter_gradients(A, *args, da, db, accumulate=True)                     # what is there plus the same again: twice it, one rounding
    torch.cuda.synchronize()
    for got, (w, err) in zip((da, db), want):
        _within(got.cpu().numpy(), 2 * w, 2 * err + 2.0 ** -22 * np.abs(w), "accumulated")


def test_factor_gradients_of_unlike_magnitudes():
    """Rows, ranks and columns of very different sizes: each element is held to its own sum of magnitudes."""
    import torch
    import paper_2602_05367_b200 as rabit
    M, N, batch, r, n = 64, 96, 200, 8, 1
    rng = np.random.default_rng(10)
    a, b, scale = _pool(M, N, n, r, 8)
    x, dy = rng.standard_normal((batch, N)).astype(np.float16), rng.standard_normal((batch, M)).astype(np.float16)
    u = (rng.standard_normal((batch, r)) * 10.0 ** rng.uniform(-12, 12, (batch, 1)) * 10.0 ** rng.uniform(-6, 6, (1, r))).astype(np.float32)
    x[rng.random(x.shape) < 0.5] = 0
    dy[rng.random(dy.shape) < 0.5] = 0
    ids = np.zeros(batch, np.int32)
    da, db = rabit.rabit_adapter_gradients(_adapters(a, b, scale), *_cuda(x, u, dy, u, ids))
    for got, v in ((da, x), (db, dy)):
        _within(got.cpu().numpy(), *ao.gradients(scale, v, u, ids, n), "gradient")


def test_gradient_argument_checks_and_other_stream():
    import torch
    import paper_2602_05367_b200 as rabit
    M, N, batch, r, n = 32, 64, 6, 4, 2
    A = _adapters(*_pool(M, N, n, r, 9))
    rng = np.random.default_rng(11)
    arrays = rng.standard_normal((batch, N)).astype(np.float16), rng.standard_normal((batch, r)).astype(np.float32), rng.standard_normal((batch, M)).astype(np.float16), \
        rng.standard_normal((batch, r)).astype(np.float32), np.array([0, 1, 1, -1, 0, 1], np.int32)
    good = _cuda(*arrays)
    for i in range(5):
        for bad in (good[i].cpu(), good[i][:3], good[i].double()):
            with pytest.raises((ValueError, rabit.RabitError)):
                rabit.rabit_adapter_gradients(A, *[bad if j == i else v for j, v in enumerate(good)])
    with pytest.raises(ValueError):
        rabit.rabit_adapter_gradients(A, *good, accumulate=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    da, db = torch.zeros(A.a.shape, device="cuda"), torch.zeros(A.b.shape, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        rabit.rabit_adapter_gradients(A, *good, da, db, True)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for got, v, low in ((da, arrays[0], arrays[3]), (db, arrays[2], arrays[1])):
        w, err = ao.gradients(A.scale.cpu().numpy(), v, low, arrays[4], n)
        _within(got.cpu().numpy(), 3 * w, 3 * err + 2.0 ** -21 * np.abs(w), "gradient")


CLIP_SIZES = [[1], [3, 0, 5], [8191, 8192, 8193, 1], [70000, 2, 40000], [0], [1] * 700, [1 << 21, 12345]]


@pytest.mark.parametrize("sizes", CLIP_SIZES, ids=str)
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("shift", [0, 1])
def test_clipping(sizes, in_place, shift):
    """Tensors that start on 16 bytes or 4 bytes behind, clipped and not."""
    import torch
    import paper_2602_05367_b200 as rabit
    rng = np.random.default_rng([12] + sizes[:4])
    flats = [rng.standard_normal(n).astype(np.float32) for n in sizes]
    for max_norm in (0.37, 1e9):
        want, norm = ao.clip(flats, max_norm)
        hold = [torch.full((n + 8,), 5.0, device="cuda") for n in sizes]
        tensors = [h[shift:shift + n] for h, n in zip(hold, sizes)]
        for t, v in zip(tensors, flats):
            t.copy_(torch.from_numpy(v))
        outs = None if in_place else [torch.full((n + 8,), 5.0, device="cuda") for n in sizes]
        G = rabit.RabitGradients(tensors, None if in_place else [o[2 - 2 * shift:2 - 2 * shift + n] for o, n in zip(outs, sizes)])
        got_norm = rabit.rabit_clip_gradients(G, max_norm)
        torch.cuda.synchronize()
        assert abs(float(got_norm) - norm) <= 2.0 ** -23 * norm
        for i, (w, v, n) in enumerate(zip(want, flats, sizes)):
            at = shift if in_place else 2 - 2 * shift
            whole = (hold if in_place else outs)[i].cpu().numpy()
            got = whole[at:at + n]
            # the factor and the product are rounded once each; 2^-149 is the smallest step of all
            assert (np.abs(got - w) <= 2.0 ** -22 * np.abs(w) + 2.0 ** -149).all()
            if norm < max_norm:
                assert np.array_equal(got, v)
            assert (np.delete(whole, np.arange(at, at + n)) == 5.0).all()
            if not in_place:
                assert np.array_equal(tensors[i].cpu().numpy(), v)
        G.free()


def test_clipping_of_large_infinite_and_nan_gradients():
    import torch
    import paper_2602_05367_b200 as rabit
    big = torch.tensor([3e30, -4e30, 1e-30], device="cuda")
    G = rabit.RabitGradients([big])
    assert abs(float(rabit.rabit_clip_gradients(G, 1.0)) / 5e30 - 1) < 1e-6
    assert np.allclose(big.cpu().numpy()[:2], [0.6, -0.8], rtol=1e-6)
    other = torch.tensor([1.0, 2.0], device="cuda")
    t = torch.tensor([1.0, float("inf")], device="cuda")
    G = rabit.RabitGradients([t, other])
    assert float(rabit.rabit_clip_gradients(G, 1.0)) == float("inf")
    assert (other == 0).all() and t[0] == 0 and torch.isnan(t[1])
    t.copy_(torch.tensor([1.0, float("nan")]))
    other.fill_(2.0)
    assert torch.isnan(rabit.rabit_clip_gradients(G, 1.0)).all() and torch.isnan(other).all()


def test_clipping_replayed_and_refused():
    import torch
    import paper_2602_05367_b200 as rabit
    src, dst = torch.randn(30000, device="cuda"), torch.zeros(30000, device="cuda")
    norm = torch.zeros(1, device="cuda")
    G = rabit.RabitGradients([src[:10000], src[10000:]], [dst[:10000], dst[10000:]])
    rabit.rabit_clip_gradients(G, 0.5, norm)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        rabit.rabit_clip_gradients(G, 0.5, norm)
    for _ in range(3):
        src.copy_(torch.randn(30000, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        (want,), n = ao.clip([src.cpu().numpy()], 0.5)
        assert abs(float(norm) - n) <= 2.0 ** -23 * n and (np.abs(dst.cpu().numpy() - want) <= 2.0 ** -22 * np.abs(want)).all()
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(rabit.RabitError):
            rabit.rabit_clip_gradients(G, bad)
    for args in (([],), ([src.half()],), ([src.cpu()],), ([src[::2]],), ([src], [dst[:5]])):
        with pytest.raises(ValueError):
            rabit.RabitGradients(*args)
    with pytest.raises(rabit.RabitError):
        rabit.RabitGradients([src, src[5:]])
    for inside in (src[5:6], dst[-1:], G.dev_buf[:4].view(torch.float32)):
        with pytest.raises(rabit.RabitError, match="norm_out"):
            rabit.rabit_clip_gradients(G, 1.0, inside)
    G.free()
    with pytest.raises(rabit.RabitError):
        rabit.rabit_clip_gradients(G, 1.0)


def test_gradients_are_not_bound_under_capture():
    """A captured copy of the table would be repeated from host memory that is gone."""
    import torch
    import paper_2602_05367_b200 as rabit
    t, s, graph = torch.ones(64, device="cuda"), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        t.mul_(2.0)
        with pytest.raises(rabit.RabitError, match="captured"):
            rabit.RabitGradients([t])
    graph.replay()
    torch.cuda.synchronize()
    assert bool((t == 2.0).all())



def test_a_training_step_of_a_group_as_it_is_used():
    """Forward of two projections, backward through the transposed layers, all factor gradients, clipping; the loss is linear in the second factors,
    so moving them changes it by exactly what the gradient says, up to the roundings of y."""
    import torch
    import paper_2602_05367_b200 as rabit
    N, batch, n, r = 256, 90, 2, 8
    rng = np.random.default_rng(13)
    x, ids = make_x(batch, N, key=(101,)), _ids(batch, n, "prompts")
    xd, idd = _cuda(x, ids)
    Ls = [make_layer(M, N, 2, key=(101, M)) for M in (128, 64)]
    pools = [_pool(L.M, N, n, r, 20 + i) for i, L in enumerate(Ls)]
    dys = [(0.1 * rng.standard_normal((batch, L.M))).astype(np.float16) for L in Ls]
    layers = [rabit.rabit_pack(L.planes, L.g, L.h) for L in Ls]
    turned = [rabit.rabit_transpose(v) for v in layers]
    As = [_adapters(*p) for p in pools]
    ys = [torch.empty((batch, L.M), dtype=torch.float16, device="cuda") for L in Ls]
    us = [torch.empty((batch, r), dtype=torch.float32, device="cuda") for _ in Ls]
    ps = [torch.empty_like(u) for u in us]
    grads = [torch.zeros(t.shape, dtype=torch.float32, device="cuda") for A in As for t in (A.a, A.b)]
    G = rabit.RabitGradients(grads)
    rabit.rabit_linear_group_adapted(layers, As, [xd, xd], idd, ys, us)
    dxs = []
    for i, A in enumerate(As):
        dyd, = _cuda(dys[i])
        dxs.append(rabit.rabit_linear_adapted(turned[i], A.transposed(), dyd, idd, u=ps[i]))
        rabit.rabit_adapter_gradients(A, xd, us[i], dyd, ps[i], idd, grads[2 * i], grads[2 * i + 1])
    raw = [g.cpu().numpy() for g in grads]
    norm = rabit.rabit_clip_gradients(G, 0.5)
    torch.cuda.synchronize()
    for i, (L, (a, b, scale)) in enumerate(zip(Ls, pools)):
        W = orc.dense_weight(L.planes, L.g, L.h)
        planes_t = _transposed_planes(L)
        want_dx, want_p, err_dx, err_p = ao.adapted(planes_t, L.h, L.g, b, a, scale, dys[i], ids)
        want_y, want_u, err_y, err_u = ao.adapted(L.planes, L.g, L.h, a, b, scale, x, ids)
        assert np.allclose(dys[i].astype(np.float64) @ W, orc.linear(planes_t, L.h, L.g, dys[i]))
        _within(dxs[i].cpu().numpy(), want_dx, err_dx, "dx")
        _within(ps[i].cpu().numpy(), want_p, err_p, "p")
        _within(ys[i].cpu().numpy(), want_y, err_y, "y")
        # the gradients' inputs are the device's own u and p
        _within(raw[2 * i], *ao.gradients(scale, x, ps[i].cpu().numpy(), ids, n), "da")
        _within(raw[2 * i + 1], *ao.gradients(scale, dys[i], us[i].cpu().numpy(), ids, n), "db")
        # differences, along the gradient's signs
        want_db, err_db = ao.gradients(scale, dys[i], us[i].cpu().numpy(), ids, n)
        move = (0.25 * np.sign(want_db)).astype(np.float16)
        b2 = (b + move).astype(np.float16)
        y2 = rabit.rabit_linear_adapted(layers[i], _adapters(a, b2, scale), xd, idd)
        change = (dys[i].astype(np.float64) * (y2.cpu().numpy().astype(np.float64) - ys[i].cpu().numpy().astype(np.float64))).sum()
        said = (raw[2 * i + 1].astype(np.float64) * (b2.astype(np.float64) - b.astype(np.float64))).sum()
        _, _, err_y2, _ = ao.adapted(L.planes, L.g, L.h, a, b2, scale, x, ids)
        bound = (np.abs(dys[i].astype(np.float64)) * (err_y + err_y2)).sum() + (err_db * np.abs(b2.astype(np.float64) - b)).sum()
        assert abs(change - said) <= bound < 0.1 * said
    want, want_norm = ao.clip(raw, 0.5)
    assert want_norm > 0.5 and abs(float(norm) - want_norm) <= 2.0 ** -23 * want_norm
    for g, w in zip(grads, want):
        assert (np.abs(g.cpu().numpy() - w) <= 2.0 ** -22 * np.abs(w) + 2.0 ** -149).all()
    for v in layers + turned:
        v.free()
