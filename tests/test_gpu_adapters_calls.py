"""Calls of the adapters, their gradients and the clipping that a program can make beside the ordinary ones."""
import numpy as np
import pytest

from oracle import adapters_oracle as ao
from synth import make_layer, make_x
from tests.test_gpu_adapters import _adapters, _cuda, _ids, _pool, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,r", [(3, 4), (200, 16), (1500, 40), (300, 100)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_slot_that_no_row_names_may_hold_any_scale(batch, r, bad):
    """Its gradient is zero, or what was there before, and the norm over all gradients is that of the others."""
    import torch
    import paper_2602_05367_b200 as rabit
    M, N, n = 96, 160, 4
    rng = np.random.default_rng([30, batch, r])
    a, b, scale = _pool(M, N, n, r, 40)
    x, dy = rng.standard_normal((batch, N)).astype(np.float16), (0.1 * rng.standard_normal((batch, M))).astype(np.float16)
    u, p = rng.standard_normal((batch, r)).astype(np.float32), (0.1 * rng.standard_normal((batch, r))).astype(np.float32)
    ids = rng.choice(np.array([-1, 0, 2], np.int32), batch).astype(np.int32)
    ids[0] = 0
    want = ao.gradients(scale, x, p, ids, n), ao.gradients(scale, dy, u, ids, n)
    scale[1] = scale[3] = bad                                                           # named by no row
    A, args = _adapters(a, b, scale), _cuda(x, u, dy, p, ids)
    da, db = rabit.rabit_adapter_gradients(A, *args)
    for got, (w, err) in zip((da, db), want):
        _within(got.cpu().numpy(), w, err, "gradient")
        assert (got[1] == 0).all() and (got[3] == 0).all()
    before = [torch.randn(t.shape, device="cuda") for t in (da, db)]
    more = [t.clone() for t in before]
    rabit.rabit_adapter_gradients(A, *args, *more, accumulate=True)
    for got, old in zip(more, before):
        assert torch.equal(got[1], old[1]) and torch.equal(got[3], old[3]) and bool(torch.isfinite(got).all())
    raw = [t.cpu().numpy() for t in (da, db)]
    norm = rabit.rabit_clip_gradients(rabit.RabitGradients([da, db]), 0.5)
    clipped, want_norm = ao.clip(raw, 0.5)
    assert abs(float(norm) - want_norm) <= 2.0 ** -23 * want_norm
    for got, w in zip((da, db), clipped):
        assert (np.abs(got.cpu().numpy() - w) <= 2.0 ** -22 * np.abs(w) + 2.0 ** -149).all()


def _beside(stream, body):
    """`body` enqueued while `stream` has work to do: 50 ms of it, more if the host was not done by then.  body(wait) enqueues wait() on the stream first and returns the
    checks of what it did."""
    import torch
    for cycles in (100_000_000, 400_000_000, 1_600_000_000):
        def wait():
            with torch.cuda.stream(stream):
                torch.cuda._sleep(cycles)
        check = body(wait)
        beside = not stream.query()
        torch.cuda.synchronize()
        check()
        if beside:
            return
    pytest.skip("the host took longer than the stream's work")


@pytest.mark.parametrize("batch", [3, 40, 300])
@pytest.mark.parametrize("call", ["linear", "u", "y", "group u", "gradients", "norm"])
def test_memory_that_a_call_makes_for_another_stream_is_not_in_use(call, batch):
    """Blocks that were just dropped, but that torch's stream has still to read: a call on another stream must not be given them."""
    import torch
    import paper_2602_05367_b200 as rabit
    M, N, n, r = 2048, 1024, 2, 16
    L = make_layer(M, N, 2, key=(111,))
    a, b, scale = _pool(M, N, n, r, 60)
    layer, A = rabit.rabit_pack(L.planes, L.g, L.h), _adapters(a, b, scale)
    rng = np.random.default_rng(61)
    x, ids = make_x(batch, N, key=(111, batch)), np.zeros(batch, np.int32)
    dy, p = rng.standard_normal((batch, M)).astype(np.float16), rng.standard_normal((batch, r)).astype(np.float32)
    xd, idd, dyd, pd = _cuda(x, ids, dy, p)
    y, u = torch.empty((batch, M), dtype=torch.float16, device="cuda"), torch.empty((batch, r), device="cuda")
    want_plain = rabit.rabit_linear(layer, xd)
    want_y = rabit.rabit_linear_adapted(layer, A, xd, idd, None, u)
    want_da, want_db = rabit.rabit_adapter_gradients(A, xd, u, dyd, pd, idd)
    shape, dtype = {"linear": (want_plain.shape, torch.float16), "y": (want_plain.shape, torch.float16), "gradients": (want_da.shape, torch.float32),
                    "norm": ((1,), torch.float32)}.get(call, ((batch, r), torch.float32))
    G = rabit.RabitGradients([torch.full((100,), 3.0, device="cuda")])
    torch.cuda.synchronize()
    here, there = torch.cuda.current_stream(), torch.cuda.Stream()

    def body(wait):
        blocks = [torch.full(shape, 7.0, dtype=dtype, device="cuda") for _ in range(24)]
        kept = torch.zeros((24,) + tuple(shape), dtype=dtype, device="cuda")
        torch.cuda.synchronize()
        wait()
        for i, block in enumerate(blocks):
            kept[i].copy_(block)
        del blocks, block
        s = there.cuda_stream
        if call == "linear":
            got, want = [rabit.rabit_linear(layer, xd, stream=s)], [want_plain]
        elif call == "u":
            got, want = [rabit.rabit_linear_adapted(layer, A, xd, idd, y, None, s)], [want_y]
        elif call == "y":
            got, want = [rabit.rabit_linear_adapted(layer, A, xd, idd, None, u, s)], [want_y]
        elif call == "group u":
            got, want = rabit.rabit_linear_group_adapted([layer], [A], [xd], idd, [y], None, s), [want_y]
        elif call == "gradients":
            got, want = rabit.rabit_adapter_gradients(A, xd, u, dyd, pd, idd, stream=s), [want_da, want_db]
        else:
            got, want = [rabit.rabit_clip_gradients(G, 1e3, stream=s)], [torch.full((1,), 30.0, device="cuda")]
        there.synchronize()

        def check():
            assert bool((kept == 7.0).all())
            assert all(torch.equal(v, w) for v, w in zip(got, want))
        return check

    _beside(here, body)
    layer.free()


@pytest.mark.parametrize("in_place", [True, False])
def test_what_a_clipping_on_another_stream_needs_outlives_its_owners(in_place):
    """The norm is not looked at, the RabitGradients is freed at once, and their memory is asked for again before the stream has come so far."""
    import torch
    import paper_2602_05367_b200 as rabit
    there = torch.cuda.Stream()

    def body(wait):
        t, hold = torch.full((10000,), 2.0, device="cuda"), torch.full((10000,), 2.0, device="cuda")
        G = rabit.RabitGradients([t], None if in_place else [hold])
        torch.cuda.synchronize()
        wait()
        rabit.rabit_clip_gradients(G, 1.0, stream=there.cuda_stream)
        size = G.dev_buf.numel()
        G.free()
        others = [torch.full((size,), 0, dtype=torch.uint8, device="cuda") for _ in range(8)] + [torch.full((1,), 5.0, device="cuda") for _ in range(8)]
        torch.cuda.current_stream().synchronize()

        def check():
            assert all(bool((v == v.flatten()[0]).all()) and float(v.flatten()[0]) in (0.0, 5.0) for v in others)
            assert float(((t if in_place else hold) - 0.01).abs().max()) < 1e-8 and (in_place or bool((t == 2.0).all()))
        return check

    _beside(there, body)


def test_a_layer_made_on_another_stream_is_not_in_memory_in_use():
    import torch
    import paper_2602_05367_b200 as rabit
    L = make_layer(256, 512, 2, key=(112,))
    image = rabit.pack_host(L.planes, L.g, L.h)
    layer = rabit.rabit_pack(L.planes, L.g, L.h)
    turned = rabit.rabit_transpose(layer)
    want = turned.dev_buf.clone()
    here, there = torch.cuda.current_stream(), torch.cuda.Stream()

    def body(wait):
        blocks = [torch.full((v.numel(),), 7, dtype=torch.uint8, device="cuda") for v in 12 * [layer.dev_buf, turned.dev_buf]]
        kept = [torch.zeros_like(v) for v in blocks]
        torch.cuda.synchronize()
        wait()
        for k, block in zip(kept, blocks):
            k.copy_(block)
        del blocks, block
        made = rabit.rabit_pack(L.planes, L.g, L.h, stream=there.cuda_stream), rabit.rabit_transpose(layer, stream=there.cuda_stream)
        there.synchronize()

        def check():
            assert all(bool((k == 7).all()) for k in kept)
            assert np.array_equal(made[0].dev_buf.cpu().numpy(), image) and torch.equal(made[1].dev_buf, want)
            for v in made:
                v.free()
        return check

    _beside(here, body)
    layer.free()
    turned.free()


@pytest.mark.parametrize("variant,batch,M", [(2, 70, 520), (2, 1100, 1031), (6, 300, 520)])
def test_what_the_layer_refuses_leaves_y_and_u_as_they_were(variant, batch, M):
    """A kernel family that cannot run the batch: nothing of the call has run, in a group nothing of the layers before it either."""
    import torch
    import paper_2602_05367_b200 as rabit
    N, n, r = 64, 3, 8
    Ls = [make_layer(M, N, 2, key=(110, M, i)) for i in range(2)]
    layers, pools = [rabit.rabit_pack(L.planes, L.g, L.h) for L in Ls], [_adapters(*_pool(M, N, n, r, 50 + i)) for i in range(2)]
    xd, idd = _cuda(make_x(batch, N, key=(110, batch)), np.zeros(batch, np.int32))
    ys = [torch.full((batch, M), 7.0, dtype=torch.float16, device="cuda") for _ in range(2)]
    us = [torch.full((batch, r), 7.0, device="cuda") for _ in range(2)]
    layers[1].set_variant(variant)
    refused = variant == 2                                                              # (6 takes the GEMM here: the same call answered)
    for call in (lambda: rabit.rabit_linear_adapted(layers[1], pools[1], xd, idd, ys[1], us[1]), lambda: rabit.rabit_linear_group_adapted(layers, pools, [xd, xd], idd, ys, us)):
        if refused:
            with pytest.raises(rabit.RabitError, match="cannot run"):
                call()
        else:
            call()
        torch.cuda.synchronize()
        assert not refused or all(bool((t == 7.0).all()) for t in ys + us)
    if not refused:
        assert not any(bool((t == 7.0).all()) for t in ys + us)
    for layer in layers:
        layer.free()


@pytest.mark.parametrize("variant,batch,M,N,r,kind", [
    (0, 2, 509, 512, 5, "one"), (0, 6, 509, 512, 33, "mixed"), (0, 12, 509, 512, 5, "mixed"), (0, 16, 509, 512, 33, "prompts"), (0, 48, 509, 512, 33, "mixed"), (0, 200, 509, 512, 5, "prompts"),
    (0, 200, 4099, 4128, 5, "mixed"), (0, 200, 4099, 4128, 33, "prompts"), (0, 300, 4099, 4128, 33, "prompts"), (0, 300, 4099, 4128, 21, "mixed"), (0, 1100, 509, 512, 5, "mixed"), (0, 1100, 509, 512, 33, "prompts"),
    (0, 1100, 509, 512, 3, "none"), (1, 1100, 509, 512, 5, "mixed"), (5, 1100, 512, 512, 16, "prompts"), (5, 1100, 509, 512, 33, "mixed"), (4, 1100, 509, 512, 100, "mixed")])
def test_a_chain_of_calls_with_odd_outputs_and_ranks(variant, batch, M, N, r, kind):
    """As the chains of square layers, in both forms, behind every kind of layer kernel: y of one call lies in the memory that the next one reads as x, u is shared, ids and
    factors change by copies on the stream.  Rows of y lie on no 16-byte boundary, u is read by single values."""
    import torch
    import paper_2602_05367_b200 as rabit
    n, steps = 3, 6
    L = make_layer(M, N, 2, key=(113, M))
    layer = rabit.rabit_pack(L.planes, (L.g.astype(np.float32) / (16 * np.sqrt(N / 512))).astype(np.float16), L.h)
    if variant:
        layer.set_variant(variant)
    (x0,) = _cuda(make_x(batch, N, key=(113, batch)))
    pools = [_cuda(*_pool(M, N, n, r, 70 + k)) for k in range(2)]
    ids = [_cuda(_ids(batch, n, kind, k))[0] for k in range(2)]
    s, outs = torch.cuda.Stream(), {}
    torch.cuda.synchronize()
    for stop in (True, False):
        A, at = rabit.RabitAdapters(*[t.clone() for t in pools[0]]), ids[0].clone()
        bufs = [x0.clone()] + [torch.zeros((batch, N), dtype=torch.float16, device="cuda") for _ in range(steps)]
        u, us = torch.zeros((batch, r), device="cuda"), [torch.zeros((batch, r), device="cuda") for _ in range(steps)]
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for k in range(steps):
                if k == 3:                                                              # calls 0-2 and 3-5 follow one another without anything between but the calls
                    at.copy_(ids[1])
                    for t, v in zip((A.a, A.b, A.scale), pools[1]):
                        t.copy_(v)
                rabit.rabit_linear_adapted(layer, A, bufs[k], at, bufs[k + 1].view(-1)[:batch * M].view(batch, M), u if k % 3 != 2 else us[k])
                if stop:
                    s.synchronize()
        torch.cuda.synchronize()
        outs[stop] = [t.cpu().numpy() for t in bufs + us + [u]]
    assert all(np.isfinite(v).all() for v in outs[True][:steps + 1]) and (outs[True][1] != 0).any()
    for k, (v, w) in enumerate(zip(outs[True], outs[False])):
        assert np.array_equal(v, w), k
    layer.free()


@pytest.mark.parametrize("r", [1, 17, 40, 128])
def test_small_low_rank_products_beside_large_ones(r):
    """The second fp16 part has steps of 2^-24 where the largest entry of the rank is scaled to 2^14: an entry is off by at most 2^-39 of the largest, and by that
    much at a tie, which goes to the even neighbour 0."""
    import torch
    import paper_2602_05367_b200 as rabit
    M, N, batch = 32, 64, 5
    a, b, _ = _pool(M, N, 1, r, 80)
    x, p = np.zeros((batch, N), np.float16), np.zeros((batch, r), np.float32)
    p[0] = 1.0                                                                          # the largest, where x is zero
    entries = np.array([2.0 ** -39, 1.5 * 2.0 ** -39, 2.0 ** -38, 2.0 ** -20 + 2.0 ** -39], np.float32)
    p[1:] = entries[:, None]
    x[np.arange(1, 5), np.arange(4)] = 1.0
    da, _ = rabit.rabit_adapter_gradients(_adapters(a, b, np.ones(1, np.float32)), *_cuda(x, p, np.zeros((batch, M), np.float16), p, np.zeros(batch, np.int32)))
    got = da[0, :, :4].cpu().numpy().astype(np.float64)
    assert (np.abs(got - entries) <= 2.0 ** -39).all()
    assert (got[:, 0] == 0).all() and (got[:, 1] == 2.0 ** -38).all() and (got[:, 2] == 2.0 ** -38).all() and not da[0, :, 4:].any()


@pytest.mark.parametrize("batch,M,r", [(1, 64, 3), (5, 64, 16), (12, 67, 4), (100, 64, 40), (1100, 1024, 16)])
def test_a_layer_sum_beyond_fp16_is_infinite_whatever_the_adapter_adds(batch, M, r):
    """y is the layer's fp16 output plus the adapter's part: rows whose layer sum is 80000 stay infinite although 40000 are taken away.  781.25 is 781 in fp16 (a tie between
    steps of 0.5), 64 of them 49984, exact: plus 12.8 * 781 that is 59980.8, in steps of 32 59968; plus 25.6 * 781 it is infinite."""
    import torch
    import paper_2602_05367_b200 as rabit
    N = 64
    L = make_layer(M, N, 1, key=(114, M))
    L.planes[:], L.g[:], L.h[:] = 0, 1, 1
    a, b = np.zeros((3, r, N), np.float16), np.zeros((3, r, M), np.float16)
    a[:, r - 1, 0], b[:, r - 1] = 1, 1                                                  # u = x[0]
    which = np.arange(batch) % 3
    x = np.full((batch, N), 50000 / 64, np.float16)       
    x[which == 0] = 80000 / 64
    scale = np.array([-40000 / 1250, 10000 / 781.25, 20000 / 781.25], np.float32)
    layer = rabit.rabit_pack(L.planes, L.g, L.h)
    y = rabit.rabit_linear_adapted(layer, _adapters(a, b, scale), *_cuda(x, which.astype(np.int32))).cpu().numpy()
    assert (y[which == 0] == np.inf).all() and (y[which == 1] == 59968).all() and (y[which == 2] == np.inf).all()
    layer.free()


def test_bound_gradients_may_be_clipped_on_any_stream():
    """Binding returns when its table is in place, however long the stream's earlier work takes."""
    import torch
    import paper_2602_05367_b200 as rabit
    s = torch.cuda.Stream()
    t = torch.full((5000,), 2.0, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(100_000_000)                                                  # some 50 ms
    G = rabit.RabitGradients([t], stream=s.cuda_stream)
    assert s.query()
    norm = rabit.rabit_clip_gradients(G, 1.0)
    torch.cuda.synchronize()
    assert abs(float(norm) - 2 * np.sqrt(5000)) < 1e-3 and abs(float(t[0]) - 1 / np.sqrt(5000)) < 1e-6


def test_the_calls_leave_no_autograd_history():
    """As they say: what they return needs no gradient, and nothing is put into .grad."""
    import torch
    import paper_2602_05367_b200 as rabit
    M, N, batch, r = 64, 96, 4, 8
    L = make_layer(M, N, 1, key=(115,))
    a, b, scale = _pool(M, N, 2, r, 90)
    layer, A = rabit.rabit_pack(L.planes, L.g, L.h), _adapters(a, b, scale)
    xd, idd, dyd = _cuda(make_x(batch, N, key=(115, 1)), np.zeros(batch, np.int32), make_x(batch, M, key=(115, 2)))
    for t in (A.a, A.b, A.scale, xd, dyd):
        t.requires_grad_()
    u = torch.empty((batch, r), device="cuda")
    y = rabit.rabit_linear_adapted(layer, A, xd, idd, None, u)
    da, db = rabit.rabit_adapter_gradients(A, xd, u, dyd, u, idd)
    assert not any(t.requires_grad for t in (y, u, da, db)) and all(t.grad is None for t in (A.a, A.b, A.scale, xd, dyd))
    layer.free()


@pytest.mark.parametrize("n_in,n_out", [(1, 7), (5, 3), (8, 2), (9, 15), (257, 1)])
@pytest.mark.parametrize("batch,r", [(1, 1), (3, 5), (70, 16), (300, 33)])
def test_factor_gradients_of_narrow_sides(n_in, n_out, batch, r):
    """Sides below the eight values of a 16-byte piece: the last rows of x and dy end inside the last piece of their buffer."""
    import torch
    import paper_2602_05367_b200 as rabit
    n = 3
    rng = np.random.default_rng([31, n_in, n_out, batch, r])
    a, b, scale = rng.standard_normal((n, r, n_in)).astype(np.float16), rng.standard_normal((n, r, n_out)).astype(np.float16), rng.uniform(0.5, 2.0, n).astype(np.float32)
    x, dy = rng.standard_normal((batch, n_in)).astype(np.float16), rng.standard_normal((batch, n_out)).astype(np.float16)
    u, p = rng.standard_normal((batch, r)).astype(np.float32), rng.standard_normal((batch, r)).astype(np.float32)
    ids = rng.integers(-1, n, batch).astype(np.int32)
    guard = [torch.full((n * r * side + 8,), 3.0, device="cuda") for side in (n_in, n_out)]
    outs = [g[:n * r * side].view(n, r, side) for g, side in zip(guard, (n_in, n_out))]
    rabit.rabit_adapter_gradients(_adapters(a, b, scale), *_cuda(x, u, dy, p, ids), *outs)
    for got, g, v, low in zip(outs, guard, (x, dy), (p, u)):
        _within(got.cpu().numpy(), *ao.gradients(scale, v, low, ids, n), "gradient")
        assert (g[-8:] == 3.0).all()


@pytest.mark.parametrize("batch,r,kind", [(2, 5, "one"), (12, 33, "mixed"), (200, 5, "prompts"), (1100, 33, "mixed")])
def test_a_captured_chain_with_odd_outputs(batch, r, kind):
    """The chain in a graph that is replayed twice without a stop: bit for bit the calls one by one."""
    import torch
    import paper_2602_05367_b200 as rabit
    M, N, n, steps = 509, 512, 3, 4
    L = make_layer(M, N, 2, key=(116,))
    layer, A = rabit.rabit_pack(L.planes, (L.g.astype(np.float32) / 16).astype(np.float16), L.h), _adapters(*_pool(M, N, n, r, 91))
    xd, idd = _cuda(make_x(batch, N, key=(116, batch)), _ids(batch, n, kind))
    bufs = [xd] + [torch.zeros((batch, N), dtype=torch.float16, device="cuda") for _ in range(steps)]
    u, s, graph = torch.zeros((batch, r), device="cuda"), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    out = [t.view(-1)[:batch * M].view(batch, M) for t in bufs]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        for k in range(steps):
            rabit.rabit_linear_adapted(layer, A, bufs[k], idd, out[k + 1], u)
    for rep in range(3):
        xd.copy_(_cuda(make_x(batch, N, key=(116, batch, rep)))[0])
        want = [xd.clone()] + [torch.zeros_like(xd) for _ in range(steps)]
        for k in range(steps):
            rabit.rabit_linear_adapted(layer, A, want[k], idd, want[k + 1].view(-1)[:batch * M].view(batch, M))
            torch.cuda.synchronize()
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(v, w) for v, w in zip(bufs, want))
    layer.free()
