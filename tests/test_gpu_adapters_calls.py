"""Calls of the adapters, their gradients and the clipping that a program can make beside the ordinary ones."""
import numpy as np
import pytest

from oracle import adapters_oracle as ao
from tests.test_gpu_adapters import _adapters, _cuda, _pool, _within

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
