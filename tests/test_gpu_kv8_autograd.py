"""The operators on torch tensors beside autograd: they have no gradients, and say so."""

from __future__ import annotations

import pytest

from tests.test_gpu_kv8 import Batch, ints, ops, rnd, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def test_tensors_that_require_gradients_are_refused(ops):
    bt = Batch(ops, [5, 6], n_kv=2, hd=64, page=16)
    bt.fill()
    k, q = (rnd(bt.rng, 2, h, 64, dtype=torch.float32) for h in (2, 4))
    kg, qg = k.clone().requires_grad_(), q.clone().requires_grad_()
    t = ops.rope_table(8, 64)
    tg = ops.RopeTable(t.cos.clone().requires_grad_(), t.sin)
    pos = ints([0, 1])
    before = bt.cache.pool.clone()
    for call in (lambda: ops.rope(qg, pos, t), lambda: ops.rope(q, pos, tg),
                 lambda: ops.rope(q, pos, t, out=qg), lambda: ops.rope(2 * qg, pos, t),
                 lambda: bt.cache.append(kg, k, bt.length), lambda: bt.cache.append(k, kg, bt.length),
                 lambda: bt.cache.append(k, k, bt.length, rope=t, q=qg),
                 lambda: bt.cache.append(k, k, bt.length, rope=t, q=q, q_out=qg),
                 lambda: bt.cache.append(k, k, bt.length, rope=tg),
                 lambda: bt.cache.read(bt.length, k=kg), lambda: bt.cache.read(bt.length, v=kg),
                 lambda: bt.cache.attend(qg, bt.length), lambda: bt.cache.attend(q, bt.length, out=qg)):
        with pytest.raises(RuntimeError, match="gradient"):
            call()
    assert torch.equal(bt.cache.pool, before)
    # where none are recorded they are values like others
    with torch.no_grad():
        assert torch.equal(ops.rope(qg, pos, tg), ops.rope(q, pos, t))
        bt.cache.append(kg, kg, bt.length)
        assert not bt.cache.attend(qg, bt.length).requires_grad
    with torch.inference_mode():
        assert torch.equal(bt.cache.attend(qg, bt.length), bt.cache.attend(q, bt.length))
    assert torch.equal(bt.cache.attend(qg.detach(), bt.length), bt.cache.attend(q, bt.length))
