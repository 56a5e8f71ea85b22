"""The operators on torch tensors beside forward-mode differentiation: a tensor with a tangent is refused as
one that requires a gradient is, and a transform's tensor is not taken for its values."""

from __future__ import annotations

import pytest

from tests.test_gpu_kv8 import Batch, ints, ops, rnd, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def test_tensors_with_a_tangent_are_refused(ops):
    import torch.autograd.forward_ad as fwd
    bt = Batch(ops, [5, 6], n_kv=2, hd=64, page=16)
    bt.fill()
    k, q = (rnd(bt.rng, 2, h, 64, dtype=torch.float32) for h in (2, 4))
    t, pos = ops.rope_table(8, 64), ints([0, 1])
    logits, scores = torch.zeros(4, 9, device="cuda"), torch.zeros(2, 2, device="cuda")
    before = bt.cache.pool.clone()
    for grad in (torch.enable_grad, torch.no_grad):
        with fwd.dual_level(), grad():
            def dual(x):
                return fwd.make_dual(x.clone(), torch.ones_like(x))
            tg = ops.RopeTable(dual(t.cos), t.sin)
            for call in (lambda: ops.rope(dual(q), pos, t), lambda: ops.rope(q, pos, tg),
                         lambda: ops.rope(q, pos, t, out=dual(q)), lambda: ops.rope(2 * dual(q), pos, t),
                         lambda: bt.cache.append(dual(k), k, bt.length), lambda: bt.cache.append(k, dual(k), bt.length),
                         lambda: bt.cache.append(k, k, bt.length, rope=t, q=dual(q)),
                         lambda: bt.cache.append(k, k, bt.length, rope=t, q=q, q_out=dual(q)),
                         lambda: bt.cache.append(k, k, bt.length, rope=tg),
                         lambda: bt.cache.read(bt.length, k=dual(k)), lambda: bt.cache.read(bt.length, v=dual(k)),
                         lambda: bt.cache.attend(dual(q), bt.length), lambda: bt.cache.attend(q, bt.length, out=dual(q)),
                         lambda: ops.beam_select(dual(logits), scores), lambda: ops.beam_select(logits, dual(scores))):
                with pytest.raises(RuntimeError, match="gradient"):
                    call()
            assert torch.equal(bt.cache.pool, before)
            # tensors without one, and the values alone
            want = bt.cache.attend(q, bt.length)
            assert torch.equal(bt.cache.attend(fwd.unpack_dual(dual(q)).primal, bt.length), want)
            assert torch.equal(bt.cache.attend(dual(q).detach(), bt.length), want)
            assert torch.equal(ops.beam_select(dual(logits).detach(), scores)[1], ops.beam_select(logits, scores)[1])


def test_transforms_are_refused(ops):
    bt = Batch(ops, [5, 6], n_kv=2, hd=64, page=16)
    bt.fill()
    q = rnd(bt.rng, 2, 4, 64, dtype=torch.float32)
    logits, scores = torch.zeros(4, 9, device="cuda"), torch.zeros(2, 2, device="cuda")
    for f, x in ((lambda x: bt.cache.attend(x, bt.length), q), (lambda x: ops.rope(x, bt.length, ops.rope_table(8, 64)), q),
                 (lambda x: ops.beam_select(x, scores)[0], logits)):
        for call in (lambda: torch.func.jvp(f, (x,), (torch.ones_like(x),)), lambda: torch.func.vjp(f, x),
                     lambda: torch.func.grad(lambda y: f(y).sum())(x), lambda: torch.func.vmap(f)(x[None])):
            with pytest.raises(RuntimeError):
                call()
