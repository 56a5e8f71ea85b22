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


def test_a_write_into_a_saved_tensor_is_noticed(ops):
    """A tensor that autograd keeps for a backward pass and that a call then writes: that pass is an
    error, as after any operation in place, and not a gradient of other values."""
    bt = Batch(ops, [5, 6], n_kv=2, hd=64, page=16)
    bt.fill()
    k, q = (rnd(bt.rng, 2, h, 64, dtype=torch.float32) for h in (2, 4))
    t, pos = ops.rope_table(8, 64), ints([0, 1])
    side = torch.cuda.Stream()
    for stream in (None, side):
        side.wait_stream(torch.cuda.current_stream())
        kw = {} if stream is None else dict(stream=stream)
        for like, write in (
                (q, lambda x: ops.rope(q, pos, t, out=x, **kw)), (q, lambda x: ops.rope(x, pos, t, out=x, **kw)),
                (q, lambda x: bt.cache.append(k, k, bt.length, rope=t, q=q, q_out=x, **kw)),
                (q, lambda x: bt.cache.attend(q, bt.length, out=x, **kw)),
                (k, lambda x: bt.cache.read(bt.length, k=x, **kw)),
                (k, lambda x: bt.cache.read(bt.length, v=x, **kw))):
            x, w = like.clone(), torch.ones_like(like, requires_grad=True)
            y = (x * w).sum()
            write(x)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                y.backward()
        # the pool, and tensors that are only read
        version, read = bt.cache.pool._version, q._version
        bt.cache.attend(q, bt.length, **kw), bt.cache.read(bt.length, **kw)
        assert bt.cache.pool._version == version
        bt.cache.append(k, k, bt.length, rope=t, q=q, **kw)
        assert bt.cache.pool._version > version and q._version == read
    torch.cuda.synchronize()
