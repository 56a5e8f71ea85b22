"""A beam search's selection and reordering without a GPU: sizes of the passes and the workspace
(csrc/beam_plan.h evaluated through wici_beam_workspace), what the entry points refuse before any GPU
call, and the oracle on cases that can be told by hand."""

from __future__ import annotations

import ctypes

import numpy as np

import oracle
from paper_2608_24204_amd import binding

FAKE = 1 << 20   # an aligned address that no refused call may touch
ARG = binding.WICI_E_ARG


def need(n, beams, vocab, dtype, k):
    size = ctypes.c_size_t()
    st = binding.load_library().wici_beam_workspace(n, beams, vocab, dtype, k, ctypes.byref(size))
    return size.value if st == 0 else st


def test_workspaces():
    for dtype, block in ((binding.WICI_F32, 4), (binding.WICI_BF16, 8)):
        for vocab in (1, 255, 256, 4096, 152064, 262144, 300000, 1 << 24):
            for rows, k in ((1, 1), (12, 8), (65535, 64)):
                loads = -(-(-(-(vocab + 2 * (block - 1) - (block - 1)) // block)) // 64)
                loads = -(-((vocab + 2 * (block - 1)) // block) // 64)
                per = 1
                while -(-loads // per) > 1024:
                    per *= 2
                groups, units = -(-loads // per), -(-loads // max(per, 2))
                assert groups <= 1024 and units <= groups
                want = sum(-(-x // 16) * 16 for x in (8 * rows * units, 8 * rows, 4 * rows * units,
                                                      4 * rows * groups, 4 * rows, 4 * rows * k, 4 * rows * k))
                assert need(rows, 1, vocab, dtype, k) == want
    assert need(0, 4, 100, binding.WICI_F32, 4) == 0
    for bad in ((-1, 4, 100, 0, 4), (1, 0, 100, 0, 4), (1, 65, 100, 0, 4), (1, 4, 0, 0, 4), (1, 4, (1 << 24) + 1, 0, 4),
                (1, 4, 100, 0, 0), (1, 4, 100, 0, 65), (1, 4, 100, 2, 4), (32768, 2, 100, 0, 4), (2 ** 31 - 1, 64, 100, 0, 4)):
        assert need(*bad) == ARG, bad


def test_select_refusals():
    lib = binding.load_library()
    size = need(3, 4, 100, 0, 5)

    def call(logits=FAKE, dtype=0, stride=100, n=3, beams=4, vocab=100, scores=FAKE, k=5, os=FAKE, op=FAKE, ot=FAKE,
             ws=FAKE, bytes_=size):
        return lib.wici_beam_select(logits, dtype, stride, n, beams, vocab, scores, k, os, op, ot, ws, bytes_, None)

    for kw in (dict(logits=None), dict(logits=FAKE + 2), dict(dtype=1, logits=FAKE + 1), dict(dtype=3), dict(stride=99),
               dict(stride=0), dict(stride=-100), dict(stride=(1 << 40) + 1), dict(beams=0), dict(beams=65), dict(vocab=0),
               dict(scores=None), dict(scores=FAKE + 2), dict(k=0), dict(k=65), dict(os=None), dict(op=None),
               dict(ot=FAKE + 1), dict(ws=None), dict(ws=FAKE + 8), dict(bytes_=size - 1), dict(n=-1), dict(n=20000)):
        assert call(**kw) == ARG, kw
    assert call(n=0, logits=None, scores=None, ws=None, bytes_=0) == 0


def test_reorder_refusals():
    lib = binding.load_library()

    def call(bits=4, pools=(FAKE, FAKE), n_pools=None, n=2, beams=3, parent=FAKE, length=FAKE, table=FAKE, spare=FAKE, **kw):
        c = binding.WiciKv8(None, 10, 64, 2, 128, None, 5, 5)
        for k, v in kw.items():
            setattr(c, k, v)
        arr = (ctypes.c_void_p * max(len(pools), 1))(*pools)
        return lib.wici_beam_reorder(c, bits, arr, len(pools) if n_pools is None else n_pools, n, beams, parent, length,
                                     table, spare, None)

    for kw in (dict(bits=16), dict(pools=(FAKE, None)), dict(pools=(FAKE + 8,)), dict(n_pools=-1), dict(n=-1),
               dict(beams=0), dict(beams=65), dict(n=30000), dict(parent=None), dict(length=FAKE + 2), dict(table=None),
               dict(spare=None), dict(page=48), dict(head_dim=96), dict(max_pages=0), dict(max_pages=6),
               dict(table_stride=-5, n=1, beams=1), dict(n_pages=0)):
        assert call(**kw) == ARG, kw
    assert lib.wici_beam_reorder(None, 4, None, 0, 1, 1, FAKE, FAKE, FAKE, FAKE, None) == ARG
    assert call(n=0, parent=None, table=None) == 0


def test_the_oracle_selects():
    z = np.log(np.array([[0.5, 0.25, 0.25], [0.1, 0.9, 0.0 + 1e-300]]))
    s, p, v = oracle.beam_select(z, [0.0, np.log(0.5)], 4)
    assert p.tolist() == [0, 1, 0, 0] and v.tolist() == [0, 1, 1, 2]
    assert np.allclose(np.exp(s), [0.5, 0.45, 0.25, 0.25])
    s, p, v = oracle.beam_select(z, [-np.inf, 0.0], 4)
    assert p.tolist() == [1, 1, 1, -1] and v.tolist() == [1, 0, 2, -1] and s[3] == -np.inf
    assert np.isnan(oracle.beam_select(np.full((1, 3), np.inf), [0.0], 2)[0]).all()


def test_the_oracle_reorders():
    pool = np.arange(8)[:, None].repeat(4, 1)
    table, spare = np.array([[0, 1], [0, 2], [3, 4]]), np.array([5, 6, 7])
    oracle.beam_reorder([pool], table, np.array([[1, 0, 1]]), np.array([6, 6, 6]), spare, 4)
    assert table.tolist() == [[0, 5], [0, 6], [0, 7]] and spare.tolist() == [1, 2, 4]
    assert pool[:, 0].tolist() == [0, 1, 2, 3, 4, 2, 1, 2]
