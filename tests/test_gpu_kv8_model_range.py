"""Models with an 8-bit KV cache (kv_dtype KV8): what their results and their sharing do not depend
on."""

from __future__ import annotations

import numpy as np
import pytest

from paper_2608_24204_amd import inputs
from tests.test_gpu_kv8_model import CFGS, model, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("chunk", [2048, 100])
@pytest.mark.parametrize("name", ["bf16_128", "bf16_64"])
def test_a_prompt_is_planned_for_itself(cuda_ok, name, chunk):
    """The attention of a prompt is split by its own length and not by the cache's capacity: logits
    are the same bits in a cache that just holds it and in one of 16384 positions."""
    cfg = CFGS[name]
    w, _ = weights(cfg)
    for n in (33, cfg.prompt_len):
        prompt = inputs.make_prompt(cfg, n)
        got = []
        for max_seq in (n, 16384):
            m = model(cfg, w, max_seq=max_seq, prefill_chunk=chunk)
            try:
                got.append(m.prefill(prompt, want_logits=True))
            finally:
                m.close()
        assert got[0][0] == got[1][0] and np.array_equal(got[0][1], got[1][1])
