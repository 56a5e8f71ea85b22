"""Models with an 8-bit KV cache (kv_dtype KV8): what their results and their sharing do not depend
on."""

from __future__ import annotations

import numpy as np
import pytest

from paper_2608_24204_amd import inputs, ops
from paper_2608_24204_amd.binding import WiciError, WiciModel
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


def test_models_that_rotate_alike_share_weights(cuda_ok):
    """Whether weights are shared goes by what the rotation is: fields that its scaling ignores, and
    names for defaults, make no difference; another step, factor or order does."""
    cfg = CFGS["bf16_128"]
    w, _ = weights(cfg)
    hd, nan = cfg.head_dim, float("nan")
    bands = dict(base=cfg.rope_base, scaling="bands", factor=4.0, original=64.0)
    prompt = inputs.make_prompt(cfg, 20)
    for rope, alike, others in (
            (None, [ops.rope_spec(hd, cfg.rope_base), ops.rope_spec(hd, cfg.rope_base, factor=nan, low=nan)],
             [ops.rope_spec(hd, cfg.rope_base, layout="pairs"), ops.rope_spec(hd // 2, cfg.rope_base)]),
            (ops.rope_spec(hd, **bands),
             [ops.rope_spec(hd, **bands, low=1.0, high=4.0)],
             [None, ops.rope_spec(hd, **bands, low=1.0, high=5.0),
              ops.rope_spec(hd, **(bands | dict(scaling="ramp")))]),
            (ops.rope_spec(64, cfg.rope_base, scaling="linear", factor=2.0, original=5.0),
             [ops.rope_spec(64, cfg.rope_base, scaling="linear", factor=2.0, high=nan)],
             [ops.rope_spec(64, cfg.rope_base, scaling="linear", factor=3.0)])):
        lead = model(cfg, w, rope=rope)
        try:
            want = lead.generate(prompt, 3)
            for r in alike:
                m = WiciModel(cfg, share_weights_of=lead, rope=r)
                try:
                    assert m.generate(prompt, 3) == want
                finally:
                    m.close()
            for r in others:
                with pytest.raises(WiciError, match="WICI_E_ARG"):
                    WiciModel(cfg, share_weights_of=lead, rope=r)
        finally:
            lead.close()
