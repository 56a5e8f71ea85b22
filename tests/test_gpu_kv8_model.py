"""The decoder with an 8-bit KV cache (kv_dtype KV8) and with rotary embeddings other than
rope_base's (wici_set_rope), through the C ABI against the float64 oracle: greedy ids
identical at every step, logits within the bounds the other cache types are held to (2e-2
bf16 weights, 1e-4 fp32; the oracle quantises its own rows, and where a row's value lies next
to the border of two codes the two sides may differ by one step of 1/127 of the row's
largest: fp32 weights are held to 2e-3, a few such steps among some hundred positions)."""

from __future__ import annotations

import ctypes

import numpy as np
import pytest

from oracle import DecoderOracle
from paper_2608_24204_amd import binding, configs, inputs, ops
from paper_2608_24204_amd.binding import WiciError
from tests.helpers import inf_rel
from tests.parity import compare, oracle_run

pytestmark = pytest.mark.gpu

BASE = dict(n_layers=2, d_model=512, n_heads=8, n_kv_heads=2, head_dim=128, ffn_dim=1024, vocab=2003,
            prompt_len=150, decode_steps=12, rope_base=500000.0, kv_dtype="kv8")
CFGS = {
    "bf16_128": configs.ModelConfig(name="t_kv8", key=140, **BASE),
    "bf16_64": configs.ModelConfig(name="t_kv8_64", key=141, **(BASE | dict(
        head_dim=64, n_heads=10, n_kv_heads=2, prompt_len=333))),
    "q8": configs.ModelConfig(name="t_kv8_q8", key=142, weight_dtype="q8", **BASE),
    "f32": configs.ModelConfig(name="t_kv8_f32", key=143, weight_dtype="f32", **(BASE | dict(
        d_model=256, n_heads=4, n_kv_heads=4, head_dim=64, ffn_dim=512, prompt_len=40))),
}
TOL = {"f32": 2e-3}
ROPES = {
    "pairs": dict(dim=128, layout="pairs", base=10000.0),
    "part": dict(dim=40, layout="half", base=10000.0, scaling="linear", factor=4.0),
    "pairs_part_bands": dict(dim=64, layout="pairs", base=500000.0, scaling="bands", factor=8.0,
                             original=64.0),
    "ramp": dict(dim=128, layout="half", base=10000.0, scaling="ramp", factor=4.0, original=50.0),
}


def weights(cfg):
    w = inputs.make_weights(cfg, gain_std=0.1)
    if cfg.weight_dtype == "q8":
        from oracle import q8_model_f64
        return w, q8_model_f64(w)
    return w, inputs.weights_f64(cfg, w)


def model(cfg, w, **kw):
    from paper_2608_24204_amd.binding import WiciModel
    m = WiciModel(cfg, **kw)
    m.load_weights(w)
    return m


@pytest.mark.parametrize("name", list(CFGS))
@pytest.mark.parametrize("page,chunk,graph", [(16, 2048, True), (64, 64, True), (128, 7, False)])
def test_greedy_run_matches_the_oracle(cuda_ok, name, page, chunk, graph):
    cfg = CFGS[name]
    w, w64 = weights(cfg)
    prompt = inputs.make_prompt(cfg)
    ids, logs = oracle_run(cfg, w64, prompt, cfg.decode_steps)
    m = model(cfg, w, kv_page=page, prefill_chunk=chunk, graph=graph)
    try:
        got, glogs = m.generate(prompt, cfg.decode_steps, want_logits=True)
        rep = compare(got, glogs, ids, logs)
        assert rep.strict_ids and rep.max_rel_err <= TOL.get(name, 2e-2), rep.summary()
        # the same tokens from one call, and a second sequence in the same cache
        m.reset_kv()
        first, _ = m.prefill(prompt)
        more, _ = m.decode_n(cfg.decode_steps)
        assert [first] + list(more) == got
    finally:
        m.close()


@pytest.mark.parametrize("name", ["bf16_128", "f32"])
def test_the_cache_holds_the_oracles_rows(cuda_ok, name):
    cfg = CFGS[name]
    w, w64 = weights(cfg)
    prompt = inputs.make_prompt(cfg)
    orc = DecoderOracle(cfg, w64)
    orc.prefill(prompt)
    m = model(cfg, w, kv_page=32)
    try:
        m.prefill(prompt)
        for layer in range(cfg.n_layers):
            K, V = m.read_kv(layer, 3, len(prompt))
            assert K.dtype == np.float32
            for got, want in ((K, orc.K[layer]), (V, orc.V[layer])):
                # one step of a row is 1/127 of its largest value
                assert inf_rel(got, want[3:len(prompt)]) <= 1.02 / 127 + 2e-3
                assert np.mean(np.abs(got - want[3:len(prompt)]) > 1e-2 * np.abs(want).max()) == 0
    finally:
        m.close()


@pytest.mark.parametrize("kv", ["kv8", "bf16"])
@pytest.mark.parametrize("rope", list(ROPES))
def test_other_rotary_embeddings(cuda_ok, kv, rope):
    cfg = CFGS["bf16_128"].with_(kv_dtype=kv)
    w, w64 = weights(cfg)
    prompt = inputs.make_prompt(cfg)
    orc = DecoderOracle(cfg, w64, rope=ROPES[rope], max_seq=cfg.max_seq)
    ids, logs = orc.generate(prompt, cfg.decode_steps)
    m = model(cfg, w, rope=ops.rope_spec(**ROPES[rope]), kv_page=16, prefill_chunk=100)
    try:
        got, glogs = m.generate(prompt, cfg.decode_steps, want_logits=True)
        rep = compare(got, glogs, ids, logs)
        assert rep.strict_ids and rep.max_rel_err <= 2e-2, rep.summary()
        K, _ = m.read_kv(1, 0, len(prompt))           # keys in the weights' order
        if K.dtype == np.uint16:
            K = inputs.bf16_bits_to_f32(K)
        assert inf_rel(K, orc.K[1][:len(prompt)]) <= 2e-2
    finally:
        m.close()


@pytest.mark.parametrize("wdt", ["q8", "f32"])
def test_other_rotary_embeddings_of_other_weights(cuda_ok, wdt):
    cfg = CFGS[wdt]
    w, w64 = weights(cfg)
    spec = dict(dim=32, layout="pairs", base=1000.0, scaling="base", factor=2.0)
    prompt = inputs.make_prompt(cfg)
    ids, logs = DecoderOracle(cfg, w64, rope=spec, max_seq=cfg.max_seq).generate(prompt, 6)
    m = model(cfg, w, rope=ops.rope_spec(**spec))
    try:
        got, glogs = m.generate(prompt, 6, want_logits=True)
        rep = compare(got, glogs, ids, logs)
        assert rep.strict_ids and rep.max_rel_err <= TOL.get(wdt, 2e-2), rep.summary()
    finally:
        m.close()


def test_a_named_default_embedding_changes_nothing(cuda_ok):
    cfg = CFGS["bf16_128"].with_(kv_dtype="bf16")
    w, _ = weights(cfg)
    prompt = inputs.make_prompt(cfg)
    out = []
    for rope in (None, ops.rope_spec(cfg.head_dim, cfg.rope_base)):
        m = model(cfg, w, rope=rope)
        try:
            out.append(m.generate(prompt, 4, want_logits=True))
        finally:
            m.close()
    assert out[0][0] == out[1][0]
    assert all(np.array_equal(a, b) for a, b in zip(out[0][1], out[1][1]))


@pytest.mark.parametrize("name", ["bf16_128", "f32"])
def test_batched_decode(cuda_ok, name):
    from paper_2608_24204_amd.binding import WiciModel
    cfg = CFGS[name]
    w, w64 = weights(cfg)
    spec = dict(dim=cfg.head_dim, layout="pairs", base=10000.0)
    kw = dict(kv_page=16, rope=ops.rope_spec(**spec))
    rng = np.random.default_rng(7)
    prompts = [rng.integers(0, cfg.vocab, n).astype(np.int32) for n in (40, 1, 17, 32)]
    lead = model(cfg, w, **kw)
    ms = [lead] + [WiciModel(cfg, share_weights_of=lead, **kw) for _ in prompts[1:]]
    try:
        ids, logs = [[] for _ in ms], [[] for _ in ms]
        for b, m in enumerate(ms):
            t, lg = m.prefill(prompts[b], want_logits=True)
            ids[b].append(t), logs[b].append(lg)
        for _ in range(8):
            toks, lg = ms[0].decode_batch(ms, want_logits=True)
            for b in range(len(ms)):
                ids[b].append(int(toks[b])), logs[b].append(lg[b])
        for b in range(len(ms)):
            want, wl = DecoderOracle(cfg, w64, rope=spec, max_seq=cfg.max_seq).generate(prompts[b], 8)
            rep = compare(ids[b], logs[b], want, wl)
            assert rep.strict_ids and rep.max_rel_err <= TOL.get(name, 2e-2), (b, rep.summary())
        other = WiciModel(cfg, share_weights_of=None, **(kw | dict(rope=None)))
        other.close()
        with pytest.raises(WiciError, match="WICI_E_ARG"):      # another embedding's tables
            WiciModel(cfg, share_weights_of=lead, kv_page=16)
    finally:
        for m in ms[::-1]:
            m.close()


def test_profiled_step_and_full_capacity(cuda_ok):
    """The eager, timed step equals the captured one; the last position of the cache is used."""
    cfg = CFGS["bf16_128"]
    w, _ = weights(cfg)
    prompt = inputs.make_prompt(cfg, 100)
    outs = []
    for timed in (False, True):
        m = model(cfg, w, max_seq=104, kv_page=32)
        try:
            m.prefill(prompt)
            toks = []
            for _ in range(4):
                if timed:
                    t, dur = m.profile_decode_step()
                    assert len(dur) == 3 + 5 * cfg.n_layers and np.all(dur[2::5][:cfg.n_layers] > 0)
                else:
                    t, _ = m.decode_step()
                toks.append(t)
            outs.append(toks)
            with pytest.raises(WiciError, match="WICI_E_CAPACITY"):
                m.decode_step()
        finally:
            m.close()
    assert outs[0] == outs[1]


def test_set_rope_refusals(cuda_ok):
    cfg = CFGS["f32"]
    m = model(cfg, weights(cfg)[0])
    try:
        r = ops.rope_spec(64)
        assert m.lib.wici_set_rope(m.h, ctypes.byref(r)) == binding.WICI_E_STATE
    finally:
        m.close()
    for bad in (ops.rope_spec(128), ops.rope_spec(60), ops.rope_spec(64, base=0.5)):
        with pytest.raises(WiciError, match="WICI_E_ARG"):
            model(cfg, {}, rope=bad)
