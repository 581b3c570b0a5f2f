"""The train step with sliding-window attention in every layer against the CPU oracle, whose attention core is replaced by the
windowed one (same rounding contract).  Tolerances are those of the whole step: loss abs 1e-2, relative L2 2e-2 on every
gradient and on the attention's own intermediate tensors."""
import math

import numpy as np
import pytest
import torch

import synth_inputs as SI
from oracle import decoder as D
from tests.parity_util import lib_config, lib_tap, load_params, oracle_config, rel_l2, to_dev

pytestmark = pytest.mark.gpu


def _windowed(window, sinks):
    """(attention_fwd, attention_bwd) with the oracle's signatures, for sequences of a few hundred tokens."""
    def scores(q, k, n_rep):
        S, d = q.shape[1], q.shape[3]
        i, j = np.arange(S)[:, None], np.arange(S)[None, :]
        seen = (j <= i) & ((i - j < window) | (j < sinks))
        kk = np.repeat(k, n_rep, axis=2)
        return np.where(seen, np.einsum("bind,bjnd->bnij", q, kk) / math.sqrt(d), -np.inf)

    def fwd(q, k, v, n_rep, R, contract):
        s2 = scores(q, k, n_rep) * D.LOG2E
        c = s2.max(-1, keepdims=True)
        c = np.ceil(c) if contract else c
        p = np.exp2(s2 - c)
        l = p.sum(-1)
        o = np.einsum("bnij,bjnd->bind", R(p), np.repeat(v, n_rep, axis=2)) / l.transpose(0, 2, 1)[..., None]
        return R(o), (c[..., 0] + np.log2(l)) * D.LN2

    def bwd(q, k, v, o, do, lse, n_rep, R):
        B, S, nh, d = q.shape
        p = np.exp(scores(q, k, n_rep) - lse[..., None])
        dp = np.einsum("bind,bjnd->bnij", do, np.repeat(v, n_rep, axis=2))
        ds = R(p * (dp - (do * o).sum(-1).transpose(0, 2, 1)[..., None]))
        group = lambda t: t.reshape(B, S, nh // n_rep, n_rep, d).sum(3)  # noqa: E731
        dq = np.einsum("bnij,bjnd->bind", ds, np.repeat(k, n_rep, axis=2)) / math.sqrt(d)
        return dq, group(np.einsum("bnij,bind->bjnd", ds, q)) / math.sqrt(d), group(np.einsum("bnij,bind->bjnd", R(p), do))
    return fwd, bwd


def _config(kind):
    if kind == "plain":
        return oracle_config(n_layers=2, d_model=256, n_heads=4, n_kv_heads=4, head_dim=64, d_ffn=688, vocab=1024), 2, 256
    if kind == "gqa":
        return oracle_config(n_layers=2, d_model=512, n_heads=4, n_kv_heads=2, head_dim=128, d_ffn=720, vocab=2048), 2, 200
    return oracle_config(n_layers=2, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ffn=688, vocab=1024, mtp=True, mtp_weight=0.3,
                         qk_norm=True, tie_embeddings=True), 3, 170


@pytest.mark.parametrize("kind,window,sinks,recompute", [("plain", 64, 4, 0), ("gqa", 33, 0, 0), ("gqa", 50, 7, 1), ("variants", 40, 3, 0), ("plain", 1, 0, 0)])
def test_step_matches_the_oracle_with_windowed_attention(kind, window, sinks, recompute, monkeypatch):
    from paper_2609_13645_b200 import binding as B
    ocfg, Bsz, S = _config(kind)
    params = D.init_params(ocfg, SI.WEIGHT_SEED)
    tok, lab = SI.batch(ocfg.vocab, Bsz, S, "zipf", seed=12)
    taps = not ocfg.mtp and not recompute  # the intermediate tensors are kept by plain steps only
    model = B.Model(lib_config(B, ocfg, Bsz, S, debug_taps=int(taps), recompute=recompute), seed=1)
    model.set_attention_window(window, sinks)
    model.set_fused_update(False)  # the gradients are compared
    load_params(model, params)
    f, b = _windowed(window, sinks)
    monkeypatch.setattr(D, "attention_fwd", f)
    monkeypatch.setattr(D, "attention_bwd", b)
    loss_o, gn_o, grads_o, taps_o = D.TrainState(ocfg, params).train_step(tok, lab, mode="contract", want_taps=True)
    loss, gn = model.train_step(to_dev(tok), to_dev(lab))
    assert abs(loss - loss_o) < 1e-2 and abs(gn - gn_o) / gn_o < 2e-3
    for name in params:
        assert rel_l2(model.get_param(name, B.KIND_GRAD), grads_o[name]) < 2e-2, name
    if taps:
        for l in range(ocfg.n_layers):
            # of one key nothing is left of d_q and d_k but the rounding of delta
            for nm in ("o", "d_o", "d_v") + (("d_q", "d_k") if window > 1 else ()):
                assert rel_l2(lib_tap(model, ocfg, nm, l, Bsz * S), taps_o[f"layers.{l}.{nm}"]) < 2e-2, (l, nm)
    model.close()


def _run(model, tok, lab, steps=4):
    return [model.train_step(tok, lab) for _ in range(steps)]


def test_graph_stream_and_recomputation_change_no_bit_and_off_is_as_never_on():
    from paper_2609_13645_b200 import binding as B
    ocfg, Bsz, S = _config("gqa")
    params = D.init_params(ocfg, 5)
    tok, lab = (to_dev(t) for t in SI.batch(ocfg.vocab, Bsz, S, "zipf", seed=8))

    def steps(window, recompute=0, graph=True, overlap=True, first=None):
        m = B.Model(lib_config(B, ocfg, Bsz, S, recompute=recompute), seed=1)
        load_params(m, params)
        m.set_graph(graph)
        m.set_overlap(overlap)
        if first is not None:
            m.set_attention_window(first, 2)
            m.forward_loss(tok, lab)
        m.set_attention_window(window, 5 if window else 0)
        out = _run(m, tok, lab), [m.get_param(n, B.KIND_MASTER) for n in params]
        m.close()
        return out
    want = steps(48)
    for kw in (dict(recompute=1), dict(graph=False), dict(overlap=False), dict(first=9)):
        got = steps(48, **kw)
        assert got[0] == want[0] and all(np.array_equal(a, b) for a, b in zip(got[1], want[1])), kw
    causal = steps(0)
    assert causal[0] != want[0]
    again = steps(0, first=16)
    assert again[0] == causal[0] and all(np.array_equal(a, b) for a, b in zip(again[1], causal[1]))


def test_shorter_batches_and_refusals():
    from paper_2609_13645_b200 import binding as B
    ocfg, Bsz, S = _config("plain")
    m = B.Model(lib_config(B, ocfg, Bsz, S), seed=1)
    m.set_attention_window(10 ** 6, 3)  # beyond the sequence
    m.set_attention_window(70, 300)
    for b, s in ((1, 1), (2, 77), (1, 129), (2, 256)):
        tok, lab = (to_dev(t) for t in SI.batch(ocfg.vocab, b, s, "zipf", seed=s))
        loss, gn = m.train_step(tok, lab)
        assert math.isfinite(loss) and math.isfinite(gn)
    for window, sinks in ((-1, 0), (5, -1)):
        with pytest.raises(B.ForgeStepError) as e:
            m.set_attention_window(window, sinks)
        assert e.value.status == B.FT_EINVAL
    L, need = B.lib(), int(B.lib().ft_attention_window_bytes(m._h, 64, 4))
    buf = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    assert L.ft_set_attention_window(m._h, 64, 4, buf.data_ptr(), need - 1) == B.FT_ENOMEM
    assert L.ft_set_attention_window(m._h, 64, 4, buf.data_ptr() + 16, need) == B.FT_EINVAL
    assert L.ft_set_attention_window(m._h, 64, 4, None, need) == B.FT_EINVAL
    assert L.ft_set_attention_window(None, 64, 4, buf.data_ptr(), need) == B.FT_EINVAL
    assert L.ft_attention_window_bytes(m._h, 0, 0) == 0
    tok, lab = (to_dev(t) for t in SI.batch(ocfg.vocab, 2, 256, "zipf", seed=1))
    m.train_step(tok, lab)  # the setting before the refused ones is still there
    m.close()
