"""The scratch of the windowed train step holds every batch that the model admits.  What a backward pass needs does not grow
steadily with the sequence: a window or a number of sink keys that the sequence does not exceed is cut to it, and with them
change the number of key blocks that are divided and the heads whose dS^T is kept at a time."""
import math

import pytest

import synth_inputs as SI
from tests.parity_util import lib_config, oracle_config, to_dev

pytestmark = pytest.mark.gpu


# query / kv heads, head dim, batch, length, window, sinks
@pytest.mark.parametrize("nh,nkv,d,max_batch,max_seq,window,sinks", [
    (4, 1, 64, 1, 256, 221, 4), (2, 1, 64, 2, 1500, 1463, 750), (16, 8, 64, 3, 256, 226, 4), (4, 4, 128, 2, 700, 1, 700),
    (16, 2, 64, 3, 5000, 2500, 5000), (12, 3, 128, 4, 8192, 1, 8192)])
def test_every_batch_fits_the_scratch_of_the_setting(nh, nkv, d, max_batch, max_seq, window, sinks):
    from paper_2609_13645_b200 import binding as B
    L = B.lib()
    ocfg = oracle_config(n_layers=1, d_model=256, n_heads=nh, n_kv_heads=nkv, head_dim=d, d_ffn=688, vocab=1024)
    m = B.Model(lib_config(B, ocfg, max_batch, max_seq), seed=1)
    have = L.ft_attention_window_bytes(m._h, window, sinks)
    need = {(b, s): L.ft_k_attention_window_scratch_bytes(b, s, nh, nkv, d, window, sinks) for b in range(1, max_batch + 1)
            for s in range(1, max_seq + 1)}
    worst = max(need, key=need.get)
    assert have == need[worst]  # enough, and not more than the largest batch needs
    if max_seq <= 1500:
        m.set_attention_window(window, sinks)
        tok, lab = (to_dev(t) for t in SI.batch(ocfg.vocab, *worst, "zipf", seed=2))
        loss, gn = m.train_step(tok, lab)
        assert math.isfinite(loss) and math.isfinite(gn)
    m.close()


def test_masks_beyond_the_sequence_need_what_those_at_its_end_need():
    from paper_2609_13645_b200 import binding as B
    L, top = B.lib(), 2 ** 31 - 1
    ocfg = oracle_config(n_layers=1, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ffn=688, vocab=1024)
    m = B.Model(lib_config(B, ocfg, 2, 700), seed=1)
    for far, near in (((top, top), (700, 700)), ((top, 0), (700, 0)), ((30, top), (30, 700)), ((top - 1, 5), (700, 5))):
        assert L.ft_attention_window_bytes(m._h, *far) == L.ft_attention_window_bytes(m._h, *near) > 0
    m.set_attention_window(top, top)
    tok, lab = (to_dev(t) for t in SI.batch(ocfg.vocab, 2, 700, "zipf", seed=2))
    assert math.isfinite(m.train_step(tok, lab)[0])
    m.close()
