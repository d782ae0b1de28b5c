"""Steps and prompts of models with MXFP4 weights where products are dealt out in runs inside a model, so that a kernel that makes a
product's input also clears the run's flags: gate-up and LM head of many tiles, `down` of hundreds of rows.  Against the float64 oracle over
the values that codes and scales stand for."""
import numpy as np
import pytest
import torch

import mxfp4_ref as ref
import oracle
import synth
import paper_2604_13519_b200 as ts
from gpu_util import GAIN_SEED, check_step, synthetic_context
from synth.shapes import ModelShape
from test_gpu_mxfp4_model import KINDS
from test_gpu_prompts import ROW_REL

pytestmark = pytest.mark.gpu
SHAPES = {"tiny": synth.SHAPES["tiny"], "1b-2l": synth.SHAPES["1b-2l"],
          "wide-ffn": ModelShape("wide-ffn", 2, 512, 8, 4, 64, 19200, 2048, 10000.0, 1e-5),        # gate-up of 300 tiles
          "wide-head": ModelShape("wide-head", 2, 512, 8, 4, 64, 1088, 38016, 10000.0, 1e-5)}      # LM head of 297, `down` of an odd width
_made = {}


def _weights(name):
    """(bf16 weights, oracle over what MXFP4 holds of them)"""
    if name not in _made:
        _made.clear()
        w = synth.make_weights(SHAPES[name], gain_seed=GAIN_SEED)
        held = dict(w)
        for n, t in w.items():
            if n == "lm_head" or n.split(".")[-1] in KINDS:
                codes, scales = ref.quantise(t.float().numpy())
                held[n] = torch.from_numpy(ref.values(codes, scales, t.shape[1])).to(torch.bfloat16)
        _made[name] = w, oracle.OracleModel(SHAPES[name], held)
    return _made[name]


def _draft(vocab, n, seed):
    g = torch.Generator().manual_seed(seed)
    return [int(x) for x in torch.randint(64, vocab, (n,), generator=g)]


@pytest.mark.parametrize("act_split", [True, False], ids=["two_planes", "one_plane"])
@pytest.mark.parametrize("name,rows", [("wide-ffn", (1,)), ("wide-ffn", (5,)), ("wide-ffn", (60,)), ("wide-ffn", (64, 40)), ("wide-ffn", (64,) * 5),
                                       ("wide-head", (3,)), ("wide-head", (60,)), ("wide-head", (64, 33, 30)), ("1b-2l", (58,) * 9), ("1b-2l", (64,) * 16)])
def test_steps(name, rows, act_split):
    shape = SHAPES[name]
    w, om = _weights(name)
    gm = ts.Model(shape, max_pages=len(rows) * 12 + 4, max_batch=len(rows), k_max=64, max_rows=max(64, sum(rows)), max_ctx=164, act_split=act_split, weights="mxfp4")
    gm.load_weights(w)
    made = [synthetic_context(shape, om, gm, 20 + 5 * i, stream=i, pending=300 + i) for i in range(len(rows))]
    drafts = [_draft(shape.vocab, k - 1, 5 + i) for i, k in enumerate(rows)]
    res = ts.ts_verify(gm, [m[1] for m in made], drafts)
    logits = [gm.read_logits(r.first_row, k).copy() for r, k in zip(res, rows)]
    for i in sorted({0, len(rows) // 2, len(rows) - 1}):
        want = om.verify(made[i][2], drafts[i], made[i][0].clone(), want_logits=True)
        if act_split:
            check_step(res[i], logits[i], want, f"{name}, sequence {i}")
        else:   # (bf16 roundings of all activations: as for steps of many rows with bf16 weights)
            lo = want["logits"].numpy()
            assert ((logits[i] - lo) ** 2).sum() <= 4e-2 ** 2 * (lo ** 2).sum()
    again = ts.ts_verify(gm, [m[1] for m in made], drafts)
    for r, k, first in zip(again, rows, logits):
        assert np.array_equal(gm.read_logits(r.first_row, k), first)
    gm.close()


@pytest.mark.parametrize("act_split", [True, False], ids=["two_planes", "one_plane"])
@pytest.mark.parametrize("name,n", [("tiny", 66), ("tiny", 1090), ("wide-head", 200), ("1b-2l", 66), ("1b-2l", 523), ("1b-2l", 1500)])
def test_prompts(name, n, act_split):
    shape = SHAPES[name]
    w, om = _weights(name)
    gm = ts.Model(shape, max_pages=(n + 32) // 16 + 10, max_batch=1, k_max=16, max_rows=16, max_ctx=n + 64, act_split=act_split, weights="mxfp4")
    gm.load_weights(w)
    prompt = synth.make_context(shape.vocab, n)
    cache = om.new_cache()
    om.forward_chunk(prompt[:n - 1], cache)
    s = ts.Session(gm, None, None)
    ts.ts_prefill(gm, s, prompt)
    for l in range(shape.n_layers):
        for got, want in zip(s.export_kv(l, n - 1), (cache.k[l], cache.v[l])):
            want = want[:n - 1].reshape(n - 1, -1)
            err = (got.reshape(n - 1, -1).double() - want).norm(dim=1) / want.norm(dim=1)
            assert float(err.max()) <= ROW_REL[1 + act_split], (l, int(err.argmax()), float(err.max()))
    draft = [100, 200, 300]
    want = om.verify(prompt[n - 1], draft, cache, want_logits=True)
    res = ts.ts_verify(gm, [s], [draft])[0]
    if act_split:
        check_step(res, gm.read_logits(0, 4), want, f"{name}, prompt of {n}")
    gm.close()


@pytest.mark.parametrize("act_split", [True, False], ids=["two_planes", "one_plane"])
@pytest.mark.parametrize("name", ["wide-ffn", "wide-head"])
def test_rows_are_the_same_bits_in_any_chunk(name, act_split):
    """Also where the chunk's last rows take a second launch of the runs."""
    shape = SHAPES[name]
    gm = ts.Model(shape, max_pages=40, max_batch=1, k_max=64, max_rows=64, max_ctx=400, act_split=act_split, weights="mxfp4")
    gm.load_weights(_weights(name)[0])
    K, V = synth.make_synthetic_kv(shape, 200)
    s = ts.Session(gm, None, None)
    for l in range(shape.n_layers):
        s.import_kv(l, K[l], V[l])
    s.set_cache(200, 9)
    d = _draft(shape.vocab, 63, 3)
    ts.ts_verify(gm, [s], [d])
    full = gm.read_logits(0, 64).copy()
    for k in (1, 2, 5, 8, 17, 32, 40, 56, 57, 63):
        ts.ts_verify(gm, [s], [d[:k - 1]])
        assert np.array_equal(gm.read_logits(0, k), full[:k]), k
    gm.close()
