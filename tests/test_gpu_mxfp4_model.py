"""A model whose projection matrices are held in MXFP4: against the float64 oracle over the values that codes and scales stand for, the
same bits whatever the chunk, and the decode loop that runs the operators together."""
import numpy as np
import pytest
import torch

import mxfp4_ref as ref
import oracle
import synth
import paper_2604_13519_b200 as ts
from gpu_util import GAIN_SEED, check_step, synthetic_context
from paper_2604_13519_b200 import binding as B

pytestmark = pytest.mark.gpu
KINDS = dict(wq=B.TS_W_Q, wk=B.TS_W_K, wv=B.TS_W_V, wo=B.TS_W_O, wg=B.TS_W_GATE, wu=B.TS_W_UP, wd=B.TS_W_DOWN)
_made = {}


# widths that are no multiples of 128 where they need not be: the stored blocks' last columns are empty
SHAPES = dict(synth.SHAPES, odd=synth.shapes.ModelShape("odd", 2, 384, 6, 2, 64, 576, 1280, 10000.0, 1e-5))


def _weights(name):
    """(bf16 weights, the same with the projection matrices as MXFP4 holds them, codes and scales per matrix)"""
    if name not in _made:
        _made.clear()
        w = synth.make_weights(SHAPES[name], gain_seed=GAIN_SEED)
        held, packed = dict(w), {}
        for n, t in w.items():
            if n == "lm_head" or n.split(".")[-1] in KINDS:
                codes, scales = ref.quantise(t.float().numpy())
                packed[n] = torch.from_numpy(codes), torch.from_numpy(scales)
                held[n] = torch.from_numpy(ref.values(codes, scales, t.shape[1])).to(torch.bfloat16)    # (exact)
        _made[name] = w, held, packed
    return _made[name]


def _model(name, batch=1, k_max=8, max_rows=None, max_ctx=1024, act_split=True, packed=False):
    shape = SHAPES[name]
    w, _, codes = _weights(name)
    gm = ts.Model(shape, max_pages=batch * ((max_ctx + 15) // 16) + 4, max_batch=batch, k_max=k_max, max_rows=max_rows or batch * k_max,
                  max_ctx=max_ctx, act_split=act_split, weights="mxfp4")
    gm.load_weights(w)
    if packed:
        gm.load_tensor_mxfp4(B.TS_W_LM_HEAD, 0, *codes["lm_head"], shape.d_model)
        for l in range(shape.n_layers):
            for n, kind in KINDS.items():
                c, s = codes[f"l{l}.{n}"]
                gm.load_tensor_mxfp4(kind, l, c.cuda() if n == "wo" else c, s.cuda() if n == "wo" else s, w[f"l{l}.{n}"].shape[1])
    return gm


def _draft(vocab, n, seed):
    g = torch.Generator().manual_seed(seed)
    return [int(x) for x in torch.randint(64, vocab, (n,), generator=g)]


@pytest.mark.parametrize("name,ctx,ks,act_split", [("tiny", 100, (1, 2, 3, 8, 33, 64), True), ("tiny", 100, (1, 3, 8, 33, 64), False),
                                                   ("odd", 60, (1, 4, 5, 64), True), ("odd", 60, (1, 4, 5, 64), False),
                                                   ("1b-2l", 300, (3, 40), True), ("1b-2l", 300, (2, 40), False), ("8b-2l", 200, (1, 60), True)])
def test_steps_against_the_oracle(name, ctx, ks, act_split):
    shape = SHAPES[name]
    om = oracle.OracleModel(shape, _weights(name)[1])
    gm = _model(name, k_max=64, max_ctx=ctx + 128, act_split=act_split)
    cache, s, pending = synthetic_context(shape, om, gm, ctx)
    for k in ks:
        d = _draft(shape.vocab, k - 1, k)
        want = om.verify(pending, d, cache.clone(), want_logits=True)
        r = ts.ts_verify(gm, [s], [d])[0]
        if act_split:
            check_step(r, gm.read_logits(0, k), want, f"k {k}")
        else:   # activations rounded to bf16 at each projection: 2^-9 each, a few of them per layer
            err = np.abs(gm.read_logits(0, k) - want["logits"].numpy())
            assert err.max() <= 0.15 and err.mean() <= 0.02, (k, err.max(), err.mean())


@pytest.mark.parametrize("name,rows", [("tiny", (64, 40, 1)), ("odd", (64, 33, 50)), ("1b-2l", (50, 64, 30)), ("8b-2l", (40, 30))])
def test_batches_against_the_oracle(name, rows):
    shape = SHAPES[name]
    om = oracle.OracleModel(shape, _weights(name)[1])
    gm = _model(name, batch=len(rows), k_max=64, max_rows=sum(rows), max_ctx=512)
    made = [synthetic_context(shape, om, gm, 100 + 37 * i, stream=i) for i in range(len(rows))]
    drafts = [_draft(shape.vocab, k - 1, 5 + i) for i, k in enumerate(rows)]
    res = ts.ts_verify(gm, [m[1] for m in made], drafts)
    for i, k in enumerate(rows):
        want = om.verify(made[i][2], drafts[i], made[i][0].clone(), want_logits=True)
        check_step(res[i], gm.read_logits(res[i].first_row, k), want, f"sequence {i}")


@pytest.mark.parametrize("name", ["tiny", "odd", "1b-2l", "8b-2l"])
def test_rows_do_not_depend_on_the_chunk_nor_on_how_the_weights_came(name):
    shape = SHAPES[name]
    logits = []
    for packed in (False, True):
        gm = _model(name, k_max=64, max_ctx=512, packed=packed)
        K, V = synth.make_synthetic_kv(shape, 200)
        s = ts.Session(gm, None, None)
        for l in range(shape.n_layers):
            s.import_kv(l, K[l], V[l])
        s.set_cache(200, 9)
        d = _draft(shape.vocab, 63, 3)
        ts.ts_verify(gm, [s], [d])
        full = gm.read_logits(0, 64).copy()
        for k in (1, 2, 3, 4, 5, 8, 17, 32, 56, 57):
            ts.ts_verify(gm, [s], [d[:k - 1]])
            assert np.array_equal(gm.read_logits(0, k), full[:k]), k
        logits.append(full)
        s.close()
        gm.close()
    assert np.array_equal(logits[0], logits[1])


def test_the_decode_loop_emits_what_vanilla_decoding_does():
    """Prompt, drafts retrieved from the model's own output and corrupted, verification and commit: the same ids as one by one; then
    a draft tree, sampling acceptance, a replay and a profile of the step."""
    name = "1b-2l"
    shape = SHAPES[name]
    gm = _model(name, k_max=16, max_ctx=512)
    prompt = synth.make_context(shape.vocab, 150)

    def start():
        s = ts.Session(gm, None, None)
        ts.ts_prefill(gm, s, prompt)
        return s
    s, truth = start(), []
    for _ in range(60):
        r = ts.ts_verify(gm, [s], [[]])[0]
        truth += list(r.emitted[:r.n_emitted])
        ts.ts_commit(s, r)
    s, out, steps = start(), [], 0
    while len(out) < 60:
        d = truth[len(out):len(out) + 9]
        if steps % 3 == 1 and len(d) > 4:
            d[4] = (d[4] + 1) % shape.vocab
        r = ts.ts_verify(gm, [s], [d])[0]
        out += list(r.emitted[:r.n_emitted])
        ts.ts_commit(s, r)
        steps += 1
    assert out[:60] == truth and steps < 20
    s = start()
    tree = [truth[0], 70, truth[1], 71]
    r, path = ts.ts_verify_tree(gm, [s], [tree], [[0, 0, 1, 1]])
    assert list(r[0].emitted[:r[0].n_emitted]) == truth[:3] and path[0] == [0, 1, 3]
    s = start()
    r = ts.ts_verify_sampled(gm, [s], [truth[:3]], 1e-3, [0.5] * 4)[0]
    assert list(r.emitted[:r.n_emitted]) == truth[:4]
    before = gm.read_logits(0, 4).copy()
    ts.ts_verify_replay(gm)
    assert np.array_equal(gm.read_logits(0, 4), before)
    prof = ts.ts_profile_step(gm)
    assert prof["gemm"][1] >= 4 * shape.n_layers + 1 and prof["rope_kv"][1] == shape.n_layers
    assert len(gm.timeline()) > 0
    gm.inject_device_error(1)
    with pytest.raises(ts.TsError):
        ts.ts_verify(gm, [s], [truth[:3]])
    ts.ts_verify(gm, [s], [truth[:3]])
    assert np.array_equal(gm.read_logits(0, 4), before)


def test_refusals():
    gm = _model("tiny")
    w, _, packed = _weights("tiny")
    c, s = packed["l0.wq"]
    for kind, layer, rows in ((B.TS_W_Q, 5, 256), (B.TS_W_EMBED, 0, 4096), (B.TS_W_GAIN1, 0, 1)):
        with pytest.raises(ts.TsError):
            gm.load_tensor_mxfp4(kind, layer, c[:rows], s[:rows], 256)
    with pytest.raises(ts.TsError):
        gm.load_tensor_mxfp4(B.TS_W_Q, 0, c[:100], s[:100], 256)
    with pytest.raises(ValueError):
        gm.load_tensor_mxfp4(B.TS_W_Q, 0, c, s, 288)
    plain = ts.Model(synth.SHAPES["tiny"], max_pages=8, max_batch=1, k_max=4, max_rows=4, max_ctx=64)
    with pytest.raises(ts.TsError) as e:
        plain.load_tensor_mxfp4(B.TS_W_Q, 0, c, s, 256)
    assert e.value.code == -2
