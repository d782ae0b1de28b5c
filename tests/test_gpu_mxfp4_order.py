"""Kernels on MXFP4 matrices that follow one another with nothing waited for in between."""
import pytest
import torch

import synth
import paper_2604_13519_b200 as ts
from synth.shapes import ModelShape

pytestmark = pytest.mark.gpu


def _draft(vocab, n, seed):
    g = torch.Generator().manual_seed(seed)
    return [int(x) for x in torch.randint(64, vocab, (n,), generator=g)]


@pytest.mark.parametrize("batch,k", [(10, 64), (3, 48), (1, 33), (1, 1)])
@pytest.mark.parametrize("act_split", [True, False], ids=["two_planes", "one_plane"])
def test_steps_back_to_back(batch, k, act_split):
    """Steps that each start under the one before, also across the end of a step: always the same bits."""
    shape = ModelShape("2560-1l", 1, 2560, 20, 4, 128, 4096, 4096, 10000.0, 1e-5)
    gm = ts.Model(shape, max_pages=batch * 12, max_batch=batch, k_max=64, max_rows=max(64, batch * k), max_ctx=164, act_split=act_split, weights="mxfp4")
    gm.load_weights(synth.make_weights(shape))
    gm.kv_pool_tensor().zero_()
    sess = [ts.Session(gm, None, None) for _ in range(batch)]
    for s in sess:
        s.set_cache(100, 70)
    ts.ts_verify(gm, sess, [_draft(shape.vocab, k - 1, i) for i in range(batch)])
    want = gm.read_logits(0, batch * k).copy()
    for _ in range(300):
        ts.ts_verify_replay(gm)
    torch.cuda.synchronize()
    assert (gm.read_logits(0, batch * k).view("u4") == want.view("u4")).all()
    gm.close()
