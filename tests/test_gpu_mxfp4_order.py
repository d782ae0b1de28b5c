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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,n", [(1, 1024), (2, 1024), (4, 640), (8, 1024), (24, 1024), (100, 1024)])
def test_a_product_reads_what_the_one_before_wrote(rows, n, dtype):
    """Products in a chain, each one's result the next one's activations, over the same two buffers again and again: the same as with the
    device waited for behind each."""
    gen = torch.Generator("cuda").manual_seed(rows)
    w = []
    for _ in range(3):
        codes = torch.randint(0, 256, (n, n // 2), dtype=torch.uint8, device="cuda", generator=gen)
        # (elements of random sign, about 2.6 in size: a sum of n of them grows by 2.6 sqrt(n), and the scales take it back)
        w.append(ts.Mxfp4Matrix(codes, torch.full((n, n // 32), 120, dtype=torch.uint8, device="cuda"), n))
    start = [torch.randn(rows, n, device="cuda", generator=gen).to(dtype) for _ in range(4)]
    ws = w[0].workspace(rows, dtype)

    def run(wait):
        a, b, out = torch.empty_like(start[0]), torch.empty_like(start[0]), []
        for i in range(40):
            a.copy_(start[i % 4])
            for j in range(3):
                ts.ts_mxfp4_product(w[(i + j) % 3], a, out=b, workspace=ws)
                if wait:
                    torch.cuda.synchronize()
                a, b = b, a
            out.append(a.clone())
        return out
    want, got = run(True), run(False)
    for x in w:
        x.check()
    for i, (x, y) in enumerate(zip(want, got)):
        assert torch.isfinite(x).all() and torch.equal(x, y), i


def test_a_matrix_may_be_used_on_any_stream_at_once():
    """Laid out on a stream that is still busy, used on another one right behind the constructor, codes and scales let go of."""
    n, k = 1024, 2048
    lays, other = torch.cuda.Stream(), torch.cuda.Stream()
    x = torch.randn(5, k, device="cuda").to(torch.bfloat16)
    codes = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((n, k // 32), 120, dtype=torch.uint8, device="cuda")
    want = ts.ts_mxfp4_product(ts.Mxfp4Matrix(codes, scales, k), x, torch.float32)
    torch.cuda.synchronize()
    for stream in (lays, None):
        c, s = codes.clone(), scales.clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(lays if stream is not None else torch.cuda.current_stream()):
            torch.cuda._sleep(200_000_000)      # (about a tenth of a second)
        w = ts.Mxfp4Matrix(c, s, k, stream=stream)
        del c, s
        lost = [torch.zeros(n, k // 2, dtype=torch.uint8, device="cuda"), torch.zeros(n, k // 32, dtype=torch.uint8, device="cuda")]
        y = ts.ts_mxfp4_product(w, x, torch.float32, stream=other)
        other.synchronize()
        assert torch.equal(y, want)
        del lost
    w.check()


def test_check_waits_for_products_on_every_stream():
    """A product on a stream that is still busy: its status word, set here behind it as an expired wait would set it, is seen, and
    taken back before anything that comes later."""
    codes = torch.randint(0, 256, (128, 64), dtype=torch.uint8, device="cuda")
    w = ts.Mxfp4Matrix(codes, torch.full((128, 4), 120, dtype=torch.uint8, device="cuda"), 128)
    x, side = torch.randn(3, 128, device="cuda"), torch.cuda.Stream()
    for sleep, code in ((1, 0), (400_000_000, 3)):      # (the first time kernels are loaded, which the device is waited for)
        w.check()
        with torch.cuda.stream(side):
            torch.cuda._sleep(sleep)
            y = ts.ts_mxfp4_product(w, x)
            w.status.fill_(code)
    assert not side.query()
    with pytest.raises(ts.TsError) as e:
        w.check()
    assert e.value.code == -6 and "code 3" in str(e.value)
    w.check()


def test_every_launch_of_a_product_is_in_the_timeline():
    """60 rows through an LM head of many tiles: the product takes two launches, each with stamps of its own."""
    shape = ModelShape("wide-head-1l", 1, 512, 8, 4, 64, 1024, 38016, 10000.0, 1e-5)     # 297 tiles
    gm = ts.Model(shape, max_pages=40, max_batch=1, k_max=64, max_rows=64, max_ctx=400, weights="mxfp4")
    gm.load_weights(synth.make_weights(shape))
    gm.kv_pool_tensor().zero_()
    s = ts.Session(gm, None, None)
    s.set_cache(200, 70)
    ts.ts_verify(gm, [s], [_draft(shape.vocab, 59, 2)])
    products = [t for t in gm.timeline() if t[0] == "gemm"]
    assert len(products) == ts.ts_profile_step(gm)["gemm"][1] == 4 * shape.n_layers + 2
    for _, start, first, last, end in products:
        assert start <= first <= last <= end
    assert products[-2][4] <= products[-1][2] and products[-2][4] < products[-1][4]      # (the second of the two waits for the first one's end)
    s.close()
    gm.close()


def test_a_matrix_is_laid_out_behind_what_makes_its_codes():
    """Codes and scales that the current stream is still to write, laid out on another one."""
    n, k = 512, 1024
    gen = torch.Generator("cuda").manual_seed(3)
    packs = [(torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda", generator=gen),
              torch.randint(118, 122, (n, k // 32), dtype=torch.uint8, device="cuda", generator=gen)) for _ in range(2)]
    x = torch.randn(5, k, device="cuda", generator=gen).to(torch.bfloat16)
    want = [ts.ts_mxfp4_product(ts.Mxfp4Matrix(*p, k), x, torch.float32) for p in packs]
    codes, scales = packs[0][0].clone(), packs[0][1].clone()
    side = torch.cuda.Stream()
    ts.Mxfp4Matrix(codes, scales, k, stream=side)      # (memory of that stream, for the next one)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    codes.copy_(packs[1][0])
    scales.copy_(packs[1][1])
    w = ts.Mxfp4Matrix(codes, scales, k, stream=side)
    assert torch.equal(ts.ts_mxfp4_product(w, x, torch.float32), want[1])
    w.check()
