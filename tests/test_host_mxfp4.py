"""CPU checks of the operators on MXFP4 matrices: refusals, sizes, and the reference that the GPU tests go by."""
import ctypes as C

import numpy as np
import pytest

import mxfp4_ref as ref
from paper_2604_13519_b200 import binding as B


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2604_13519_b200 import build
    build.build()


P = 1 << 20     # an address that is never followed: every call below is refused before any device work


def _refused(code, why):
    assert code == -1, code
    text = B.lib().ts_last_error().decode()
    assert why in text, text


def test_conversions_refuse():
    L = B.lib()
    _refused(L.ts_mxfp4_quantise(P, 3, 4, 64, 64, P, P, None), "element type")
    _refused(L.ts_mxfp4_quantise(P, 0, -1, 64, 64, P, P, None), "sides")
    _refused(L.ts_mxfp4_quantise(P, 0, 4, (1 << 21) + 1, 1 << 22, P, P, None), "sides")
    _refused(L.ts_mxfp4_quantise(P, 0, 4, 64, 63, P, P, None), "stride")
    _refused(L.ts_mxfp4_quantise(None, 0, 4, 64, 64, P, P, None), "x is null")
    _refused(L.ts_mxfp4_quantise(P + 1, 0, 4, 64, 64, P, P, None), "aligned")
    _refused(L.ts_mxfp4_quantise(P + 2, 2, 4, 64, 64, P, P, None), "aligned")
    _refused(L.ts_mxfp4_quantise(P, 0, 4, 64, 64, P + 8, P, None), "16-byte")
    _refused(L.ts_mxfp4_quantise(P, 0, 4, 64, 64, P, None, None), "null")
    _refused(L.ts_mxfp4_dequantise(None, P, 4, 64, P, 0, 64, None), "null")
    _refused(L.ts_mxfp4_dequantise(P, P, 4, 64, P, 9, 64, None), "element type")
    _refused(L.ts_mxfp4_dequantise(P, P, 4, 64, None, 0, 64, None), "y is null")
    _refused(L.ts_mxfp4_lay_out(P, P, 4, 64, None, None), "matrix")
    _refused(L.ts_mxfp4_lay_out(P, P, 4, 64, P + 4, None), "matrix")
    _refused(L.ts_mxfp4_matrix_bytes(4, 64, None), "null")


def test_product_refuses():
    L = B.lib()
    good = dict(rows=4, ldx=64, ldy=100, x_type=0, y_type=2, x=P, y=P)

    def call(n=100, k=64, **over):
        m = B.ts_mxfp4_matrix(n, k, P)
        a = B.ts_mxfp4_product_args()
        a.matrix = C.pointer(m)
        for name, v in {**good, **over}.items():
            setattr(a, name, v)
        return L.ts_mxfp4_product(C.byref(a), None)

    _refused(L.ts_mxfp4_product(None, None), "null")
    _refused(L.ts_mxfp4_product(C.byref(B.ts_mxfp4_product_args()), None), "null")
    _refused(call(x_type=5), "element type")
    _refused(call(y_type=-1), "element type")
    _refused(call(rows=-4), "sides")
    _refused(call(k=1 << 22, ldx=1 << 22), "sides")
    _refused(call(ldx=60), "stride")
    _refused(call(ldy=99), "stride")
    _refused(call(x=None), "x is null")
    _refused(call(y=None), "y is null")
    _refused(call(y=P + 2), "aligned")
    _refused(call(status=P + 2), "status")
    assert call(rows=0) == 0 and call(n=0, ldy=0) == 0      # nothing to do
    _refused(L.ts_mxfp4_matrix_init(None, P, 4, 64), "null")
    m = B.ts_mxfp4_matrix()
    _refused(L.ts_mxfp4_matrix_init(C.byref(m), P + 64, 4, 64), "aligned")
    _refused(L.ts_mxfp4_matrix_init(C.byref(m), P, -1, 64), "sides")
    assert L.ts_mxfp4_matrix_init(C.byref(m), None, 0, 64) == 0 and (m.n, m.k) == (0, 64)


def test_sizes():
    L = B.lib()
    out = C.c_uint64()
    size = lambda f, *a: (f(*a, C.byref(out)), out.value)
    assert size(L.ts_mxfp4_matrix_bytes, 128, 128) == (0, 8704)
    assert size(L.ts_mxfp4_matrix_bytes, 129, 1) == (0, 2 * 8704)
    assert size(L.ts_mxfp4_matrix_bytes, 0, 5) == (0, 0)
    # room for fewer rows too: what is asked for the most is never less than what is asked for fewer
    for x_type in (0, 1, 2):
        for n in (100, 5000, 151936):
            most = 0
            for rows in list(range(0, 300)) + [1024, 5000]:
                code, b = size(L.ts_mxfp4_product_workspace, rows, n, 4100, x_type)
                assert code == 0 and b >= most
                most = b
    assert L.ts_mxfp4_product_workspace(3, 100, 33, 7, C.byref(out)) == -1


def test_reference_rounds_by_hand():
    x = np.zeros((1, 32))
    x[0, :16] = [6, 5, 5.1, 4.9, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, 0.26, -0.25, -5, 7.9, -7.5, 0]
    codes, scales = ref.quantise(x)
    assert scales[0, 0] == 127
    v = ref.values(codes, scales, 16)[0]
    assert list(v) == [6, 4, 6, 4, 4, 2, 2, 1, 1, 0, 0.5, 0, -4, 6, -6, 0]
    assert list(ref.quantise(np.full((1, 1), 2.0 ** -126))[1][0]) == [0]
    assert list(ref.quantise(np.full((1, 1), np.inf))[1][0]) == [255]


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        B.ts_mxfp4_quantise(torch.zeros(2, 64))                       # not on a device
    with pytest.raises(TypeError):
        B._mx_type(torch.float64)
    with pytest.raises(ValueError):
        B._mx_packed(torch.zeros(2, 32, dtype=torch.uint8), torch.zeros(2, 2, dtype=torch.uint8), 64)


def test_model_configuration_refuses():
    import synth
    L, out = B.lib(), B.ts_buffer_sizes()
    s = synth.SHAPES["8b"]
    c = B.ts_model_config()
    for n in ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab", "rope_theta", "rms_eps"):
        setattr(c, n, getattr(s, n))
    c.max_pages, c.max_batch, c.k_max, c.max_rows, c.max_ctx, c.act_split = 1024, 1, 32, 32, 16384, 1
    assert L.ts_query_buffer_sizes(C.byref(c), C.byref(out)) == 0
    full, work = out.weights_bytes, out.workspace_bytes
    c.weights = B.TS_WEIGHTS_MXFP4
    assert L.ts_query_buffer_sizes(C.byref(c), C.byref(out)) == 0
    embed = 2 * s.vocab * s.d_model
    assert abs((out.weights_bytes - embed) / (full - embed) - 17 / 64) < 1e-3 and out.workspace_bytes > work
    c.path = 2
    _refused(L.ts_query_buffer_sizes(C.byref(c), C.byref(out)), "path 2")
    c.path, c.weights = 0, 2
    _refused(L.ts_query_buffer_sizes(C.byref(c), C.byref(out)), "weights")
    _refused(L.ts_load_tensor_mxfp4(None, 3, 0, P, P, 4, 64), "null")


def test_workspaces_are_no_larger_than_the_matrix_can_need():
    """Partial sums take memory only where a matrix has tiles enough to be dealt out in runs, and then for no more CTAs than it has work for."""
    L, out = B.lib(), C.c_uint64()

    def size(*a):
        assert L.ts_mxfp4_product_workspace(*a, C.byref(out)) == 0
        return out.value
    planes = lambda rows, k, n: n * (rows + 112) * (k + 127) // 128 * 128 * 2       # (elements; scales and rounding up: twice that)
    assert size(3, 128, 128, 0) <= planes(3, 128, 2)
    assert size(256, 256, 256, 0) <= planes(256, 256, 2)
    assert size(256, 1024, 4096, 2) <= planes(256, 4096, 5) + 24 * 32 * 512 * 16
    assert size(64, 151936, 4096, 0) <= planes(64, 4096, 2) + 512 * 112 * 512 + 4096
    for x_type in (0, 1, 2):
        for k in (1, 128, 300, 4100):
            for rows in (1, 64, 300, 2000):
                most = 0
                for n in (1, 100, 128, 129, 1000, 4096, 19000, 38000, 151936):
                    b = size(rows, n, k, x_type)
                    assert b >= most
                    most = b


def test_a_model_takes_codes_and_scales_of_one_byte_each():
    torch = pytest.importorskip("torch")
    m = B.Model.__new__(B.Model)      # (refused before anything is asked of a model)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    for codes, scales in ((u8(4, 32).int(), u8(4, 2)), (u8(4, 32), u8(4, 2).short()), (u8(4, 32).float(), u8(4, 2)), (u8(128), u8(8)), (u8(4, 32), u8(8))):
        with pytest.raises(ValueError):
            m.load_tensor_mxfp4(B.TS_W_Q, 0, codes, scales, 64)
