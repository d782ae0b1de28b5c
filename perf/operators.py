"""The operators on weights held in MXFP4 (microscaled 4-bit floating point), as a list of cases with their inputs, one
pass of each and what a pass cannot do without.

Three kinds of pass:
  quantise    a matrix into MXFP4 and its values back: what bringing a checkpoint's matrix into four bits and looking at
              what became of it costs
  dequantise  the values of a matrix that is held in MXFP4
  product     y = x W^T with the weights in MXFP4 and the activations x in 16 or 32 bits: a projection of a decoder

MXFP4: blocks of 32 consecutive elements of a row share a scale 2^(s - 127), s one byte (255: not a number); an element
is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 in four bits, two to a byte, the even one in the low half.  A row whose
length is not a multiple of 32 ends in a block filled up with zeros.
"""
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
MOST_WEIGHTS = 151936 * 4096       # the widest LM head
MOST_FLOPS = 2 * 1024 * 24576 * 4096


def _quantise(name, rows, cols, dtype, stride=0):
    return dict(name=name, kind="quantise", rows=rows, cols=cols, dtype=dtype, stride=stride or cols)


def _dequantise(name, rows, cols, dtype):
    return dict(name=name, kind="dequantise", rows=rows, cols=cols, dtype=dtype)


def _product(name, m, n, k, x, y, stride=0):
    return dict(name=name, kind="product", m=m, n=n, k=k, x=x, y=y, stride=stride or k)


def listed():
    return [
        # the smallest matrix there is: a projection of the tiny decoder
        _quantise("quantise_256x256_bf16", 256, 256, "bf16"),
        # the gate and up rows of one layer of the 8B shape, from a bf16 checkpoint
        _quantise("quantise_24576x4096_bf16", 24576, 4096, "bf16"),
        # a master copy in fp32, odd sizes, columns of a wider matrix
        _quantise("quantise_5001x4100_f32", 5001, 4100, "f32", 4352),
        # an attention output projection of the 8B shape back in bf16
        _dequantise("dequantise_4096x4096_bf16", 4096, 4096, "bf16"),
        # the down projection of the 1B shape, odd sizes, in fp32 for a check by eye
        _dequantise("dequantise_2047x8190_f32", 2047, 8190, "f32"),
        # vanilla decoding, one row: the 8B shape's attention output projection (latency) and its gate-up (bandwidth)
        _product("product_1x4096x4096_bf16", 1, 4096, 4096, "bf16", "bf16"),
        _product("product_1x24576x4096_bf16", 1, 24576, 4096, "bf16", "bf16"),
        # a chunk of eight positions through the 1B shape's down projection, added up in fp32 by its caller
        _product("product_8x2048x8192_bf16_f32", 8, 2048, 8192, "bf16", "f32"),
        # the LM head over a verified chunk of 32 positions: logits in fp32
        _product("product_32x151936x4096_bf16_f32", 32, 151936, 4096, "bf16", "f32"),
        # a ragged batch of fp32 rows, every size odd, rows of a wider buffer
        _product("product_57x5003x4100_f32", 57, 5003, 4100, "f32", "f32", 4608),
        # several sessions' chunks in fp16 through the 8B shape's down projection
        _product("product_301x4096x12288_f16", 301, 4096, 12288, "f16", "f16"),
        # a piece of a prompt through the 8B shape's gate-up: bound by the tensor cores
        _product("product_1024x24576x4096_bf16", 1024, 24576, 4096, "bf16", "bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    kind = rng.choice(["quantise", "dequantise", "product", "product", "product"])
    if kind != "product":
        rows, cols = _log(rng, 1, 32768), _log(rng, 1, 16384)
        if rng.random() < 0.5:
            rows, cols = -(-rows // 128) * 128, -(-cols // 128) * 128
        rows = max(1, min(rows, 24576 * 4096 // cols))
        dtype = rng.choice(["bf16", "bf16", "f32", "f16"])
        case = dict(kind=kind, rows=rows, cols=cols, dtype=dtype)
        if kind == "quantise":
            case["stride"] = cols + rng.choice([0, 0, 8, 13])
        return case
    n, k, m = _log(rng, 64, 151936), _log(rng, 64, 12288), _log(rng, 1, 2048)
    if rng.random() < 0.6:
        n, k = -(-n // 128) * 128, -(-k // 128) * 128
    n = min(n, MOST_WEIGHTS // k)
    m = max(1, min(m, MOST_FLOPS // (2 * n * k)))
    x = rng.choice(["bf16", "bf16", "f32", "f16"])
    return dict(kind="product", m=m, n=n, k=k, x=x, y=rng.choice([x, "f32"]), stride=k + rng.choice([0, 0, 8, 13]))


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _matrix(gen, rows, cols, dtype, stride):
    """Rows of a wider buffer, normally distributed, with a spread of scales from row to row as trained matrices have."""
    full = torch.empty(rows, stride, dtype=TYPES[dtype], device="cuda").normal_(generator=gen)
    full *= torch.exp2(torch.randint(-7, 3, (rows, 1), device="cuda", generator=gen)).to(full.dtype)
    return full[:, :cols]


def _packed(gen, rows, cols):
    """Codes and scales of normally distributed weights with a standard deviation of about 0.02."""
    nb = -(-cols // 32)
    z = torch.empty(rows, 32 * nb, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    z[:, cols:] = 0
    scales = torch.randint(118, 122, (rows, nb), dtype=torch.uint8, device="cuda", generator=gen)
    a = z.abs().mul_(2)
    mag = torch.zeros_like(z, dtype=torch.uint8)
    for border in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
        mag += a > border
    mag += (z < 0).to(torch.uint8) * 8
    return (mag[:, 0::2] + mag[:, 1::2] * 16).contiguous(), scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = dict(case=dict(case))
    if case["kind"] == "quantise":
        state["x"] = _matrix(gen, case["rows"], case["cols"], case["dtype"], case["stride"])
    elif case["kind"] == "dequantise":
        state["codes"], state["scales"] = _packed(gen, case["rows"], case["cols"])
    else:
        state["codes"], state["scales"] = _packed(gen, case["n"], case["k"])
        state["x"] = _matrix(gen, case["m"], case["k"], case["x"], case["stride"])
        if own:
            import paper_2604_13519_b200 as ts
            # weights laid out once, and the scratch memory that a caller keeps beside them
            state["w"] = ts.Mxfp4Matrix(state["codes"], state["scales"], case["k"])
            state["ws"] = state["w"].workspace(case["m"], TYPES[case["x"]])
    return state


# ---- the plain form -----------------------------------------------------------------------------------------------------
def _power(e):
    """2^e in 64 bits, to the last bit: the exponent put in its place (an exponential may be off by one step, and a value
    on a border then falls to the wrong side)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _values(codes, scales, cols):
    """The values that codes and scales stand for, in 32 bits."""
    c = torch.stack((codes & 15, codes >> 4), dim=-1).view(codes.shape[0], -1)
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    s = _power(scales.long() - 127).masked_fill(scales == 255, float("nan")).float()
    v = table[c.int()].view(codes.shape[0], -1, 32) * s[:, :, None]
    return v.view(codes.shape[0], -1)[:, :cols]


def _quantised(x):
    """Codes and scales of a matrix."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    b = torch.zeros(rows, 32 * nb, dtype=torch.float32, device=x.device)
    b[:, :cols] = x
    b = b.view(rows, nb, 32)
    most = b.abs().amax(-1)
    fine = torch.isfinite(most)
    e = (torch.frexp(most)[1] - 3).clamp(-127, 127)          # frexp: most = m 2^e with m in [0.5, 1)
    e = torch.where(most == 0, torch.full_like(e, -127), e)
    a = b.abs().double() * _power(-e)[:, :, None]
    code = torch.zeros(b.shape, dtype=torch.uint8, device=x.device)
    # a value on a border goes to the neighbour with the even code
    for i, border in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (a >= border) if i % 2 else (a > border)
    code += torch.signbit(b).to(torch.uint8) * 8
    code *= fine[:, :, None]
    code = code.view(rows, -1)
    scales = torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8)
    return code[:, 0::2] + code[:, 1::2] * 16, scales


def run(state):
    case = state["case"]
    if own:
        import paper_2604_13519_b200 as ts
        if case["kind"] == "quantise":
            codes, scales = ts.ts_mxfp4_quantise(state["x"])
            return {"scales": scales, "values": ts.ts_mxfp4_dequantise(codes, scales, case["cols"], torch.float32)}
        if case["kind"] == "dequantise":
            return ts.ts_mxfp4_dequantise(state["codes"], state["scales"], case["cols"], TYPES[case["dtype"]])
        return ts.ts_mxfp4_product(state["w"], state["x"], TYPES[case["y"]], workspace=state["ws"])
    if case["kind"] == "quantise":
        codes, scales = _quantised(state["x"])
        return {"scales": scales, "values": _values(codes, scales, case["cols"])}
    if case["kind"] == "dequantise":
        return _values(state["codes"], state["scales"], case["cols"]).to(TYPES[case["dtype"]])
    w = _values(state["codes"], state["scales"], case["k"])
    return torch.matmul(state["x"].float(), w.t()).to(TYPES[case["y"]])


# ---- what a pass cannot do without --------------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": n * -(-k // 32) * 17 + m * k * SIZE[case["x"]] + m * n * SIZE[case["y"]], "flops": 2 * m * n * k}
    elements, blocks = case["rows"] * case["cols"], case["rows"] * -(-case["cols"] // 32)
    if case["kind"] == "dequantise":
        return {"bytes": blocks * 17 + elements * SIZE[case["dtype"]], "flops": elements}
    # x in, codes and scales out, the values out
    return {"bytes": elements * SIZE[case["dtype"]] + blocks * 17 + elements * 4, "flops": 2 * elements}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------
def _two_to(power):
    """2^power for whole powers of -200 to 200: one factor for each binary digit of the distance from -200."""
    digits = (power + 200).to(torch.int64)
    out = torch.full(power.shape, 2.0 ** -200, dtype=torch.float64, device=power.device)
    for i in range(9):
        out = torch.where((digits >> i) & 1 == 1, out * 2.0 ** (1 << i), out)
    return out


def _meant(codes, scales, cols):
    out = torch.empty(codes.shape[0], scales.shape[1] * 32, dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        c = (codes >> (4 * half)).to(torch.int16)
        power, odd, minus = (c >> 1) & 3, c & 1, (c >> 3) & 1
        # the lowest power has no leading one: 0 and a half
        size = torch.where(power == 0, 0.5 * odd.double(), (1 + 0.5 * odd.double()) * (0.5 * (1 << power.long())))
        out[:, half::2] = torch.where(minus == 1, -size, size)
    scale = _two_to(scales.double() - 127)
    scale[scales == 255] = float("nan")
    out *= scale.repeat_interleave(32, dim=1)
    return out[:, :cols]


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "dequantise":
        return _meant(state["codes"], state["scales"], case["cols"])
    if case["kind"] == "product":
        x = state["x"].double()
        out = torch.empty(case["m"], case["n"], dtype=torch.float64, device="cuda")
        for r in range(0, case["n"], 32768):
            out[:, r:r + 32768] = x @ _meant(state["codes"][r:r + 32768], state["scales"][r:r + 32768], case["k"]).t()
        return out
    x = state["x"].double()
    nb = -(-case["cols"] // 32)
    x = torch.nn.functional.pad(x, (0, 32 * nb - case["cols"])).view(-1, 32)
    top = x.abs().max(dim=1, keepdim=True).values
    power = torch.floor(torch.log2(top)).clamp(-150, 150) - 2
    # a logarithm next to a whole number may have been rounded to it
    power = power + (_two_to(power + 3) <= top).double() - (_two_to(power + 2) > top).double()
    power = power.clamp(-127, 127)
    power[top == 0] = -127
    scale = _two_to(power)
    z = x / scale
    step = torch.where(z.abs() < 2, 0.5, torch.where(z.abs() < 4, 1.0, 2.0)).double()
    z = (torch.round(z / step) * step).clamp(-6, 6) * scale
    return {"scales": None, "values": z.view(case["rows"], -1)[:, :case["cols"]]}
