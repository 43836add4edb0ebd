"""Timed cases of the 8-bit activations: making them (``quantize_fp8``,
``rmsnorm_fp8``) and the products that read them (``matmul_fp8``,
``dequant_matmul_fp8``).

Values are held in e4m3, with one scale for each block of 128 features of a
token (or of 128 rows x 128 features of a weight); the scales made here are
powers of two (e8m0), those of a weight may be any float32.  Both are returned
in torch's types of these names, whose numbers are the values themselves.

Inputs are synthetic with the distributions of the package's own workloads:
Gaussian weights, activations with log-normal channel scales and 1% outlier
channels.
"""

import math

import torch

own = False

BLOCK = 128
EPS = 1e-5
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    norm, quant = dict(kind="norm"), dict(kind="quantize")
    product, codes = dict(kind="product"), dict(kind="codes", group=128)
    return [
        # one decoding step of a 7B model: latency
        dict(norm, name="norm 1x4096", T=1, m=4096, x="f16", r="f16"),
        # an odd number of tokens of a width that is no multiple of 128, the
        # product's float32 output added to a float32 stream
        dict(norm, name="norm 1999x2500", T=1999, m=2500, x="f32", r="f32"),
        # four prompts of 2048 tokens at a 70B model's width
        dict(norm, name="norm 8192x8192", T=8192, m=8192, x="bf16", r="bf16"),
        # calibration activations as dequant_matmul takes them, features first
        dict(quant, name="quantize 4096x32768 features first", T=32768, m=4096, x="f16", first="features", rows=1),
        # an 8B up projection brought to 8 bits in blocks of 128 x 128
        dict(quant, name="quantize weights 14336x4096", T=14336, m=4096, x="f32", first="rows", rows=128),
        # a decoding step through a layer whose checkpoint has float32 scales
        dict(product, name="product 4096x4096, 1 token", n=4096, m=4096, T=1, scales="f32", rows=128, y="f32", first="tokens"),
        # an odd number of tokens through a 7B down projection with e8m0 scales
        dict(product, name="product 4096x11008, 1999 tokens", n=4096, m=11008, T=1999, scales="e8m0", rows=128, y="bf16", first="tokens"),
        # prefill of 16 sequences of 2048 tokens
        dict(product, name="product 4096x4096, 32768 tokens", n=4096, m=4096, T=32768, scales="f32", rows=128, y="bf16", first="tokens"),
        # the layer as this package quantizes it: one token, a small batch of
        # an up projection, an odd number of tokens with 3-bit codes whose
        # results are the next layer's runtime activations in calibration
        # (float32, features first), and prefill
        dict(codes, name="codes 4096x4096, 1 token", n=4096, m=4096, T=1, bits=4, y="f32", first="features"),
        dict(codes, name="codes 14336x4096, 24 tokens", n=14336, m=4096, T=24, bits=4, y="f16", first="tokens"),
        dict(codes, name="codes 4096x11008, 1999 tokens", n=4096, m=11008, T=1999, bits=3, y="f32", first="features"),
        dict(codes, name="codes 4096x4096, 32768 tokens", n=4096, m=4096, T=32768, bits=4, y="bf16", first="tokens"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def size(lo, hi, step):
        """Log-uniform; half of the draws multiples of `step`, half any number."""
        v = log_int(lo, hi)
        return max(lo, v // step * step) if rng.random() < 0.5 else v

    while True:
        kind = rng.choice(["norm", "norm", "quantize", "quantize", "product", "product", "product", "codes", "codes", "codes"])
        T, m = size(1, 32768, 8), size(1024, 14336, 128)
        if kind == "norm":
            c = dict(kind=kind, T=T, m=m, x=rng.choice(list(TYPES)), r=rng.choice(["none"] + list(TYPES)))
            fits = T * m <= 8192 * 8192
        elif kind == "quantize":
            c = dict(kind=kind, T=T, m=m, x=rng.choice(list(TYPES)), first=rng.choice(["rows", "features"]), rows=1)
            if rng.random() < 0.4:
                c.update(T=size(1024, 14336, 128), first="rows", rows=128)
            fits = c["T"] * m <= 4096 * 32768
        else:
            c = dict(kind=kind, n=size(1024, 14336, 128), m=m, T=T, y=rng.choice(list(TYPES)), first=rng.choice(["tokens", "features"]))
            if kind == "product":
                c.update(scales=rng.choice(["f32", "e8m0"]), rows=rng.choice([128, 128, 1]))
            else:
                c.update(bits=rng.choice([2, 3, 4, 4]), group=rng.choice([128, 128, 128, 256, 0]))
            fits = c["n"] * m * T <= 4096 * 4096 * 32768 and c["n"] * T <= 1.4e8
        if fits:
            return c


# ---- inputs -----------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _channel_scales(m, g):
    sig = torch.exp(torch.randn(m, generator=g, device="cuda"))
    sig[torch.randperm(m, generator=g, device="cuda")[: max(1, round(0.01 * m))]] *= 50.0
    return sig


def _activations(T, m, g):
    return torch.randn(T, m, generator=g, device="cuda").mul_(_channel_scales(m, g))


def _padded(rows, m, dtype):
    """[rows, m] in rows of a multiple of 128 numbers, as the package lays 8-bit arrays out."""
    wide = torch.zeros(rows, -(-m // BLOCK) * BLOCK, dtype=torch.uint8, device="cuda").view(dtype)
    return wide[:, :m]


def _in_8_bits(x, rows):
    """An 8-bit array and its e8m0 scales, made beforehand for the products."""
    T, m = x.shape
    G = -(-m // BLOCK)
    blocks = -(-T // rows)
    p = torch.zeros(blocks * rows, G * BLOCK, device="cuda")
    p[:T, :m] = x
    p = p.view(blocks, rows, G, BLOCK)
    f, e = torch.frexp(p.abs().amax((1, 3)))
    e = e - 9 + (f > 0.875).int()
    q = (p * _pow2(-e).float().view(blocks, 1, G, 1)).view(blocks * rows, G * BLOCK)[:T, :m]
    out = _padded(T, m, E4M3)
    out.copy_(q.to(E4M3))
    s = torch.zeros(blocks, -(-G // 4) * 4, dtype=torch.uint8, device="cuda")
    s[:, :G] = (e + 127).to(torch.uint8)
    return out, s.view(E8M0)[:, :G]


def _packed_codes(n, m, bits, g):
    """Codes as ``pack_codes`` stores them: a row is a little-endian stream of fields of `bits` bits."""
    words = (m * bits + 31) // 32
    q = torch.randint(0, 1 << bits, (n, m), generator=g, device="cuda", dtype=torch.uint8)
    stream = torch.zeros(n, words * 32, dtype=torch.uint8, device="cuda")
    for b in range(bits):
        stream[:, b:m * bits:bits] = (q >> b) & 1
    stream = stream.view(n, words * 4, 8)
    by = sum(stream[:, :, b] << b for b in range(8)).to(torch.uint8)
    return by.contiguous().view(torch.int32)


def prepare(case, seed):
    g = _gen(seed)
    kind, m, T = case["kind"], case["m"], case["T"]
    s = dict(case)
    if kind == "norm":
        s["X"] = _activations(T, m, g).to(TYPES[case["x"]])
        s["R"] = None if case["r"] == "none" else _activations(T, m, g).to(TYPES[case["r"]])
        s["R2"] = None if s["R"] is None else torch.empty_like(s["R"])
        s["gain"] = 1 + 0.2 * torch.randn(m, generator=g, device="cuda")
    elif kind == "quantize":
        x = torch.randn(T, m, generator=g, device="cuda").mul_(0.02) if case["rows"] > 1 else _activations(T, m, g)
        s["X"] = (x.t() if case["first"] == "features" else x).to(TYPES[case["x"]]).contiguous()
    else:
        n, G = case["n"], -(-m // BLOCK)
        s["X8"], s["xs"] = _in_8_bits(_activations(T, m, g), 1)
        if kind == "product":
            s["W8"], s["ws"] = _in_8_bits(torch.randn(n, m, generator=g, device="cuda").mul_(0.02), case["rows"])
            if case["scales"] == "f32":   # as a checkpoint from elsewhere has them
                s["ws"] = s["ws"].float() * (1 + torch.rand(s["ws"].shape, generator=g, device="cuda"))
        else:
            groups = 1 if case["group"] <= 0 else -(-m // case["group"])
            s["P"] = _packed_codes(n, m, case["bits"], g)
            s["S"] = 0.005 * (0.5 + torch.rand(n, groups, generator=g, device="cuda"))
            s["Z"] = torch.randint(0, 1 << case["bits"], (n, groups), generator=g, device="cuda").float()
    return s


# ---- one pass ---------------------------------------------------------------


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    import paper_2602_08376_amd as ok
    if s["kind"] == "norm":
        # the stream's new state goes to a buffer of its own, so that a pass can be repeated
        x8, xs = ok.rmsnorm_fp8(s["X"], s["gain"], EPS, residual=s["R"], residual_out=s["R2"])
        return dict(x8=x8, scales=xs, residual=s["R2"])
    if s["kind"] == "quantize":
        x8, xs = ok.quantize_fp8(s["X"], block_rows=s["rows"], features_first=s["first"] == "features")
        return dict(x8=x8, scales=xs)
    how = dict(tokens_first=s["first"] == "tokens", dtype=TYPES[s["y"]])
    if s["kind"] == "product":
        return ok.matmul_fp8(s["W8"], s["ws"], s["X8"], s["xs"], **how)
    return ok.dequant_matmul_fp8(s["P"], s["S"], s["Z"], s["m"], s["bits"], s["group"], s["X8"], s["xs"], **how)


def _blocks(x, rows):
    """x [T, m] as [blocks of rows, rows, blocks of features, 128], zeros past its ends."""
    T, m = x.shape
    p = torch.nn.functional.pad(x, (0, -m % BLOCK, 0, -T % rows))
    return p.view(p.shape[0] // rows, rows, p.shape[1] // BLOCK, BLOCK)


def _pow2(e):
    """2^e for whole e of a float64's normal range, exactly (torch.ldexp goes through pow)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _to_8_bits(x, rows):
    """The e4m3 values and e8m0 scales of finite x [T, m], in 64 bits: the rounding is that of x itself."""
    T, m = x.shape
    p = _blocks(x.double(), rows)
    a = p.abs().amax((1, 3), keepdim=True)
    f, e = torch.frexp(a)                                   # a = f 2^e, 0.5 <= f < 1
    e = (e - 9 + (f > 0.875).int()).clamp_(min=-127)        # 448 = 0.875 2^9
    e = torch.where(a > 0, e, torch.zeros_like(e))
    v = p * _pow2(-e)
    step = _pow2(torch.frexp(v)[1].clamp_(min=-5) - 4)      # of e4m3 at v: 2^(exponent - 3), at least 2^-9
    v = (v / step).round_().mul_(step)
    x8 = v.reshape(v.shape[0] * rows, -1)[:T, :m].float().to(E4M3)
    return x8, _pow2(e)[:, 0, :, 0].float().to(E8M0)


def _wide(v8, scales, rows):
    """float32 of an 8-bit array: each value times its block's scale."""
    T, m = v8.shape
    s = scales.float().repeat_interleave(BLOCK, 1)[:, :m].repeat_interleave(rows, 0)[:T]
    return v8.float().mul_(s)


def _weights(s):
    """float32 S (Q - Z) from the packed codes."""
    m, bits = s["m"], s["bits"]
    at = torch.arange(m, device="cuda") * bits
    word, off = at // 32, at % 32
    w = s["P"].to(torch.int64) & 0xFFFFFFFF
    after = (word + 1).clamp_(max=w.shape[1] - 1)
    q = ((w[:, word] >> off) | (w[:, after] << (32 - off))) & ((1 << bits) - 1)
    g = m if s["group"] <= 0 else min(m, s["group"])
    S, Z = (v.repeat_interleave(g, 1)[:, :m] for v in (s["S"], s["Z"]))
    return q.float().sub_(Z).mul_(S)


def _plain(s):
    if s["kind"] == "norm":
        h, r = s["X"].float(), None
        if s["R"] is not None:
            h = h + s["R"].float()
            r = h.to(s["R"].dtype)
        h = h.double()
        y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * s["gain"].double()
        x8, xs = _to_8_bits(y, 1)
        return dict(x8=x8, scales=xs, residual=r)
    if s["kind"] == "quantize":
        x8, xs = _to_8_bits(s["X"].t() if s["first"] == "features" else s["X"], s["rows"])
        return dict(x8=x8, scales=xs)
    W = _wide(s["W8"], s["ws"], s["rows"]) if s["kind"] == "product" else _weights(s)
    X = _wide(s["X8"], s["xs"], 1)
    Y = X @ W.t() if s["first"] == "tokens" else W @ X.t()
    return Y.to(TYPES[s["y"]])


# ---- the operators' definitions in 64 bits ------------------------------------


def _grid():
    """Every finite e4m3 number, ascending."""
    v = torch.arange(256, dtype=torch.uint8, device="cuda").view(E4M3).double()
    return torch.unique(v[v.isfinite()])


def _rounded(v):
    """v rounded to e4m3: the nearer neighbour on the grid, the one with an even last bit at equal distance."""
    grid = _grid()
    up = torch.searchsorted(grid, v.contiguous()).clamp_(max=len(grid) - 1)
    down = (up - 1).clamp_(min=0)
    hi, lo = grid[up], grid[down]
    even = (down - len(grid) // 2) % 2 == 0                  # the grid's middle is 0; every other number is even
    return torch.where((v - lo < hi - v) | ((v - lo == hi - v) & even), lo, hi)


def _exact_8_bits(x, rows):
    T, m = x.shape
    x8 = torch.empty(T, m, dtype=torch.float64, device="cuda")
    out = torch.empty(-(-T // rows), -(-m // BLOCK), dtype=torch.float64, device="cuda")
    power = torch.tensor([2.0 ** k for k in range(-128, 129)], dtype=torch.float64, device="cuda")
    step = max(rows, 512 // rows * rows)
    for a in range(0, T, step):
        p = _blocks(x[a:a + step].double(), rows)
        most = p.abs().amax((1, 3))
        sc = power[torch.searchsorted(448.0 * power, most).clamp_(min=1)]   # the least with most <= 448 sc
        sc = torch.where(most > 0, sc, torch.ones_like(sc))
        v = _rounded(p / sc[:, None, :, None]).reshape(-1, p.shape[2] * BLOCK)
        x8[a:a + step] = v[:x[a:a + step].shape[0], :m]
        out[a // rows:a // rows + sc.shape[0]] = sc
    return x8, out


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "norm":
        h, r = s["X"].float(), None
        if s["R"] is not None:
            h = (s["X"].double() + s["R"].double()).float()  # a sum in 64 bits rounded to 32 is that of 32 for these types
            r = h.to(s["R"].dtype).double()
        norm = torch.linalg.vector_norm(h.double(), dim=1, keepdim=True)
        y = h.double() / torch.sqrt(norm * norm / s["m"] + EPS) * s["gain"].double()
        x8, xs = _exact_8_bits(y, 1)
        return dict(x8=x8, scales=xs, residual=r)
    if s["kind"] == "quantize":
        x8, xs = _exact_8_bits(s["X"].t() if s["first"] == "features" else s["X"], s["rows"])
        return dict(x8=x8, scales=xs)
    n, m, T = s["n"], s["m"], s["T"]
    block = torch.arange(m, device="cuda") // BLOCK
    X = s["X8"].double() * s["xs"].double()[:, block]
    if s["kind"] == "product":
        W = s["W8"].double() * s["ws"].double()[torch.arange(n, device="cuda") // s["rows"]][:, block]
    else:
        # bit by bit
        bit = (s["P"].view(torch.uint8).unsqueeze(-1) >> torch.arange(8, device="cuda", dtype=torch.uint8)) & 1
        bit = bit.view(n, -1)[:, :m * s["bits"]].reshape(n, m, s["bits"])
        q = sum(bit[:, :, b].double() * 2.0 ** b for b in range(s["bits"]))
        grp = torch.arange(m, device="cuda") // (m if s["group"] <= 0 else s["group"])
        W = s["S"].double()[:, grp] * (q - s["Z"].double()[:, grp])
    return X @ W.t() if s["first"] == "tokens" else (X @ W.t()).t()


def work(case):
    m, T, G = case["m"], case["T"], -(-case["m"] // BLOCK)
    if case["kind"] == "norm":
        r = 0 if case["r"] == "none" else 2 * SIZE[case["r"]]
        return {"bytes": T * m * (SIZE[case["x"]] + r + 1) + 4 * m + T * G, "flops": 8 * T * m}
    if case["kind"] == "quantize":
        return {"bytes": T * m * (SIZE[case["x"]] + 1) + -(-T // case["rows"]) * G, "flops": 3 * T * m}
    n = case["n"]
    if case["kind"] == "product":
        w = n * m + -(-n // case["rows"]) * G * (4 if case["scales"] == "f32" else 1)
    else:
        groups = 1 if case["group"] <= 0 else -(-m // case["group"])
        w = n * ((m * case["bits"] + 31) // 32 * 4 + 8 * groups)
    return {"bytes": w + T * (m + G) + n * T * SIZE[case["y"]], "flops": 2 * n * m * T}
