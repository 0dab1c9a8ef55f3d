"""The cases that the microscaled 4-bit operators and the quantizing norm are measured on.

They are what one decoder layer of a 7B-class model (hidden 4096, MLP 11008) calls around its
linears when weights and activations are held in the block-scaled 4-bit format: quantizing
activations, the product with weights laid out at load time, and the RMS norm that adds the
residual and leaves the next product's operand (8-bit codes with a scale per token, or the 4-bit
format).  Small, ragged and single-token calls stand beside the large ones.

``run`` computes them in elementary torch operations, in 32 bits (sums of squares in 64), or,
where ``own`` is set, through the package's entry points.
"""
import math

import torch

own = False

#: 2 M N K of the largest listed product: no drawn one does more.
MOST = 2 * 2048 * 11008 * 4096
EPS = 1e-5
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
#: Magnitudes of the eight E2M1 codes without their sign.
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # one token's activations on their way into the 4-bit format: latency
        {"name": "quantize_token_1x4096", "kind": "quantize", "M": 1, "K": 4096, "type": "fp16"},
        # fp32 rows that divide by nothing: a partial last block, unaligned rows
        {"name": "quantize_ragged_333x2999", "kind": "quantize", "M": 333, "K": 2999, "type": "fp32"},
        # the input of the down projection of a 2048-token prompt
        {"name": "quantize_prompt_2048x11008", "kind": "quantize", "M": 2048, "K": 11008, "type": "bf16"},
        # the smallest product, where launches are everything
        {"name": "product_16x512x512", "kind": "product", "M": 16, "N": 512, "K": 512, "type": "fp16",
         "out": "fp32"},
        # one token through the gate projection
        {"name": "product_token_1x11008x4096", "kind": "product", "M": 1, "N": 11008, "K": 4096,
         "type": "bf16", "out": "bf16"},
        # a decode batch through the down projection: few rows, a long K
        {"name": "product_batch_64x4096x11008", "kind": "product", "M": 64, "N": 4096, "K": 11008,
         "type": "fp16", "out": "fp16"},
        # sizes that divide by nothing
        {"name": "product_ragged_333x5003x2999", "kind": "product", "M": 333, "N": 5003, "K": 2999,
         "type": "bf16", "out": "fp32"},
        # the gate projection of a 2048-token prompt
        {"name": "product_prompt_2048x11008x4096", "kind": "product", "M": 2048, "N": 11008, "K": 4096,
         "type": "bf16", "out": "bf16"},
        # one token's norm in front of a linear on 8-bit codes
        {"name": "norm_codes_token_1x4096", "kind": "norm", "M": 1, "K": 4096, "type": "fp16", "to": "codes",
         "q": 8, "residual": True},
        # a prompt's norm in front of a linear on 8-bit codes
        {"name": "norm_codes_prompt_2048x4096", "kind": "norm", "M": 2048, "K": 4096, "type": "fp16",
         "to": "codes", "q": 8, "residual": True},
        # a prompt's norm into the 4-bit format
        {"name": "norm_mx4_prompt_2048x4096", "kind": "norm", "M": 2048, "K": 4096, "type": "bf16", "to": "mx4",
         "q": 4, "residual": True},
        # the front half of a layer's MLP for a 256-token chunk: residual, norm, gate product
        {"name": "layer_256x11008x4096", "kind": "layer", "M": 256, "N": 11008, "K": 4096, "type": "bf16",
         "out": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A width: half of them multiples of 128 as models have, half as they come."""
    v = _log(rng, lo, hi)
    return max(lo, v // 128 * 128) if v >= 256 and rng.random() < 0.5 else v


def draw(rng):
    kind = rng.choice(["quantize", "product", "product", "product", "norm", "norm", "layer"])
    if kind == "quantize":
        M, K, t = _log(rng, 1, 2048), _size(rng, 64, 11008), rng.choice(["fp16", "bf16", "fp32"])
        return {"kind": kind, "M": M, "K": K, "type": t}
    if kind == "norm":
        return {"kind": kind, "M": _log(rng, 1, 2048), "K": _size(rng, 64, 8192), "type": rng.choice(["fp16", "bf16"]),
                "to": rng.choice(["codes", "mx4"]), "q": rng.randint(2, 8), "residual": rng.random() < 0.7}
    N, K = _size(rng, 64, 12288), _size(rng, 64, 11008)
    M = max(1, min(_log(rng, 1, 2048), MOST // (2 * N * K)))
    return {"kind": kind, "M": M, "N": N, "K": K, "type": rng.choice(["fp16", "bf16"]),
            "out": rng.choice(["fp16", "bf16", "fp32"])}


# ---- inputs ---------------------------------------------------------------------

def _generator(seed, *sub):
    g = torch.Generator(device="cuda")
    for s in sub:
        seed = (seed * 1000003 + s + 17) % (1 << 62)
    g.manual_seed(seed)
    return g


def _activations(seed, sub, rows, K, dtype):
    """Activations of a decoder layer: a Gaussian body with a per-token spread (log-normal) and 1%
    outlier channels, 10 to 50 times larger."""
    g = _generator(seed, sub)
    x = torch.randn((rows, K), device="cuda", generator=g)
    x *= torch.exp(0.75 * torch.randn((rows, 1), device="cuda", generator=g))
    boost = 10.0 + 40.0 * torch.rand(K, device="cuda", generator=g)
    pick = torch.rand(K, device="cuda", generator=g) < 0.01
    return (x * torch.where(pick, boost, torch.ones_like(boost))).to(dtype)


def _weights(seed, N, K):
    """A 4-bit checkpoint's tensor as it is stored, row by row: codes two to a byte, the even
    element low, and the scale bytes of the blocks of 32."""
    g = _generator(seed, 1)
    blocks = -(-K // 32)
    codes = torch.randint(0, 256, (N, -(-K // 2)), dtype=torch.uint8, device="cuda", generator=g)
    if K % 2:
        codes[:, -1] &= 15
    # scales of Gaussian weights of deviation 0.02: block maxima between about 0.03 and 0.08
    scales = torch.randint(119, 122, (N, blocks), dtype=torch.uint8, device="cuda", generator=g)
    return codes, scales


def prepare(case, seed):
    t, M, K = TYPES[case["type"]], case["M"], case["K"]
    state = {"case": case, "x": _activations(seed, 2, M, K, t)}
    if case["kind"] in ("norm", "layer"):
        state["gain"] = (1.0 + 0.25 * torch.randn(K, device="cuda", generator=_generator(seed, 3))).to(t)
        if case.get("residual", True):
            state["r"] = _activations(seed, 4, M, K, t)
    if case["kind"] in ("product", "layer"):
        codes, scales = _weights(seed, case["N"], K)
        # laid out once, when the model is loaded: as the values that the plain product takes, or
        # as the operand that the framework's product takes
        if own:
            import paper_2508_19087_amd as apt
            state["w"] = apt.mx4_pack(codes, scales, K)
        else:
            state["w"] = _stored_values(codes, scales, K)
    return state


def _power_of_two(e):
    """fp32 2^e for whole e of the normal range, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _stored_values(codes, scales, K):
    """fp32 values [N][K] of stored codes and scale bytes."""
    nibbles = torch.stack((codes & 15, codes >> 4), dim=2).reshape(codes.shape[0], -1)[:, :K].long()
    v = torch.tensor(E2M1 + tuple(-x for x in E2M1), device="cuda")[nibbles]
    return v * _power_of_two(scales.int() - 127).repeat_interleave(32, dim=1)[:, :K]


# ---- one pass, in plain operations ----------------------------------------------

def _mx4_values(x):
    """The fp32 values that rows of x become in the 4-bit format."""
    R, K = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -K % 32)).reshape(R, -1, 32)
    step = _power_of_two(torch.frexp(b.abs().amax(dim=2, keepdim=True))[1] - 3)  # floor(log2) - 2
    a = (b / step).abs()
    near = torch.where(a < 2.0, (2.0 * a).round() / 2.0, torch.where(a < 4.0, a.round(), 2.0 * (a / 2.0).round()))
    return (torch.copysign(near.clamp(max=6.0), b) * step).reshape(R, -1)[:, :K]


def _code_values(y, q):
    """The fp32 values that rows of y become as q-bit codes 2x + 1 with an fp16 scale per row."""
    top = float((1 << q) - 1)
    s = (y.float().abs().amax(dim=1, keepdim=True) / top).half().float()
    t = torch.where(s > 0, y.float() / s, torch.zeros_like(y, dtype=torch.float32))
    return (2.0 * torch.floor(t / 2.0) + 1.0).clamp(-top, top) * s


def _norm(state):
    """(h, y): the residual stream and its norm, both in the inputs' type."""
    x, t = state["x"], state["x"].dtype
    h = (x.float() + state["r"].float()).to(t) if "r" in state else x
    mean = h.double().square().mean(dim=1, keepdim=True)
    rstd = (1.0 / torch.sqrt(mean + EPS)).float()
    return h, (h.float() * rstd * state["gain"].float()).to(t)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(state):
    case = state["case"]
    kind = case["kind"]
    if kind == "quantize":
        return _mx4_values(state["x"]).bfloat16()
    if kind == "product":
        return (_mx4_values(state["x"]) @ state["w"].t()).to(TYPES[case["out"]])
    h, y = _norm(state)
    if kind == "layer":
        return h, (_mx4_values(y) @ state["w"].t()).to(TYPES[case["out"]])
    v = _code_values(y, case["q"]).half() if case["to"] == "codes" else _mx4_values(y).bfloat16()
    return (h, v) if "r" in state else v


def _run_own(state):
    import paper_2508_19087_amd as apt
    case = state["case"]
    kind = case["kind"]
    if kind == "quantize":
        return apt.mx4_dequantize(apt.mx4_quantize(state["x"]), torch.bfloat16)
    if kind == "product":
        return apt.mx4_gemm_act(state["x"], state["w"], TYPES[case["out"]])
    r = state.get("r")
    if kind == "layer":
        a, h = apt.rmsnorm_mx4(state["x"], state["gain"], EPS, residual=r)
        return h, apt.mx4_gemm(a, state["w"], TYPES[case["out"]])
    if case["to"] == "codes":
        codes, scale, h = apt.rmsnorm_codes(state["x"], state["gain"], case["q"], EPS, residual=r)
        v = apt.dequantize(codes, scale)
    else:
        a, h = apt.rmsnorm_mx4(state["x"], state["gain"], EPS, residual=r)
        v = apt.mx4_dequantize(a, torch.bfloat16)
    return (h, v) if r is not None else v


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    kind, M, K = case["kind"], case["M"], case["K"]
    size = {"fp16": 2, "bf16": 2, "fp32": 4}
    read = M * K * size[case["type"]]
    if kind == "quantize":
        return {"bytes": read + 2 * M * K, "flops": 0}
    if kind == "norm":
        res = 2 * read if case["residual"] else 0
        return {"bytes": read + res + 2 * K + 2 * M * K, "flops": 0}
    N = case["N"]
    bytes_ = read + N * K * 17 / 32 + M * N * size[case["out"]]
    if kind == "layer":
        bytes_ += 2 * read + 2 * K
    return {"bytes": bytes_, "flops": 2.0 * M * N * K}


# ---- the same in 64 bits ----------------------------------------------------------

def _nearest(v):
    """v (64 bits, not negative) at its nearest E2M1 magnitude, a tie at the even code."""
    grid = torch.tensor(E2M1, dtype=torch.float64, device=v.device)
    middle = (grid[1:] + grid[:-1]) / 2
    below, above = torch.bucketize(v, middle, right=False), torch.bucketize(v, middle, right=True)
    return grid[torch.where(below % 2 == 0, below, above)]


def _exact_mx4(x):
    R, K = x.shape
    out = torch.zeros((R, -(-K // 32) * 32), dtype=torch.float64, device=x.device)
    out[:, :K] = x.double()
    b = out.view(R, -1, 32)
    m = b.abs().max(dim=2, keepdim=True).values
    m = torch.where(m > 0, m, torch.ones_like(m))
    unit = m / torch.frexp(m).mantissa / 8.0  # m's own power of two, over 4
    return (torch.sign(b) * _nearest(b.abs() / unit) * unit).view(R, -1)[:, :K]


def _exact_norm(state):
    """The definition rounds where the operator's outputs and operands are held in fewer bits: h
    and y to the inputs' type, the row's factor and its two products to fp32."""
    t = state["x"].dtype
    h = state["x"].double()
    if "r" in state:
        h = (h + state["r"].double()).to(torch.float32).to(t).double()
    f = torch.rsqrt((h * h).sum(dim=1) / h.shape[1] + EPS).float().double()[:, None]
    y = ((h * f).float().double() * state["gain"].double()).float().to(t)
    return h, y.double()


def exact(case, seed):
    kind = case["kind"]
    state = prepare({k: v for k, v in case.items() if k != "N"} | {"kind": "norm" if kind == "layer" else "quantize" if kind == "product" else kind}, seed)
    if kind == "quantize":
        return _exact_mx4(state["x"])
    if kind in ("product", "layer"):
        codes, scales = _weights(seed, case["N"], case["K"])
        w = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device="cuda")
        for at, nibble in ((0, codes & 15), (1, codes >> 4)):
            v = torch.tensor(E2M1, dtype=torch.float64, device="cuda")[(nibble & 7).long()]
            w[:, at::2] = torch.where(nibble > 7, -v, v)
        w = w[:, :case["K"]] * ((scales.long() + 896) << 52).view(torch.float64).repeat_interleave(32, dim=1)[:, :case["K"]]
        if kind == "product":
            return _exact_mx4(state["x"]) @ w.t()
        h, y = _exact_norm(state)
        return h, _exact_mx4(y) @ w.t()
    h, y = _exact_norm(state)
    if case["to"] == "codes":
        top = 2.0 ** case["q"] - 1.0
        s = (y.abs().amax(dim=1) / top).float().half().double()[:, None]
        # the nearest odd level, ties upward
        v = torch.where(s > 0, 2.0 * torch.floor(y / s / 2.0) + 1.0, torch.ones_like(y)).clamp(-top, top) * s
    else:
        v = _exact_mx4(y)
    return (h, v) if "r" in state else v
