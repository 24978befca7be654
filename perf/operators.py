"""Performance cases of the operators beside the filter: what the rest of a training step needs.

Every case is one pass. `kind` says which entry points of `paper_2609_21102_b200.binding` it goes through:

  adamw      defl_adamw_step: one AdamW step over a list of tensors (the parameters that a Muon step does not take), with
             moments in 32 bits or in 8; with `clip` defl_grad_norm first, whose factor and step counter stay on the GPU
  quantize   defl_mx4_quantize: a batch of matrices to microscaled 4-bit floating point, blocks along the rows and along
             the columns from one read, then defl_mx4_dequantize of both (the values that the codes stand for)
  linear     defl_mx4_quantize of the activations, then defl_mx4_gemm with weights that are held in 4 bits
  train      forward and backward of a linear layer: three quantisations, three products

The plain forms are elementary torch operations in 32 bits; `exact` restates the operators in 64 bits.

Formats. Elements are e2m1 (0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives). "mxfp4": blocks of 32 along the contracted
dimension, the scale a power of two, the smallest with which the block's largest magnitude is at most 6. "nvfp4":
blocks of 16, the scale an e4m3 number (largest magnitude / 6, to nearest even) times one power of two per matrix, the
smallest with which the largest block's scale is at most 448. Codes: two a byte, even column in the low half, rows padded
with zeros to a multiple of 32 columns. Scales: one byte a block in tiles of 128 rows x 4 blocks, 512 bytes each: row r,
block c of a tile at byte (r % 32) * 16 + (r // 32) * 4 + c; padding is zero.

8-bit moments. Blocks of 256 consecutive elements of a tensor; the first moment and the square ROOT of the second are
e4m3 numbers (torch.float8_e4m3fn) times a fp32 scale per block (largest magnitude / 448). Rounding is stochastic:
y = |x| * 448 / largest goes to delta * floor(y / delta + u), delta its spacing and u 16 random bits / 65536.
"""
import math

import torch

own = False

LR, BETA1, BETA2, EPS, DECAY, MAX_NORM = 1e-3, 0.9, 0.999, 1e-8, 0.1, 1.0
TORCH = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = {"mxfp4": 32, "nvfp4": 16}
QBLOCK = 256

_context = None


def _binding():
    from paper_2609_21102_b200 import binding
    return binding


def _ctx():
    """The one context a single-stream program keeps for the life of the process."""
    global _context
    if _context is None:
        _context = _binding().Context(0)
    return _context


def listed():
    a = {"kind": "adamw", "p": "fp32", "g": "bf16", "bits": 32, "clip": False, "copy": False, "packed": False, "step": 100}
    return [
        # a handful of gains and biases: latency is all
        dict(a, name="adamw_tiny", rows=0, width=256, layers=2, g="fp32"),
        # every vector of a 48-layer transformer of width 1600 (386 tensors), gradients clipped by their global norm
        dict(a, name="adamw_vectors_clip", rows=0, width=1600, layers=48, clip=True),
        # the token embedding of that model with its vectors: fp32 master weights, bf16 gradients and a bf16 copy for the forward pass
        dict(a, name="adamw_embedding", rows=50257, width=1600, layers=48, copy=True),
        # the same with moments in 8 bits
        dict(a, name="adamw8_embedding", rows=50257, width=1600, layers=48, bits=8),
        # bf16 weights without a master copy, fp32 gradients, tensors of odd sizes packed back to back, first steps, clipped
        dict(a, name="adamw8_ragged_clip", rows=10007, width=517, layers=12, bits=8, p="bf16", g="fp32", packed=True, clip=True, step=2),
        # the activations of a wide layer for 8192 tokens, both block directions
        {"name": "quantize_wide", "kind": "quantize", "fmt": "mxfp4", "b": 1, "rows": 8192, "cols": 6400, "dtype": "bf16"},
        # odd-sided fp32 matrices (a shape group of master weights)
        {"name": "quantize_ragged", "kind": "quantize", "fmt": "nvfp4", "b": 3, "rows": 517, "cols": 1003, "dtype": "fp32"},
        # one token through a wide layer
        {"name": "linear_token", "kind": "linear", "fmt": "nvfp4", "tokens": 1, "k": 1600, "n": 6400},
        # a layer whose sides are multiples of nothing
        {"name": "linear_ragged", "kind": "linear", "fmt": "mxfp4", "tokens": 333, "k": 1003, "n": 517},
        # a prompt of 8192 tokens through a wide layer
        {"name": "linear_prompt", "kind": "linear", "fmt": "mxfp4", "tokens": 8192, "k": 1600, "n": 6400},
        # training: a small square layer, and the wide one
        {"name": "train_small", "kind": "train", "fmt": "mxfp4", "tokens": 1024, "k": 768, "n": 768},
        {"name": "train_wide", "kind": "train", "fmt": "nvfp4", "tokens": 8192, "k": 1600, "n": 6400},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["adamw", "adamw", "quantize", "linear", "linear", "train"])
    if kind == "adamw":
        p = rng.choice(["fp32", "fp32", "bf16"])
        return {"kind": kind, "rows": rng.choice([0, _log_int(rng, 64, 40000)]), "width": _log_int(rng, 48, 1600), "layers": rng.randint(1, 48),
                "p": p, "g": rng.choice(["fp32", "bf16"]), "bits": rng.choice([8, 32]), "clip": rng.random() < 0.5,
                "copy": p == "fp32" and rng.random() < 0.3, "packed": rng.random() < 0.3, "step": _log_int(rng, 1, 2000)}
    fmt = rng.choice(["mxfp4", "nvfp4"])
    if kind == "quantize":
        return {"kind": kind, "fmt": fmt, "b": rng.randint(1, 4), "rows": _log_int(rng, 1, 4096), "cols": _log_int(rng, 16, 3000),
                "dtype": rng.choice(["bf16", "fp32"])}
    k, n = _log_int(rng, 48, 1600), _log_int(rng, 32, 6400)
    if rng.random() < 0.5:
        k, n = (k + 31) // 32 * 32, (n + 31) // 32 * 32
    if rng.random() < 0.3 and k <= 1600 and n <= 1600:
        k, n = n, k
    tokens = _log_int(rng, 1, 8192) if kind == "linear" else _log_int(rng, 32, 4096)
    return {"kind": kind, "fmt": fmt, "tokens": tokens, "k": k, "n": n}


# ---- inputs -----------------------------------------------------------------------------------------------------


def _sizes(case):
    """Numbers of elements of the tensors of an AdamW case: per layer two norms (gain and bias) and four biases, the last
    norm, and the embedding where there is one."""
    d = case["width"]
    sizes = [d, d, d, d, 3 * d, d, 4 * d, d] * case["layers"] + [d, d]
    return ([case["rows"] * d] if case["rows"] else []) + sizes


def _views(flat, sizes, packed):
    """The tensors as parts of one buffer: back to back, or each starting at a multiple of 256 elements."""
    out, at = [], 0
    for n in sizes:
        out.append(flat[at:at + n])
        at += n if packed else (n + 255) // 256 * 256
    return out


def _blocks(n):
    return (n + QBLOCK - 1) // QBLOCK


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    s = {"case": dict(case), "seed": int(seed)}
    if case["kind"] == "adamw":
        sizes = _sizes(case)
        total = sum(sizes if case["packed"] else [(n + 255) // 256 * 256 for n in sizes])
        p = (0.05 * randn(total)).to(TORCH[case["p"]])
        # gradients of one layer's width differ in size from column to column; the embedding rows of tokens that the batch
        # does not hold have none
        spread = torch.exp(randn(case["width"])).repeat(total // case["width"] + 1)[:total]
        grad = 1e-3 * spread * randn(total)
        if case["rows"]:
            seen = torch.rand(case["rows"], generator=g, device="cuda") < 0.3
            grad[:sizes[0]] *= seen.repeat_interleave(case["width"])
        root = 1e-3 * spread * (0.5 + torch.rand(total, generator=g, device="cuda"))
        m = 0.3 * root * randn(total)
        if case["step"] == 1:
            root, m = torch.zeros_like(root), torch.zeros_like(m)
        s.update(sizes=sizes, p=p, grad=grad.to(TORCH[case["g"]]), t=case["step"] - 1,
                 step=torch.full((1,), case["step"] - 1, dtype=torch.int64, device="cuda"))
        if case["bits"] == 32:
            s.update(m=m, v=root * root)
        else:
            # the state of a run that is under way, as an earlier step left it
            nb = [_blocks(n) for n in sizes]
            s.update(m=torch.empty(total, dtype=torch.float8_e4m3fn, device="cuda"), v=torch.empty(total, dtype=torch.float8_e4m3fn, device="cuda"),
                     ms=torch.empty(sum(nb), device="cuda"), vs=torch.empty(sum(nb), device="cuda"))
            for x, q, sc in ((m, s["m"], s["ms"]), (root, s["v"], s["vs"])):
                q.copy_(torch.zeros_like(x).to(torch.float8_e4m3fn))
                at = 0
                for xv, qv, n in zip(_views(x, sizes, case["packed"]), _views(q, sizes, case["packed"]), nb):
                    y = torch.nn.functional.pad(xv, (0, n * QBLOCK - xv.numel())).view(n, QBLOCK)
                    big = y.abs().amax(1)
                    inv = torch.where(big > 0, 448.0 / big, torch.zeros_like(big))
                    qv.copy_((y * inv[:, None]).clamp(-448, 448).reshape(-1)[:xv.numel()].to(torch.float8_e4m3fn))
                    sc[at:at + n] = big / 448.0
                    at += n
            s["nb"] = nb
        if case["copy"]:
            s["copy"] = p.to(torch.bfloat16)
        return s
    if case["kind"] == "quantize":
        # matrices with rows of different size and a few large columns, as activations have
        x = randn(case["b"], case["rows"], case["cols"]) * torch.exp(0.7 * randn(case["b"], case["rows"], 1))
        x = x * (1.0 + 20.0 * (torch.rand(1, 1, case["cols"], generator=g, device="cuda") < 0.01))
        s["x"] = x.to(TORCH[case["dtype"]])
        return s
    t, k, n = case["tokens"], case["k"], case["n"]
    s["x"] = (randn(1, t, k) * (1.0 + 20.0 * (torch.rand(1, 1, k, generator=g, device="cuda") < 0.01))).to(torch.bfloat16)
    w = (randn(1, n, k) / math.sqrt(k)).to(torch.bfloat16)
    if case["kind"] == "linear":
        s["codes"], s["scales"], s["scale"] = _pack(*_quantize(w, case["fmt"]), case["fmt"])
    else:
        s["w"], s["dy"] = w, (1e-3 * randn(1, t, n)).to(torch.bfloat16)
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------


def _pow2(e):
    """2^e to the bit in 32 bits, -127 <= e <= 127 (the GPU's pow may be a unit off)."""
    return torch.where(e > -127, (e.int() + 127) << 23, torch.full_like(e, 1 << 22, dtype=torch.int32)).view(torch.float32)


def _quantize(x, fmt):
    """(magnitude index 0..7 with the sign in bit 3, scale byte, scale value, the matrices' scale) of x [b, rows, cols]: the
    blocks run along the last dimension, padded with zeros to a multiple of 32."""
    x = x.float()
    b, rows, cols = x.shape
    width = (cols + 31) // 32 * 32
    y = torch.nn.functional.pad(x, (0, width - cols)).view(b, rows, width // BLOCK[fmt], BLOCK[fmt])
    big = y.abs().amax(-1)
    whole = torch.ones(b, device=x.device)
    if fmt == "mxfp4":
        frac, e = torch.frexp(big)
        e = torch.where(big > 0, e - torch.where(frac <= 0.75, 3, 2), torch.full_like(e, -127)).clamp(min=-127)
        byte = (e + 127).to(torch.uint8)
        y = y * _pow2(-e)[..., None]
        value = _pow2(e)
    else:
        top = big.amax((1, 2))
        frac, e = torch.frexp(top)
        e = torch.where(top > 0, e - torch.where(frac <= 2688.0 / 4096.0, 12, 11), torch.zeros_like(e)).clamp(min=-126)
        whole = _pow2(e)
        # (a quotient, not a product with 1/6: large values often make it an exact tie of e4m3)
        s8 = torch.div(big * _pow2(-e)[:, None, None], torch.full_like(big, 6.0)).to(torch.float8_e4m3fn)
        byte = s8.view(torch.uint8)
        s = s8.float()[..., None]
        y = torch.where(s > 0, y * _pow2(-e)[:, None, None, None] / s, torch.zeros_like(y))
        value = s8.float() * whole[:, None, None]
    a = y.abs()
    index = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = (index + 8 * (y < 0).int()).view(b, rows, width)
    return code.to(torch.uint8), byte, value, whole


def _values(code, value, fmt, cols):
    """What the codes stand for, in 32 bits."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    v = grid[(code & 7).long()] * (1.0 - 2.0 * (code >> 3).float())
    return (v.view(*value.shape, BLOCK[fmt]) * value[..., None]).view(code.shape)[..., :cols]


def _pack(code, byte, value, whole, fmt):
    """Two codes a byte, and the scale bytes in their tiles."""
    b, rows, nb = byte.shape
    rt, ct = (rows + 127) // 128, (nb + 3) // 4
    full = torch.nn.functional.pad(byte, (0, ct * 4 - nb, 0, rt * 128 - rows))
    tiles = full.view(b, rt, 4, 32, ct, 4).permute(0, 1, 4, 3, 2, 5).contiguous().view(b, rt, ct, 512)
    return code[..., 0::2] | (code[..., 1::2] << 4), tiles, whole


def _unpack(codes, tiles, whole, fmt, rows, cols):
    """The values of packed codes and tiled scales, in 32 bits."""
    b, rt, ct, _ = tiles.shape
    code = torch.stack([codes & 15, codes >> 4], -1).view(b, rows, -1)
    byte = tiles.view(b, rt, ct, 32, 4, 4).permute(0, 1, 4, 3, 2, 5).reshape(b, rt * 128, ct * 4)[:, :rows, :code.shape[-1] // BLOCK[fmt]]
    value = _pow2(byte.int() - 127) if fmt == "mxfp4" else byte.contiguous().view(torch.float8_e4m3fn).float() * whole[:, None, None]
    return _values(code, value, fmt, cols)


def _fake(x, fmt):
    """x rounded to the format and back, blocks along the last dimension."""
    code, byte, value, whole = _quantize(x, fmt)
    return _values(code, value, fmt, x.shape[-1])


def _mix(x):
    """The 64-bit mixing function of the library's generator, in wrapping arithmetic. (The random bits are inputs: `exact` takes them too.)"""
    x = x + -7046029254386353131
    x = (x ^ ((x >> 30) & 0x3FFFFFFFF)) * -4658895280553007687
    x = (x ^ ((x >> 27) & 0x1FFFFFFFFF)) * -7723592293110705685
    return x ^ ((x >> 31) & 0x1FFFFFFFF)


def _random(seed, step, tensor, n, device):
    """Two arrays of 16 random bits for the n elements of tensor number `tensor` at this step (a [1] tensor)."""
    key = _mix(_mix(_mix(torch.full((1,), seed, dtype=torch.int64, device=device)) ^ step) ^ tensor)
    word = _mix(key ^ torch.arange((n + 1) // 2, dtype=torch.int64, device=device))
    word = torch.stack([word & 0xFFFFFFFF, (word >> 32) & 0xFFFFFFFF], -1).view(-1)[:n]
    return word & 0xFFFF, word >> 16


def _e4m3_stochastic(y, bits):
    """y >= 0 in 32 bits, at most 448, rounded to a neighbouring e4m3 value by 16 random bits."""
    y = y.clamp(max=448.0)
    low = y < 2.0 ** -6
    z = torch.where(low, y + 2.0 ** -6, y)
    z = ((z.view(torch.int32) + (bits.int() << 4)) & ~0xFFFFF).view(torch.float32)
    return torch.where(low, z - 2.0 ** -6, z)


def _store8(x, bits, q, scale, keep):
    """Stores x in 8 bits with a scale per block; `keep`: what is not zero does not become zero (the root of v)."""
    n, nb = x.numel(), scale.numel()
    y = torch.nn.functional.pad(x, (0, nb * QBLOCK - n)).view(nb, QBLOCK)
    big = y.abs().amax(1)
    top = torch.full_like(big, 448.0)
    inv = torch.where(big > 2.0 ** -100, torch.div(top, big), torch.zeros_like(big))
    scale.copy_(torch.where(big > 2.0 ** -100, torch.div(big, top), torch.zeros_like(big)))
    y = (y.abs() * inv[:, None]).view(-1)[:n]
    z = _e4m3_stochastic(y, bits)
    if keep:
        z = torch.where((x > 0) & (y > 0), z.clamp(min=2.0 ** -9), z)
    q.copy_(torch.where(x < 0, -z, z).to(torch.float8_e4m3fn))


def _adamw(s):
    case = s["case"]
    c, step = None, None
    if case["clip"]:
        used = [v.float() for v in _views(s["grad"], s["sizes"], case["packed"])]
        norm = torch.stack([torch.sum(v.double() ** 2) for v in used]).sum().sqrt()
        c = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0).float()
        s["step"] += 1
        step = s["step"]
        s["norm"] = norm.float().view(1)
    else:
        s["t"] += 1
        step = torch.full((1,), s["t"], dtype=torch.int64, device="cuda")
    t = step.double()
    size = (LR / (1.0 - BETA1 ** t)).float()
    rc2 = (1.0 / torch.sqrt(1.0 - BETA2 ** t)).float()
    at = 0
    for i, n in enumerate(s["sizes"]):
        where = slice(s["offsets"][i], s["offsets"][i] + n)
        g = s["grad"][where].float()
        if c is not None:
            g = g * c
        if case["bits"] == 32:
            m, v = s["m"][where], s["v"][where]
        else:
            nb = s["nb"][i]
            ms, vs = s["ms"][at:at + nb], s["vs"][at:at + nb]
            m = s["m"][where].float() * ms.repeat_interleave(QBLOCK)[:n]
            v = (s["v"][where].float() * vs.repeat_interleave(QBLOCK)[:n]) ** 2
        m = BETA1 * m + (1.0 - BETA1) * g
        v = BETA2 * v + (1.0 - BETA2) * (g * g)
        root = torch.sqrt(v)
        p = s["p"][where].float() * (1.0 - LR * DECAY) - size * (m / (root * rc2 + EPS))
        low, high = _random(s["seed"], step, i, n, "cuda") if case["bits"] == 8 else (None, None)
        if case["p"] == "bf16" and case["bits"] == 8:
            # bf16 weights round stochastically too, by the same 16 bits as the root of v
            s["p"][where] = ((p.view(torch.int32) + high.int()) & ~0xFFFF).view(torch.float32).to(torch.bfloat16)
        else:
            s["p"][where] = p.to(s["p"].dtype)
        if case["copy"]:
            s["copy"][where] = p.to(torch.bfloat16)
        if case["bits"] == 32:
            s["m"][where], s["v"][where] = m, v
        else:
            _store8(m, low, s["m"][where], ms, False)
            _store8(root, high, s["v"][where], vs, True)
            at += nb
    return _adamw_out(s)


def _adamw_out(s):
    out = {"p": s["p"], "m": s["m"], "v": s["v"]}
    for name in ("ms", "vs", "copy", "norm"):
        if name in s:
            out[name] = s[name]
    return out


def _offsets(case, sizes):
    out, at = [], 0
    for n in sizes:
        out.append(at)
        at += n if case["packed"] else (n + 255) // 256 * 256
    return out


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "adamw":
        if "offsets" not in s:
            s["offsets"] = _offsets(case, s["sizes"])
        return _adamw(s)
    fmt = case["fmt"]
    if kind == "quantize":
        x = s["x"]
        return {"rows": _fake(x, fmt).to(torch.bfloat16), "cols": _fake(x.transpose(1, 2), fmt).to(torch.bfloat16)}
    if kind == "linear":
        w = _unpack(s["codes"], s["scales"], s["scale"], fmt, case["n"], case["k"])
        return torch.matmul(_fake(s["x"], fmt), w.transpose(1, 2)).to(torch.bfloat16)
    x, w, dy = s["x"], s["w"], s["dy"]
    t = lambda a: a.transpose(1, 2)  # noqa: E731
    y = torch.matmul(_fake(x, fmt), t(_fake(w, fmt)))
    dx = torch.matmul(_fake(dy, fmt), t(_fake(t(w), fmt)))
    dw = torch.matmul(_fake(t(dy), fmt), t(_fake(t(x), fmt)))
    return {"y": y.to(torch.bfloat16), "dx": dx.to(torch.bfloat16), "dw": dw}


# ---- the framework's calls ---------------------------------------------------------------------------------------


def _own(s):
    case, ctx, binding = s["case"], _ctx(), _binding()
    kind = case["kind"]
    if kind == "adamw":
        if "group" not in s:
            # what a program makes once of its parameters and moments; the gradients come anew with every step
            part = lambda x: _views(x, s["sizes"], case["packed"]) if x is not None else None  # noqa: E731
            ms = list(torch.split(s["ms"], s["nb"])) if case["bits"] == 8 else None
            vs = list(torch.split(s["vs"], s["nb"])) if case["bits"] == 8 else None
            s["group"] = binding.AdamWGroup(part(s["p"]), part(s["m"]), part(s["v"]), ms, vs, copies=part(s.get("copy")))
            s["grads"] = part(s["grad"])
            s["clip"] = torch.zeros(2, device="cuda")
            s["norm"] = s["clip"][:1]
            if not case["clip"]:
                del s["norm"]
        kw = dict(betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY, stochastic=case["bits"] == 8, seed=s["seed"])
        if case["clip"]:
            ctx.defl_grad_norm(s["grads"], MAX_NORM, out=s["clip"], step=s["step"])
            ctx.defl_adamw_step(s["group"], s["grads"], LR, step=s["step"], grad_scale=s["clip"], **kw)
        else:
            s["t"] += 1
            ctx.defl_adamw_step(s["group"], s["grads"], LR, step=s["t"], **kw)
        return _adamw_out(s)
    fmt = case["fmt"]
    if kind == "quantize":
        q, qt = ctx.defl_mx4_quantize(s["x"], fmt, both=True)
        return {"rows": ctx.defl_mx4_dequantize(q), "cols": ctx.defl_mx4_dequantize(qt)}
    if kind == "linear":
        w = binding.Mx4(s["codes"], s["scales"], s["scale"], fmt, case["n"], case["k"])
        return ctx.defl_mx4_gemm(ctx.defl_mx4_quantize(s["x"], fmt), w)
    x, xt = ctx.defl_mx4_quantize(s["x"], fmt, both=True)
    w, wt = ctx.defl_mx4_quantize(s["w"], fmt, both=True)
    y = ctx.defl_mx4_gemm(x, w)
    dy, dyt = ctx.defl_mx4_quantize(s["dy"], fmt, both=True)
    return {"y": y, "dx": ctx.defl_mx4_gemm(dy, wt), "dw": ctx.defl_mx4_gemm(dyt, xt, out_dtype=torch.float32)}


def run(s):
    return _own(s) if own else _plain(s)


# ---- what a pass cannot do without --------------------------------------------------------------------------------


def work(case):
    if case["kind"] == "adamw":
        n = sum(_sizes(case))
        es = {"bf16": 2, "fp32": 4}
        state = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / QBLOCK
        each = 2 * es[case["p"]] + es[case["g"]] + state + (2 if case["copy"] else 0)
        return {"bytes": n * each, "flops": n * (18 if case["clip"] else 15)}
    held = 0.5 + 1.0 / BLOCK[case["fmt"]]
    if case["kind"] == "quantize":
        n = case["b"] * case["rows"] * case["cols"]
        # codes and scales of both directions are written, then read to be returned as values
        return {"bytes": n * ((2 if case["dtype"] == "bf16" else 4) + 4 * held + 4), "flops": 8 * n}
    t, k, n = case["tokens"], case["k"], case["n"]
    if case["kind"] == "linear":
        return {"bytes": 2 * t * k + held * n * k + 2 * t * n, "flops": 2.0 * t * k * n}
    return {"bytes": 2 * (t * k + n * k + t * n) + 2 * (t * n + t * k) + 4 * n * k, "flops": 6.0 * t * k * n}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------


def _pow2_64(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _round_e2m1_64(y):
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=y.device)
    a = y.abs().contiguous()
    hi = torch.searchsorted(grid, a).clamp(max=7)          # the first value that is not below
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - a, a - grid[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    pick = torch.where(grid[hi] <= a, hi, pick)
    return grid[pick] * torch.sign(y)


def _e4m3_near_64(x):
    """x >= 0 to the nearest e4m3 value, ties to even."""
    e = torch.floor(torch.log2(torch.clamp(x, min=2.0 ** -6)))
    e = torch.where(_pow2_64(e + 1) <= x, e + 1, e)
    step = _pow2_64(e - 3)
    return torch.clamp(torch.round(x / step) * step, max=448.0)


def _fake_64(x, fmt):
    x = x.double()
    b, rows, cols = x.shape
    width = (cols + 31) // 32 * 32
    y = torch.zeros(b, rows, width, dtype=torch.float64, device=x.device)
    y[..., :cols] = x
    y = y.view(b, rows, width // BLOCK[fmt], BLOCK[fmt])
    big = y.abs().amax(-1, keepdim=True)
    if fmt == "mxfp4":
        e = torch.ceil(torch.log2(torch.where(big > 0, big, torch.ones_like(big)) / 6.0))
        e = torch.where(big > 6.0 * _pow2_64(e), e + 1, e)
        e = torch.where(big <= 6.0 * _pow2_64(e - 1), e - 1, e)
        scale = _pow2_64(torch.clamp(e, min=-127))
    else:
        top = big.amax((1, 2, 3), keepdim=True)
        e = torch.ceil(torch.log2(torch.where(top > 0, top, torch.full_like(top, 2688.0)) / 2688.0))
        e = torch.where(top > 2688.0 * _pow2_64(e), e + 1, e)
        e = torch.where(top <= 2688.0 * _pow2_64(e - 1), e - 1, e)
        whole = torch.where(top > 0, _pow2_64(torch.clamp(e, min=-126)), torch.ones_like(e))
        scale = _e4m3_near_64(big / whole / 6.0) * whole
    q = _round_e2m1_64(torch.where(scale > 0, y / torch.where(scale > 0, scale, torch.ones_like(scale)), torch.zeros_like(y))) * scale
    return q.view(b, rows, width)[..., :cols]


def _store_64(x, bits, nb, keep):
    n = x.numel()
    y = torch.zeros(nb * QBLOCK, dtype=torch.float64, device=x.device)
    y[:n] = x.abs()
    big = y.view(nb, QBLOCK).amax(1)
    some = big > 2.0 ** -100
    y = (y.view(nb, QBLOCK) * torch.where(some, 448.0 / torch.where(some, big, torch.ones_like(big)), torch.zeros_like(big))[:, None]).view(-1)[:n]
    e = torch.frexp(torch.clamp(y, min=2.0 ** -6))[1] - 1
    step = _pow2_64(e - 3)
    z = torch.clamp(torch.floor(y / step + bits.double() / 65536.0) * step, max=448.0)
    if keep:
        z = torch.where(y > 0, torch.clamp(z, min=2.0 ** -9), z)
    return torch.sign(x) * z, torch.where(some, big / 448.0, torch.zeros_like(big))


def _adamw_64(s):
    case, sizes = s["case"], s["sizes"]
    grad = s["grad"].double()
    c, out = 1.0, {}
    offsets = _offsets(case, sizes)
    if case["clip"]:
        total = sum(float((grad[o:o + n] ** 2).sum()) for o, n in zip(offsets, sizes))
        out["norm"] = torch.tensor([math.sqrt(total)], dtype=torch.float64)
        c = min(1.0, MAX_NORM / (math.sqrt(total) + 1e-6))
    t = case["step"]
    p, m8, v8 = s["p"].double(), s["m"].double(), s["v"].double()
    pn, mn, vn = p.clone(), m8.clone(), v8.clone()
    msn, vsn = [], []
    at = 0
    for i, (o, n) in enumerate(zip(offsets, sizes)):
        w = slice(o, o + n)
        g = grad[w] * c
        if case["bits"] == 32:
            m, v = m8[w], v8[w]
        else:
            nb = _blocks(n)
            m = m8[w] * s["ms"][at:at + nb].double().repeat_interleave(QBLOCK)[:n]
            v = (v8[w] * s["vs"][at:at + nb].double().repeat_interleave(QBLOCK)[:n]) ** 2
            at += nb
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g * g
        pn[w] = p[w] - LR * DECAY * p[w] - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
        if case["bits"] == 32:
            mn[w], vn[w] = m, v
            continue
        low, high = _random(s["seed"], torch.full((1,), t, dtype=torch.int64, device="cuda"), i, n, "cuda")
        mn[w], a = _store_64(m, low, _blocks(n), False)
        vn[w], b = _store_64(torch.sqrt(v), high, _blocks(n), True)
        msn.append(a)
        vsn.append(b)
        if case["p"] == "bf16":
            e = torch.frexp(torch.clamp(pn[w].abs(), min=2.0 ** -126))[1] - 1
            step = _pow2_64(e - 7)
            pn[w] = torch.sign(pn[w]) * torch.floor(pn[w].abs() / step + high.double() / 65536.0) * step
    out.update(p=pn, m=mn, v=vn)
    if case["bits"] == 8:
        out.update(ms=torch.cat(msn), vs=torch.cat(vsn))
    if case["copy"]:
        out["copy"] = pn
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adamw":
        return _adamw_64(s)
    fmt = case["fmt"]
    t = lambda a: a.transpose(1, 2)  # noqa: E731
    if case["kind"] == "quantize":
        return {"rows": _fake_64(s["x"], fmt), "cols": _fake_64(t(s["x"]), fmt)}
    if case["kind"] == "linear":
        grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], dtype=torch.float64, device="cuda")
        codes, tiles = s["codes"][0].long(), s["scales"][0].long()
        n, k, blk = case["n"], case["k"], BLOCK[fmt]
        row = torch.arange(n, device="cuda")[:, None]
        col = torch.arange(k, device="cuda")[None, :]
        code = torch.where(col % 2 == 0, codes[row, col // 2] & 15, codes[row, col // 2] >> 4)
        at = col // blk
        byte = tiles[row // 128, at // 4, (row % 32) * 16 + (row % 128) // 32 * 4 + at % 4]
        if fmt == "mxfp4":
            scale = _pow2_64(byte - 127)
        else:
            e, f = byte >> 3, (byte & 7).double()
            scale = torch.where(e > 0, _pow2_64(e - 7) * (1 + f / 8), 2.0 ** -6 * f / 8) * float(s["scale"][0])
        w = grid[code] * scale
        return torch.matmul(_fake_64(s["x"], fmt)[0], w.t())[None]
    x, w, dy = s["x"], s["w"], s["dy"]
    return {"y": torch.matmul(_fake_64(x, fmt), t(_fake_64(w, fmt))), "dx": torch.matmul(_fake_64(dy, fmt), t(_fake_64(t(w), fmt))),
            "dw": torch.matmul(_fake_64(t(dy), fmt), t(_fake_64(t(x), fmt)))}
