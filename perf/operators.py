"""Timed cases of the 4-bit operators and of the orthogonalised update, with their plain forms.

Every operator is computed in two ways: in elementary torch operations in 32 bits (``own`` false) and by the calls a
user makes of ``paper_2101_10761_b200.binding`` (``own`` true).  ``prepare`` gives both the same inputs.

Format of a 4-bit matrix (``quantize``, ``matmul``): blocks of 32 neighbours along a row; a block's 32 E2M1 codes are
16 bytes (element 2i in the low half of byte i), a row of codes is 16 * ceil(cols / 32) bytes; its scale is one E8M0
byte.  The scale of (row r, block j) lies at ((r/128) * ceil(nb/4) + j/4) * 512 + (r%32) * 16 + (r%128/32) * 4 + j%4.
A flat 4-bit vector (``compress``, ``mean``) is 16 bytes and one scale byte per block, in order.
"""
import math
import random

import torch

own = False

A, B, C, EPS = 3.4445, -4.7750, 2.0315, 1e-7
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
BITS = 17 / 32                        # bytes of an element and its share of the scale


def _conv(cin, cout, n=1):
    return [(cout, 9 * cin)] * n


# Weight matrices of three models: every convolution as (channels out, 9 * channels in), classifiers, LSTM gates,
# embedding and output projection.
MODELS = {
    "resnet20": _conv(3, 16) + _conv(16, 16, 6) + _conv(16, 32) + _conv(32, 32, 5) + _conv(32, 64) + _conv(64, 64, 5)
    + [(10, 64)],
    "vgg16": _conv(3, 64) + _conv(64, 64) + _conv(64, 128) + _conv(128, 128) + _conv(128, 256) + _conv(256, 256, 2)
    + _conv(256, 512) + _conv(512, 512, 5) + [(10, 512)],
    "lstm-ptb": [(10000, 1500)] + [(6000, 1500)] * 4 + [(10000, 1500)],
}


def listed():
    return [
        # activations of a step (20 sequences of 35 tokens, hidden size 1500): both forms, for forward and backward
        {"name": "quantize 700x1500", "op": "quantize", "rows": 700, "cols": 1500, "type": "bf16"},
        # the largest weight of the LSTM language model, quantised from its fp32 master copy
        {"name": "quantize 10000x1500", "op": "quantize", "rows": 10000, "cols": 1500, "type": "fp32"},
        # one token through the LSTM's gate matrix: latency and weight bandwidth
        {"name": "matmul 1x6000x1500", "op": "matmul", "m": 1, "n": 6000, "k": 1500, "type": "bf16", "add": False},
        # weight gradient of a gate matrix over 700 tokens, added to the fp32 gradient (odd k: 700 = 21.9 blocks)
        {"name": "matmul 6000x1500x700 add", "op": "matmul", "m": 6000, "n": 1500, "k": 700, "type": "fp32",
         "add": True},
        # a large product, bound by the tensor cores
        {"name": "matmul 8192^3", "op": "matmul", "m": 8192, "n": 8192, "k": 8192, "type": "bf16", "add": False},
        # whole-model gradients, error-compensated: a small model, and a ResNet-50 with bf16 gradients
        {"name": "compress 269722", "op": "compress", "d": 269722, "type": "fp32"},
        {"name": "compress 25557032 bf16", "op": "compress", "d": 25557032, "type": "bf16"},
        # mean of the gathered gradients of 8 workers (ResNet-50) and of 2 (ResNet-20)
        {"name": "mean 2x269722", "op": "mean", "d": 269722, "workers": 2},
        {"name": "mean 8x25557032", "op": "mean", "d": 25557032, "workers": 8},
        # the orthogonalised update of whole models: twenty small matrices (latency), medium ones, large ones
        {"name": "orthogonalize resnet20", "op": "orthogonalize", "model": "resnet20", "mats": "", "nesterov": True,
         "type": "fp32"},
        {"name": "orthogonalize vgg16", "op": "orthogonalize", "model": "vgg16", "mats": "", "nesterov": False,
         "type": "fp32"},
        {"name": "orthogonalize lstm-ptb", "op": "orthogonalize", "model": "lstm-ptb", "mats": "", "nesterov": True,
         "type": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "matmul", "compress", "mean", "orthogonalize"])
    if op == "quantize":
        rows = _log(rng, 1, 16384)
        return {"op": op, "rows": rows, "cols": _log(rng, 8, min(8192, 3e7 / rows)), "type": rng.choice(list(TYPES))}
    if op == "matmul":
        return {"op": op, "m": _log(rng, 1, 8192), "n": _log(rng, 16, 8192), "k": _log(rng, 32, 8192),
                "type": rng.choice(list(TYPES)), "add": rng.random() < 0.3}
    if op == "compress":
        return {"op": op, "d": _log(rng, 1000, 66034000), "type": rng.choice(list(TYPES))}
    if op == "mean":
        workers = rng.randint(1, 16)
        return {"op": op, "d": _log(rng, 1000, 2e8 / workers), "workers": workers}
    shapes, left = [], 2e7
    for _ in range(rng.randint(1, 8)):
        s = _log(rng, 8, 1600)
        r, c = s, min(8192, int(s * math.exp(rng.uniform(0, 2.5))))
        if r * c > left:
            break
        left -= r * c
        shapes += [(c, r) if rng.random() < 0.5 else (r, c)] * rng.randint(1, max(1, min(4, int(left / (r * c)))))
        left -= r * c * shapes.count(shapes[-1])
    shapes = shapes or [(rng.randint(8, 1000), 257)]
    return {"op": op, "model": "", "mats": " ".join("%dx%d" % x for x in shapes), "nesterov": rng.random() < 0.5,
            "type": rng.choice(list(TYPES))}


# ---------------------------------------------------------------------------------------------- plain pieces


def _layout(rows, nb, device):
    """Where the scale byte of every (row, block) lies."""
    r = torch.arange(rows, device=device)[:, None]
    j = torch.arange(nb, device=device)[None, :]
    return (r // 128 * -(-nb // 4) + j // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + j % 4


def _blocks(x):
    """[rows, cols] as [rows, blocks, 32] in 32 bits, the last block filled with zeros."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    return torch.nn.functional.pad(x.float(), (0, nb * 32 - cols)).view(rows, nb, 32)


def _quantize(blocks):
    """(magnitudes on the E2M1 grid with their signs, exponents of the scales) of [..., 32]."""
    top = blocks.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top)[1] - 3, -127).clamp(-127, 125)
    t = torch.ldexp(blocks.abs(), -e)
    step = torch.where(t < 2, 0.5, torch.where(t < 4, 1.0, 2.0))
    return torch.copysign((torch.round(t / step) * step).clamp(max=6.0), blocks), e


def _pack(q):
    """Codes of values on the grid, two to a byte."""
    m = q.abs()
    code = torch.where(m < 2, m * 2, torch.where(m < 4, m + 2, m / 2 + 4)).to(torch.uint8)
    code = code | (torch.signbit(q).to(torch.uint8) << 3)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).contiguous()


def _unpack(codes):
    """Values on the grid, in 32 bits, of packed codes [..., n] -> [..., 2 n]."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    return table[c.int()]


def _decode_matrix(codes, scales, rows, cols, dtype=torch.float32):
    nb = codes.shape[1] // 16
    e = scales[_layout(rows, nb, codes.device)].to(dtype) - 127
    return (_unpack(codes).to(dtype).view(rows, nb, 32) * torch.exp2(e)[..., None]).view(rows, nb * 32)[:, :cols]


def _encode_matrix(x):
    """(codes, scales) of a matrix in the layouts above."""
    q, e = _quantize(_blocks(x))
    rows, nb = q.shape[:2]
    scales = torch.zeros(-(-rows // 128) * -(-nb // 4) * 512, dtype=torch.uint8, device=x.device)
    scales[_layout(rows, nb, x.device)] = (e[..., 0] + 127).to(torch.uint8)
    return _pack(q).view(rows, nb * 16), scales


def _shapes(case):
    if case["model"]:
        return MODELS[case["model"]]
    return [tuple(int(v) for v in m.split("x")) for m in case["mats"].split()]


def _offsets(shapes):
    """Element offsets of the matrices in the flat vector; each is followed by a vector of one value per row."""
    off, at = [], 0
    for r, c in shapes:
        off.append(at)
        at += r * c + r
    return off, at


def _laplace(n, scale, g):
    u = torch.rand(n, generator=g, device="cuda") - 0.5
    return -scale * torch.sign(u) * torch.log1p(-2 * u.abs().clamp(max=0.49999997))


# ---------------------------------------------------------------------------------------------- the contract


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": case}
    if case["op"] == "quantize":
        # rows of different scale, as activations and weights of different units have
        x = torch.randn(case["rows"], case["cols"], generator=g, device="cuda")
        x *= torch.exp(torch.randn(case["rows"], 1, generator=g, device="cuda"))
        s["x"] = x.to(TYPES[case["type"]])
    elif case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        for name, rows, scale in (("a", m, 1.0), ("b", n, k ** -0.5)):
            s[name] = _encode_matrix(torch.randn(rows, k, generator=g, device="cuda") * scale)
        s["c"] = torch.randn(m, n, generator=g, device="cuda").to(TYPES[case["type"]])
    elif case["op"] == "compress":
        s["grad"] = _laplace(case["d"], 1e-3, g).to(TYPES[case["type"]])
        s["residual"] = _laplace(case["d"], 1e-4, g)
    elif case["op"] == "mean":
        nb = -(-case["d"] // 32)
        codes, scales = [], []
        for _ in range(case["workers"]):
            q, e = _quantize(torch.nn.functional.pad(_laplace(case["d"], 1e-3, g), (0, nb * 32 - case["d"])).view(-1, 32))
            codes.append(_pack(q).view(-1))
            scales.append((e[:, 0] + 127).to(torch.uint8))
        s["codes"], s["scales"] = torch.cat(codes), torch.cat(scales)
    else:
        shapes = _shapes(case)
        s["offsets"], d = _offsets(shapes)
        grad = _laplace(d, 1e-3, g)
        for (r, c), o in zip(shapes, s["offsets"]):     # a few strong directions over the noise
            k = min(8, r, c)
            left, right = (torch.randn(n, k, generator=g, device="cuda") for n in (r, c))
            left *= 1e-3 * torch.exp2(-torch.arange(k, device="cuda", dtype=torch.float32))
            grad[o:o + r * c] += (left @ right.T).view(-1)
        s["grad"] = grad.to(TYPES[case["type"]])
        s["momentum"] = _laplace(d, 1e-3, g)
        s["rows"], s["cols"] = [r for r, _ in shapes], [c for _, c in shapes]
        s["out"] = torch.zeros(d, dtype=torch.bfloat16, device="cuda")
    return s


def _plain_orthogonalize(s):
    mu, case = 0.95, s["case"]
    grad, out = s["grad"].float(), s["out"]
    groups = {}
    for o, r, c in zip(s["offsets"], s["rows"], s["cols"]):
        groups.setdefault((r, c), []).append(o)
    for (r, c), offs in groups.items():
        at = [slice(o, o + r * c) for o in offs]
        mom = torch.stack([s["momentum"][i] for i in at]) * mu + torch.stack([grad[i] for i in at])
        u = torch.stack([grad[i] for i in at]) + mu * mom if case["nesterov"] else mom
        x = u.view(-1, r, c)
        x = x.mT if r > c else x
        x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
        for _ in range(5):
            a = x @ x.mT
            x = A * x + (B * a + C * (a @ a)) @ x
        x = x.mT if r > c else x
        for n, i in enumerate(at):
            s["momentum"][i] = mom[n]
            out[i] = x[n].reshape(-1).to(out.dtype)
    return {"out": out, "momentum": s["momentum"]}


def _plain(s):
    case = s["case"]
    if case["op"] == "quantize":
        def form(x):
            q, e = _quantize(_blocks(x))
            return torch.ldexp(q, e).view(x.shape[0], -1)[:, :x.shape[1]].to(torch.bfloat16)
        return {"rows": form(s["x"]), "cols": form(s["x"].T)}
    if case["op"] == "matmul":
        a = _decode_matrix(*s["a"], case["m"], case["k"])
        b = _decode_matrix(*s["b"], case["n"], case["k"])
        c = a @ b.T
        s["c"].copy_(s["c"].float() + c if case["add"] else c)
        return s["c"]
    if case["op"] == "compress":
        d = case["d"]
        acc = s["grad"].float() + s["residual"]
        q, e = _quantize(torch.nn.functional.pad(acc, (0, -d % 32)).view(-1, 32))
        value = torch.ldexp(q, e).view(-1)[:d]
        s["residual"].copy_(acc - value)
        return {"value": value, "residual": s["residual"]}
    if case["op"] == "mean":
        n = case["workers"]
        e = s["scales"].view(n, -1, 1).float() - 127
        v = _unpack(s["codes"]).view(n, -1, 32) * torch.exp2(e)
        return (v.sum(0) / n).view(-1)[:case["d"]]
    return _plain_orthogonalize(s)


def _kept(s, name, make):
    """A buffer that the caller keeps from one call to the next."""
    if name not in s:
        s[name] = make()
    return s[name]


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def _framework(s):
    from paper_2101_10761_b200 import binding as K
    case = s["case"]
    if case["op"] == "quantize":
        x, (rows, cols) = s["x"], s["x"].shape

        def buffers():
            return ([_bytes(K.sidco_mx4_code_bytes(r, c)) for r, c in ((rows, cols), (cols, rows))]
                    + [_bytes(K.sidco_mx4_scale_bytes(r, c)) for r, c in ((rows, cols), (cols, rows))]
                    + [torch.empty(r, c, dtype=torch.bfloat16, device="cuda") for r, c in ((rows, cols), (cols, rows))])
        codes, codes_t, scales, scales_t, out, out_t = _kept(s, "buffers", buffers)
        K.sidco_mx4_quantize(x, rows, cols, cols, codes, scales, codes_t, scales_t)
        K.sidco_mx4_dequantize(codes, scales, rows, cols, out, cols)
        K.sidco_mx4_dequantize(codes_t, scales_t, cols, rows, out_t, rows)
        return {"rows": out, "cols": out_t}
    if case["op"] == "matmul":
        K.sidco_mx4_matmul(*s["a"], *s["b"], case["m"], case["n"], case["k"], s["c"], case["n"], case["add"])
        return s["c"]
    if case["op"] == "compress":
        d, nb = case["d"], -(-case["d"] // 32)
        codes, scales, value = _kept(s, "buffers", lambda: (
            _bytes(16 * nb), _bytes(nb), torch.empty(d, dtype=torch.float32, device="cuda")))
        K.sidco_mx4_compress(s["grad"], s["residual"], d, codes, scales)
        K.sidco_mx4_mean(codes, scales, 1, d, value)      # of one worker: what the codes stand for
        return {"value": value, "residual": s["residual"]}
    if case["op"] == "mean":
        out = _kept(s, "dense", lambda: torch.empty(case["d"], dtype=torch.float32, device="cuda"))
        K.sidco_mx4_mean(s["codes"], s["scales"], case["workers"], case["d"], out)
        return out
    need = _kept(s, "need", lambda: K.sidco_orthogonalize_workspace_bytes(s["rows"], s["cols"]))
    K.sidco_orthogonalize(s["grad"], s["momentum"], 0.95, case["nesterov"], s["offsets"], s["rows"], s["cols"], 5,
                          s["out"], _kept(s, "workspace", lambda: _bytes(need)), need, eps=EPS)
    return {"out": s["out"], "momentum": s["momentum"]}


def run(state):
    return _framework(state) if own else _plain(state)


def work(case):
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (SIZE[case["type"]] + 2 * (BITS + 2)), "flops": 0}
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * k * BITS + m * n * SIZE[case["type"]] * (2 if case["add"] else 1),
                "flops": 2 * m * n * k}
    if case["op"] == "compress":
        return {"bytes": case["d"] * (SIZE[case["type"]] + 8 + BITS + 4), "flops": 0}
    if case["op"] == "mean":
        return {"bytes": case["d"] * (case["workers"] * BITS + 4), "flops": 0}
    size, flops = 0, 0
    for r, c in _shapes(case):
        s, n = min(r, c), max(r, c)
        size += r * c * (SIZE[case["type"]] + 8 + 2)
        # products of symmetric results at half their cost, the five steps taken as three and two: a Gram product and
        # one application to the matrix for each group, the other products between small symmetric matrices
        flops += 6 * s * s * n + 14 * s ** 3
    return {"bytes": size, "flops": flops}


# ---------------------------------------------------------------------------------------------- in 64 bits


def _grid64(v, dim):
    """The nearest values (ties to the even code) of blocks of 32 along `dim`, in 64 bits, by comparison."""
    v = v.double().movedim(dim, -1)
    n = v.shape[-1]
    full = torch.zeros(*v.shape[:-1], -(-n // 32) * 32, dtype=torch.float64, device=v.device)
    full[..., :n] = v
    full = full.view(*v.shape[:-1], -1, 32)
    peak = full.abs().max(-1, keepdim=True).values
    e = torch.floor(torch.log2(peak.clamp(min=2.0 ** -140)))
    e = e + (peak >= torch.exp2(e + 1)).double() - (peak < torch.exp2(e)).double()      # log2 may round
    unit = torch.exp2((e - 2).clamp(-127, 125))
    t = full.abs() / unit
    q = torch.zeros_like(t)
    # (smallest magnitude that goes there, whether the tie does, the value)
    for edge, tie, value in ((.25, False, .5), (.75, True, 1.), (1.25, False, 1.5), (1.75, True, 2.), (2.5, False, 3.),
                             (3.5, True, 4.), (5., False, 6.)):
        q = torch.where(t >= edge if tie else t > edge, value, q)
    return (torch.sign(full) * q * unit).flatten(-2)[..., :n].movedim(-1, dim)


def _values64(codes, scales, rows, cols):
    """Decoded by arithmetic on the code's bits: sign, two bits of exponent, one of mantissa."""
    pitch = codes.shape[1]
    out = torch.zeros(rows, pitch, 2, dtype=torch.float64, device=codes.device)
    for half in (0, 1):
        c = (codes.long() >> (4 * half)) & 15
        ex, man = (c >> 1) & 3, c & 1
        mag = torch.where(ex == 0, man * 0.5, (1 + 0.5 * man.double()) * 2.0 ** (ex - 1).double())
        out[..., half] = torch.where(c >= 8, -mag, mag)
    nb = pitch // 16
    tiles = scales.view(-(-rows // 128), -(-nb // 4), 32, 4, 4)                # row tile, block tile, r%32, r/32, j%4
    e = tiles.permute(0, 3, 2, 1, 4).reshape(-(-rows // 128) * 128, -1)[:rows, :nb].double() - 127
    return (out.view(rows, nb, 32) * torch.exp2(e)[..., None]).view(rows, -1)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        return {"rows": _grid64(s["x"], 1), "cols": _grid64(s["x"], 0).T.contiguous()}
    if case["op"] == "matmul":
        c = _values64(*s["a"], case["m"], case["k"]) @ _values64(*s["b"], case["n"], case["k"]).T
        return c + s["c"].double() if case["add"] else c
    if case["op"] == "compress":
        acc = (s["grad"].double() + s["residual"].double()).float().double()     # the sum is one addition in 32 bits
        value = _grid64(acc, 0)
        return {"value": value, "residual": acc - value}
    if case["op"] == "mean":
        n, nb = case["workers"], -(-case["d"] // 32)
        total = torch.zeros(case["d"], dtype=torch.float64, device="cuda")
        for w in range(n):
            c = s["codes"].view(n, nb, 16)[w].long()
            c = torch.stack((c % 16, c // 16), -1).view(nb, 32)
            ex, man = c % 8 // 2, (c % 2).double()
            v = torch.where(ex == 0, man / 2, (1 + man / 2) * torch.exp2(ex.double() - 1)) * (1 - 2 * (c // 8)).double()
            total += (v * torch.exp2(s["scales"].view(n, nb)[w].double() - 127)[:, None]).view(-1)[:case["d"]]
        return total / n
    out, moved = torch.zeros(s["out"].numel(), dtype=torch.float64, device="cuda"), s["momentum"].double()
    for o, r, c in zip(s["offsets"], s["rows"], s["cols"]):
        grad = s["grad"][o:o + r * c].double()
        mom = 0.95 * moved[o:o + r * c] + grad
        moved[o:o + r * c] = mom
        x = (grad + 0.95 * mom if case["nesterov"] else mom).view(r, c)
        x = x / (torch.linalg.norm(x) + EPS)
        for _ in range(5):
            if r <= c:
                gram = x @ x.T
                x = A * x + B * (gram @ x) + C * (gram @ (gram @ x))
            else:
                gram = x.T @ x
                x = A * x + B * (x @ gram) + C * ((x @ gram) @ gram)
        out[o:o + r * c] = x.reshape(-1)
    return {"out": out, "momentum": moved}


if __name__ == "__main__":
    for case in listed() + [draw(random.Random(n)) for n in range(6)]:
        print(case, work(case))
