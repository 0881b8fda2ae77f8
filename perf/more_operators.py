"""Performance cases of decoding on 8-bit projections, from the block's norm to the drawn byte.

Kinds, each one pass through one operator of paper_2401_13660_gb300.mbscan:

* norm     mb_rmsnorm_q8: residual add and RMS norm, the output in 8 bits with scales.
* quant    mb_quantize_q8: activations (a scale for 128 elements of a row) or weights (one for 128 x 128).
* matmul   mb_matmul_q8: the product of 8-bit activations and weights.
* sample   mb_sample: temperature, top-k, top-p, min-p and the draw from given random numbers.

8-bit values are e4m3, scales powers of two with the exponent in a byte (0 is 2^-127): the smallest that
keeps a block's largest value within 448. What comes back of 8-bit outputs is the values they stand for.

Sizes are those of the MambaByte models this repository names (d_model 1024, 2304 with d_inner twice that,
[x | z] of twice that again; 256 bytes; 256 streams; 8192-byte spans), with small, ragged and odd ones
around them, and vocabularies of tens of thousands for subword drafters.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 128
SPAN = 65536 * 1024            # elements of the largest normalised span
PRODUCT = 8192 * 2304 * 9216   # multiplications of the largest product
LOGITS = 256 * 32001           # logits of the largest draw


def listed():
    return [
        # One decode step of 256 streams of the widest model: a block's opening.
        dict(name="norm_n256_W2304", kind="norm", n=256, W=2304, add="bf16"),
        # A full-context batch of 8 x 8192 bytes through the 353M-sized model.
        dict(name="norm_n65536_W1024", kind="norm", n=65536, W=1024, add="bf16"),
        # The scan's output of a decode step, before the output projection.
        dict(name="quant_n256_W4608", kind="quant", n=256, W=4608, rows=1, dtype="bf16", wide=False),
        # The widest input projection when a model is loaded.
        dict(name="quant_n9216_W2304_blocks", kind="quant", n=9216, W=2304, rows=128, dtype="bf16", wide=False),
        # One stream of the 353M-sized model: latency, and every weight read for one row.
        dict(name="matmul_n1_K1024_N4096", kind="matmul", n=1, K=1024, N=4096, out="bf16", parts=2),
        # The widest model's decode step of 256 streams: x and z, then the output projection (few columns,
        # a long sum).
        dict(name="matmul_n256_K2304_N9216", kind="matmul", n=256, K=2304, N=9216, out="bf16", parts=2),
        dict(name="matmul_n256_K4608_N2304", kind="matmul", n=256, K=4608, N=2304, out="bf16", parts=1),
        # Ragged in every size, fp32 out.
        dict(name="matmul_f32_n1003_K1552_N2072", kind="matmul", n=1003, K=1552, N=2072, out="f32", parts=1),
        # A full-context prompt through the widest input projection.
        dict(name="matmul_n8192_K2304_N9216", kind="matmul", n=8192, K=2304, N=9216, out="bf16", parts=2),
        # The next bytes of 256 streams, each with its own settings.
        dict(name="sample_n256_V256", kind="sample", n=256, V=256, dtype="bf16", tokens="i64", t=True, k=True, p=True,
             m=True),
        # A subword drafter of few streams, nucleus sampling alone.
        dict(name="sample_f32_n32_V32001", kind="sample", n=32, V=32001, dtype="f32", tokens="i64", t=True, k=False,
             p=True, m=False),
        # The same of many streams, every setting on.
        dict(name="sample_n256_V32001", kind="sample", n=256, V=32001, dtype="bf16", tokens="i32", t=True, k=True,
             p=True, m=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["norm", "quant", "matmul", "matmul", "matmul", "sample", "sample"])
    if kind == "norm":
        W = rng.choice([1024, 1792, 2304, 16 * _log(rng, 1, 288)])
        return dict(kind=kind, n=_log(rng, 1, min(65536, SPAN // W)), W=W, add=rng.choice(["bf16", "bf16", "f32", "none"]))
    if kind == "quant":
        W = rng.choice([1024, 2048, 4608, 16 * _log(rng, 1, 576)])
        return dict(kind=kind, n=_log(rng, 1, min(65536, SPAN // W)), W=W, rows=rng.choice([1, 1, 128]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), wide=rng.random() < 0.3)
    if kind == "matmul":
        K = rng.choice([1024, 1792, 2304, 4608, 16 * _log(rng, 1, 288)])
        parts = rng.choice([1, 1, 2])
        N = rng.choice([1024, 2304, 128 * parts * _log(rng, 1, 36), 8 * _log(rng, 1, 1152)])
        if N % (128 * parts):
            parts = 1
        return dict(kind=kind, n=_log(rng, 1, min(65536, PRODUCT // (K * N), 2 ** 28 // N)), K=K, N=N,
                    out=rng.choice(["bf16", "bf16", "f32"]), parts=parts)
    V = rng.choice([256, 256, _log(rng, 2, 64000)])
    return dict(kind=kind, n=_log(rng, 1, min(32768, LOGITS // V)), V=V, dtype=rng.choice(["f32", "bf16"]),
                tokens=rng.choice(["i32", "i64"]), t=rng.random() < 0.8, k=rng.random() < 0.5, p=rng.random() < 0.6,
                m=rng.random() < 0.4)


# ---------------------------------------------------------------------------
# inputs

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}
E4M3 = torch.float8_e4m3fn


def _stride(width):
    """Bytes between rows of scales: whole 32-bit words."""
    return 4 * -(-width // (4 * BLOCK))


def _inputs(case, seed):
    """Everything random in a case."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind = case["kind"]

    def rnd(*shape):
        return torch.randn(*shape, device=DEV, generator=g)
    if kind == "norm":
        n, W = case["n"], case["W"]
        # a residual stream with a few strong channels
        strong = torch.where(torch.rand(W, device=DEV, generator=g) < 0.01, 8.0, 1.0)
        return dict(residual=rnd(n, W) * strong, w=0.5 + torch.rand(W, device=DEV, generator=g),
                    add=None if case["add"] == "none" else (0.3 * rnd(n, W)).to(TYPES[case["add"]]))
    if kind == "quant":
        n, W = case["n"], case["W"]
        x = rnd(n, (2 if case["wide"] else 1) * W)
        if case["rows"] == 1:
            x *= torch.exp(rnd(n, 1))
        else:
            x *= 1 / math.sqrt(W)
        return dict(x=x.to(TYPES[case["dtype"]])[:, :W])
    if kind == "matmul":
        n, K, N = case["n"], case["K"], case["N"]
        # 8-bit values as quantising leaves them (the largest of a block between 224 and 448), with scales
        # that vary as activations' and weights' do
        a = (rnd(n, K) * 90).clamp(-448, 448).to(E4M3)
        w = (rnd(N, K) * 80).clamp(-448, 448).to(E4M3)
        sa = torch.randint(118, 122, (n, _stride(K)), device=DEV, generator=g).to(torch.uint8)
        sw = torch.randint(114, 117, (-(-N // BLOCK), _stride(K)), device=DEV, generator=g).to(torch.uint8)
        return dict(a=a, w=w, sa=sa, sw=sw)
    n, V = case["n"], case["V"]
    logits = 2.0 * rnd(n, V)
    likely = torch.randint(0, V, (n, 3), device=DEV, generator=g)
    logits.scatter_add_(1, likely, math.log(V) * torch.rand(n, 3, device=DEV, generator=g) * 1.5)
    if V > 8:   # tokens that a grammar forbids
        banned = torch.rand(n, V, device=DEV, generator=g) < 0.02
        logits.masked_fill_(banned.scatter_(1, likely, False), -math.inf)

    def choose(values, dtype):
        return torch.tensor(values, device=DEV, dtype=dtype)[
            torch.randint(0, len(values), (n,), device=DEV, generator=g)]
    return dict(logits=logits.to(TYPES[case["dtype"]]), u=torch.rand(n, device=DEV, generator=g),
                temperature=choose([0.0, 0.6, 0.8, 1.0, 1.0, 1.3], torch.float32) if case["t"] else None,
                top_k=choose([0, 1, 5, 40, 200], torch.int32) if case["k"] else None,
                top_p=choose([0.5, 0.8, 0.9, 0.95, 1.0], torch.float32) if case["p"] else None,
                min_p=choose([0.0, 0.02, 0.1], torch.float32) if case["m"] else None)


# ---------------------------------------------------------------------------
# what a program has before the call, and the call

def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    kind = case["kind"]
    if kind in ("norm", "quant"):
        n, W, rows = case["n"], case["W"], case.get("rows", 1)
        s["q"] = torch.empty(n, W, dtype=E4M3, device=DEV)
        s["scales"] = torch.empty(-(-n // rows), _stride(W), dtype=torch.uint8, device=DEV)
        s["values"] = torch.empty(n, W, dtype=torch.bfloat16, device=DEV)
    elif kind == "matmul":
        parts, N = case["parts"], case["N"]
        shape = (case["n"], N) if parts == 1 else (parts, case["n"], N // parts)
        s["out"] = torch.empty(shape, dtype=TYPES[case["out"]], device=DEV)
        s["ws"] = torch.zeros(256, dtype=torch.uint8, device=DEV)
    else:
        s["token"] = torch.empty(case["n"], dtype=TYPES[case["tokens"]], device=DEV)
        s["prob"] = torch.empty(case["n"], device=DEV)
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2401_13660_gb300 import mbscan as mb
    kind = s["case"]["kind"]
    if kind == "norm":
        mb.mb_rmsnorm_q8(s["residual"], s["w"], s["q"], s["scales"], add=s["add"], eps=1e-5)
        return {"residual": s["residual"], "values": mb.mb_dequantize_q8(s["q"], s["scales"], s["values"])}
    if kind == "quant":
        rows = s["case"]["rows"]
        mb.mb_quantize_q8(s["x"], s["q"], s["scales"], block_rows=rows)
        return {"values": mb.mb_dequantize_q8(s["q"], s["scales"], s["values"], block_rows=rows)}
    if kind == "matmul":
        return {"out": mb.mb_matmul_q8(s["a"], s["sa"], s["w"], s["sw"], s["out"], ws=s["ws"])}
    mb.mb_sample(s["logits"], s["u"], s["token"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                 min_p=s["min_p"], prob=s["prob"])
    return {"token": s["token"], "prob": s["prob"]}


def _blocks(x, rows):
    """x padded with zeros to whole blocks: [row blocks, rows, column blocks, 128]."""
    n, W = x.shape
    x = torch.nn.functional.pad(x, (0, -W % BLOCK, 0, -n % rows))
    return x.view(-1, rows, x.shape[1] // BLOCK, BLOCK)


def _quantized(x, rows):
    """The values that x is rounded to in 8 bits: e4m3 times the block's power of two."""
    b = _blocks(x, rows)
    mantissa, exponent = torch.frexp(b.abs().amax((1, 3), keepdim=True))   # amax = mantissa 2^exponent, 0.5 <= mantissa < 1
    # 448 = 0.875 2^9
    e = (exponent - 9 + (mantissa > 0.875).int()).clamp(-126, 127)
    q = torch.ldexp(b, -e).to(E4M3).float()
    v = torch.ldexp(q, e)
    return v.flatten(2).flatten(0, 1)[:x.shape[0], :x.shape[1]]


def _expand(s, rows, n, K):
    """Scales [row blocks, stride] as factors [n, K]."""
    f = torch.ldexp(torch.ones((), device=DEV), s.int() - 127)
    return f.repeat_interleave(rows, 0)[:n].repeat_interleave(BLOCK, 1)[:, :K]


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        r = s["residual"]
        if s["add"] is not None:
            r += s["add"]
        y = r / torch.sqrt((r * r).mean(1, keepdim=True) + 1e-5) * s["w"]
        return {"residual": r, "values": s["values"].copy_(_quantized(y, 1))}
    if kind == "quant":
        return {"values": s["values"].copy_(_quantized(s["x"].float(), case["rows"]))}
    if kind == "matmul":
        n, K, N = case["n"], case["K"], case["N"]
        a = s["a"].float() * _expand(s["sa"], 1, n, K)
        w = s["w"].float() * _expand(s["sw"], BLOCK, N, K)
        product = a @ w.t()
        if case["parts"] > 1:
            product = product.view(n, case["parts"], -1).transpose(0, 1)
        return {"out": s["out"].copy_(product)}
    # in 64 bits: a draw next to a border, a sum next to top-p
    n, V = case["n"], case["V"]
    l = s["logits"].double()
    t = torch.ones(n, device=DEV) if s["temperature"] is None else s["temperature"]
    greedy = ~(t > 0)
    weight = torch.exp((l - l.amax(1, keepdim=True)) / torch.where(greedy, 1.0, t)[:, None])
    down, order = torch.sort(l, dim=1, descending=True, stable=True)
    ranked = weight.gather(1, order)
    rank = torch.arange(V, device=DEV)
    keep = (down > -math.inf) & (~greedy[:, None] | (rank == 0))
    if s["top_k"] is not None:
        keep &= (rank < s["top_k"][:, None]) | (s["top_k"] <= 0)[:, None]
    if s["top_p"] is not None:
        kept = ranked * keep
        before = torch.nn.functional.pad(kept.cumsum(1), (1, -1))
        keep &= (before < kept.sum(1, keepdim=True) * s["top_p"][:, None]) | (s["top_p"] >= 1)[:, None]
    if s["min_p"] is not None:
        keep &= ranked >= s["min_p"][:, None]
    weight = torch.zeros_like(weight).scatter_(1, order, ranked * keep)
    upto = weight.cumsum(1)
    total = upto[:, -1:]
    token = (upto <= s["u"][:, None] * total).sum(1)
    s["token"].copy_(token)
    s["prob"].copy_(weight.gather(1, token[:, None])[:, 0] / total[:, 0])
    return {"token": s["token"], "prob": s["prob"]}


# ---------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    """Each input read once, each output written once."""
    kind = case["kind"]
    size = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8, "none": 0}
    if kind == "norm":
        n, W = case["n"], case["W"]
        return {"bytes": n * W * (9 if case["add"] != "none" else 5) + n * W * size[case["add"]] + n * _stride(W) + 4 * W,
                "flops": 6 * n * W}
    if kind == "quant":
        n, W = case["n"], case["W"]
        return {"bytes": n * W * (size[case["dtype"]] + 1) + -(-n // case["rows"]) * _stride(W), "flops": 3 * n * W}
    if kind == "matmul":
        n, K, N = case["n"], case["K"], case["N"]
        return {"bytes": (n + N) * K + (n + -(-N // BLOCK)) * _stride(K) + n * N * size[case["out"]], "flops": 2 * n * K * N}
    n, V = case["n"], case["V"]
    return {"bytes": n * V * size[case["dtype"]] + n * (size[case["tokens"]] + 8 + 4 * sum(case[k] for k in "tkpm")),
            "flops": 4 * n * V}


# ---------------------------------------------------------------------------
# the same in 64 bits

def _grid(x, rows):
    """x rounded block by block, 64 bits: to the nearest multiple of the spacing of e4m3 there, ties to even."""
    n, W = x.shape
    v = torch.zeros(-(-n // rows) * rows, -(-W // BLOCK) * BLOCK, device=DEV, dtype=torch.float64)
    v[:n, :W] = x
    v = v.unfold(0, rows, rows).unfold(1, BLOCK, BLOCK)      # [row blocks, column blocks, rows, 128]
    top = v.abs().amax((2, 3), keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, 448.0) / 448.0)).clamp(-126, 127))
    v = v / scale
    spacing = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    v = torch.round(v / spacing) * spacing * scale
    return v.transpose(1, 2).flatten(2).flatten(0, 1)[:n, :W]


def exact(case, seed):
    i = _inputs(case, seed)
    kind = case["kind"]
    if kind == "norm":
        # the residual stream is fp32: the sum is rounded there, and the norm is of what is kept
        r = i["residual"].double()
        if i["add"] is not None:
            r = (r + i["add"].double()).float().double()
        y = r * torch.rsqrt(r.square().sum(1, keepdim=True) / case["W"] + 1e-5) * i["w"].double()
        return {"residual": r, "values": _grid(y, 1)}
    if kind == "quant":
        return {"values": _grid(i["x"].double(), case["rows"])}
    if kind == "matmul":
        n, K, N = case["n"], case["K"], case["N"]
        out = torch.zeros(n, N, device=DEV, dtype=torch.float64)
        a, w = i["a"].double(), i["w"].double()
        for b in range(-(-K // BLOCK)):   # one block of the sum after the other, scaled as a whole
            at = slice(b * BLOCK, min(K, (b + 1) * BLOCK))
            left = a[:, at] * torch.exp2(i["sa"][:, b].double() - 127)[:, None]
            right = w[:, at] * torch.exp2(i["sw"][:, b].double() - 127).repeat_interleave(BLOCK)[:N, None]
            out.addmm_(left, right.t())
        if case["parts"] > 1:
            out = torch.stack(out.chunk(case["parts"], 1))
        return {"out": out}
    # rows one after the other are slow: all at once by sorted logits, thresholds in place of ranks
    n, V = case["n"], case["V"]
    z = i["logits"].double()
    t = torch.ones(n, device=DEV, dtype=torch.float64) if i["temperature"] is None else i["temperature"].double()
    first = z.argmax(1)
    p = torch.softmax(z / torch.where(t > 0, t, 1.0)[:, None], 1)
    p[t <= 0] = 0.0
    p[t <= 0, first[t <= 0]] = 1.0
    position = torch.argsort(z, dim=1, descending=True, stable=True).argsort(1)   # of each token among its row's
    if i["top_k"] is not None:
        p = torch.where((position >= i["top_k"][:, None]) & (i["top_k"] > 0)[:, None], 0.0, p)
    if i["top_p"] is not None:
        p = p / p.sum(1, keepdim=True)
        above = torch.zeros_like(p).scatter_(1, position, p).cumsum(1).gather(1, position) - p   # mass of the likelier
        out = (above >= i["top_p"].double()[:, None]) & (position > 0) & (i["top_p"] < 1)[:, None]
        p = torch.where(out, 0.0, p)
    if i["min_p"] is not None:
        p = torch.where(p < i["min_p"].double()[:, None] * p.amax(1, keepdim=True), 0.0, p)
    p = p / p.sum(1, keepdim=True)
    token = torch.searchsorted(p.cumsum(1), i["u"].double()[:, None], right=True).clamp(max=V - 1)
    return {"token": None, "prob": p.gather(1, token)[:, 0]}
