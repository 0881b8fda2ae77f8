"""Performance cases of the operators that a training step runs around the scan.

Kinds, each one pass through one operator of paper_2401_13660_gb300.mbscan:

* conv        mb_conv1d: the causal convolution (kernel 4) and SiLU over a span.
* conv_grad   mb_conv1d_backward: its gradients.
* embed       mb_embed: byte or subword embedding, scaled, into the residual stream.
* embed_grad  mb_embed_backward: the table's gradient.
* xent        mb_cross_entropy: next-token losses and the logits' gradient.
* clip        mb_grad_norm and mb_grad_clip over the gradients of a whole model.

Sizes are those of the MambaByte models this repository names (d_model 1024, 1792, 2304 with d_inner
twice that; 53 and 48 layers; 8192-byte spans; 256 bytes), with small, ragged and odd ones around
them, and vocabularies of tens of thousands for subword drafters. Activations have unit variance,
tokens the skewed frequencies of text (rank to the power -1), logits a model that is often right.
"""
import math

import torch

own = False

DEV = "cuda"
SPAN = 8 * 8192 * 2048     # elements of the largest convolved span
ROWS = 65536 * 1024        # elements of the largest embedded span
LOGITS = 1003 * 32001      # logits of the largest loss
STATE = 16                 # states per channel of a layer (A is [d_inner, 16])


def listed():
    return [
        # Verifying drafts: 32 streams, 16 drafted bytes each, from their cached windows. Latency.
        dict(name="conv_b32_L16_D2048", kind="conv", batch=32, L=16, D=2048, dtype="bf16", wide=False, state=True,
             bias=True),
        # Training or evaluation at the full context: x is half of the in-projection's [x | z] rows.
        dict(name="conv_b8_L8192_D2048", kind="conv", batch=8, L=8192, D=2048, dtype="bf16", wide=True, state=False,
             bias=True),
        # Fine-tuning in fp32 on ragged spans of an odd width, windows carried across spans.
        dict(name="conv_grad_f32_b3_L1003_D1544", kind="conv_grad", batch=3, L=1003, D=1544, dtype="f32", wide=False,
             state=True, bias=True),
        # The backward of the full-context training span.
        dict(name="conv_grad_b8_L8192_D2048", kind="conv_grad", batch=8, L=8192, D=2048, dtype="bf16", wide=True,
             state=False, bias=True),
        # One decode step of 256 streams of the widest model: the residual stream's first value.
        dict(name="embed_n256_V256_W2304", kind="embed", n=256, V=256, W=2304, tokens="i64", table="bf16", out="f32",
             scale=1.0),
        # A training batch of 8 x 8192 bytes.
        dict(name="embed_n65536_V256_W1024", kind="embed", n=65536, V=256, W=1024, tokens="u8", table="bf16",
             out="f32", scale=32.0),
        # The byte table's gradient of that batch: few rows, each summed over many tokens.
        dict(name="embed_grad_n65536_V256_W1024", kind="embed_grad", n=65536, V=256, W=1024, tokens="u8", out="f32",
             scale=32.0),
        # A subword drafter's: many rows, most of them of a few tokens or none.
        dict(name="embed_grad_n8200_V32001_W1792", kind="embed_grad", n=8200, V=32001, W=1792, tokens="i64",
             out="bf16", scale=1.0),
        # Next-byte losses of the training batch.
        dict(name="xent_n65536_V256", kind="xent", n=65536, V=256, dtype="bf16", targets="u8", weight=False),
        # A subword vocabulary of odd size in fp32, some positions weighted out.
        dict(name="xent_f32_n1003_V32001", kind="xent", n=1003, V=32001, dtype="f32", targets="i64", weight=True),
        # Tiny model (tests, experiments): two layers, launches only.
        dict(name="clip_2x64", kind="clip", layers=2, d=64, rank=8, proj="f32", out="f32", clips=True),
        # The 353M-sized model: bf16 gradients of the projections, fp32 ones of the rest, clipped into the
        # fp32 tensors that an optimizer reads.
        dict(name="clip_53x1024", kind="clip", layers=53, d=1024, rank=64, proj="bf16", out="f32", clips=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["conv", "conv_grad", "conv_grad", "embed", "embed_grad", "embed_grad", "xent", "xent", "clip"])
    if kind in ("conv", "conv_grad"):
        D = rng.choice([2048, 3584, 4608, 8 * _log(rng, 2, 576), 8 * _log(rng, 8, 576)])
        dtype = "f32" if rng.random() < 0.3 else "bf16"
        L = _log(rng, 1, 8192)
        most = SPAN // (2 if dtype == "f32" else 1) // (L * D)
        return dict(kind=kind, batch=_log(rng, 1, min(64, most)), L=L, D=D, dtype=dtype, wide=rng.random() < 0.5,
                    state=rng.random() < 0.5, bias=rng.random() < 0.8)
    if kind in ("embed", "embed_grad"):
        W = rng.choice([1024, 1792, 2304, 8 * _log(rng, 1, 288)])
        V = rng.choice([256, 256, _log(rng, 2, 32001)])
        return dict(kind=kind, n=_log(rng, 1, min(65536, ROWS // W)), V=V, W=W,
                    tokens=rng.choice(["u8", "i32", "i64"]) if V <= 256 else rng.choice(["i32", "i64"]),
                    out=rng.choice(["f32", "bf16"]), scale=rng.choice([1.0, math.sqrt(W)]),
                    **({"table": rng.choice(["f32", "bf16"])} if kind == "embed" else {}))
    if kind == "xent":
        V = rng.choice([256, 256, _log(rng, 2, 64000)])
        dtype = rng.choice(["f32", "bf16"])
        return dict(kind=kind, n=_log(rng, 1, min(65536, LOGITS // (2 if dtype == "f32" else 1) // V)), V=V,
                    dtype=dtype, targets=rng.choice(["u8", "i32", "i64"]) if V <= 256 else rng.choice(["i32", "i64"]),
                    weight=rng.random() < 0.5)
    d = rng.choice([64, 1024, 1792, 8 * _log(rng, 8, 224)])
    most = max(1, 53 * 1024 * 1024 // (d * d))
    proj = rng.choice(["f32", "bf16"])
    return dict(kind=kind, layers=_log(rng, 1, min(53, most // (2 if proj == "f32" else 1) or 1)), d=d,
                rank=max(8, d // 16 // 8 * 8), proj=proj, out=rng.choice(["f32", "same", "inplace"]),
                clips=rng.random() < 0.7)


# ---------------------------------------------------------------------------
# inputs

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "u8": torch.uint8, "i32": torch.int32, "i64": torch.int64}


def _text(g, n, V, kind):
    """Tokens with the frequencies of text; a few of a signed type are padding (-1)."""
    weight = 1.0 / torch.arange(1, V + 1, device=DEV, dtype=torch.float32)
    order = torch.randperm(V, device=DEV, generator=g)
    tok = order[torch.multinomial(weight, n, replacement=True, generator=g)]
    if kind != "u8":
        tok = torch.where(torch.rand(n, device=DEV, generator=g) < 0.03, torch.full_like(tok, -1), tok)
    return tok.to(TYPES[kind])


def _model(case):
    """Shapes of a model's gradients and whether each is of a projection."""
    d, E, R = case["d"], 2 * case["d"], case["rank"]
    layer = [((d,), False), ((2, E, d), True), ((E, 4), False), ((E,), False), ((R + 2 * STATE, E), True),
             ((E, R), True), ((E,), False), ((E, STATE), False), ((E,), False), ((d, E), True)]
    return layer * case["layers"] + [((256, d), True), ((d,), False)]


def _numel(shape):
    return math.prod(shape)


def _views(case, dtype_of, fill):
    """A model's tensors as views of one flat buffer for each type: ({type: buffer}, tensors)."""
    model = [(shape, dtype_of(big)) for shape, big in _model(case)]
    flat = {}
    for dtype in dict.fromkeys(t for _, t in model):
        flat[dtype] = fill(sum(_numel(shape) for shape, t in model if t == dtype), dtype)
    at, views = dict.fromkeys(flat, 0), []
    for shape, dtype in model:
        views.append(flat[dtype][at[dtype]:at[dtype] + _numel(shape)].view(shape))
        at[dtype] += _numel(shape)
    return flat, views


def _inputs(case, seed):
    """Everything random in a case."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind = case["kind"]

    def rnd(*shape, dtype=torch.float32):
        return torch.randn(*shape, device=DEV, generator=g).to(dtype)
    if kind in ("conv", "conv_grad"):
        b, L, D, td = case["batch"], case["L"], case["D"], TYPES[case["dtype"]]
        i = dict(x=rnd(b, L, (2 if case["wide"] else 1) * D, dtype=td)[..., :D])
        i["w"] = torch.rand(D, 4, device=DEV, generator=g) - 0.5
        i["bias"] = 0.1 * rnd(D) if case["bias"] else None
        i["state"] = rnd(b, 3, D, dtype=td) if case["state"] else None
        if kind == "conv_grad":
            i["dout"] = rnd(b, L, D, dtype=td)
            i["dstate_out"] = rnd(b, 3, D, dtype=td) if case["state"] else None
        return i
    if kind in ("embed", "embed_grad"):
        i = dict(tokens=_text(g, case["n"], case["V"], case["tokens"]))
        if kind == "embed":
            i["table"] = rnd(case["V"], case["W"], dtype=TYPES[case["table"]])
        else:
            i["dout"] = rnd(case["n"], case["W"], dtype=TYPES[case["out"]])
        return i
    if kind == "xent":
        n, V = case["n"], case["V"]
        targets = _text(g, n, V, case["targets"])
        logits = 2.0 * rnd(n, V)
        right = (torch.rand(n, 1, device=DEV, generator=g) < 0.7).float() * math.log(V) * 1.5
        logits.scatter_add_(1, targets.long().clamp(min=0)[:, None], right)
        weight = None
        if case["weight"]:
            weight = torch.rand(n, device=DEV, generator=g)
            weight = torch.where(weight < 0.1, torch.zeros_like(weight), weight)
        return dict(logits=logits.to(TYPES[case["dtype"]]), targets=targets, weight=weight, scale=1.0 / n)
    total = sum(_numel(s) for s, _ in _model(case))
    flat, grads = _views(case, lambda big: TYPES[case["proj"]] if big else torch.float32,
                         lambda n, dtype: (0.01 * rnd(n)).to(dtype))
    return dict(flat=flat, grads=grads, max_norm=0.01 * math.sqrt(total) * (0.4 if case["clips"] else 4.0))


# ---------------------------------------------------------------------------
# what a program has before the call, and the call

def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    kind = case["kind"]
    if kind in ("conv", "conv_grad"):
        b, L, D, td = case["batch"], case["L"], case["D"], s["x"].dtype
        rows = torch.empty(b, L, (2 if case["wide"] else 1) * D, device=DEV, dtype=td)
        if kind == "conv":
            s["out"] = torch.empty(b, L, D, device=DEV, dtype=td)
            s["state_out"] = torch.empty(b, 3, D, device=DEV, dtype=td)
        else:
            s["grads"] = dict(dx=rows[..., :D], dw=torch.empty(D, 4, device=DEV))
            if case["bias"]:
                s["grads"]["dbias"] = torch.empty(D, device=DEV)
            if case["state"]:
                s["grads"]["dstate"] = torch.empty(b, 3, D, device=DEV, dtype=td)
    elif kind == "embed":
        s["out"] = torch.empty(case["n"], case["W"], device=DEV, dtype=TYPES[case["out"]])
    elif kind == "embed_grad":
        s["dtable"] = torch.empty(case["V"], case["W"], device=DEV)
    elif kind == "xent":
        s["loss"], s["dlogits"] = torch.empty(case["n"], device=DEV), torch.empty_like(s["logits"])
    else:
        s["norm"] = torch.empty(1, device=DEV)
        if case["out"] == "inplace" and not case["clips"]:   # clipped in place, a second pass would have other inputs
            s["out"], s["out_flat"] = s["grads"], s["flat"]
        else:
            s["out_flat"], s["out"] = _views(
                case, lambda big: TYPES[case["proj"]] if big and case["out"] != "f32" else torch.float32,
                lambda n, dtype: torch.empty(n, device=DEV, dtype=dtype))
    if own:
        from paper_2401_13660_gb300 import mbscan as mb
        if kind == "conv_grad":
            s["ws"] = torch.zeros(mb.mb_conv1d_backward_workspace_size(case["batch"], case["L"], case["D"]),
                                  dtype=torch.uint8, device=DEV)
        elif kind == "embed_grad":
            s["ws"] = torch.zeros(mb.mb_embed_backward_workspace_size(case["n"], case["V"], case["W"]),
                                  dtype=torch.uint8, device=DEV)
        elif kind == "clip":
            s["list"] = mb.mb_tensor_list(s["grads"])
            s["out_list"] = None if s["out"] is s["grads"] else mb.mb_tensor_list(s["out"])
            s["ws"] = torch.zeros(mb.mb_grad_norm_workspace_size(), dtype=torch.uint8, device=DEV)
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2401_13660_gb300 import mbscan as mb
    case, kind = s["case"], s["case"]["kind"]
    if kind == "conv":
        mb.mb_conv1d(s["x"], s["w"], s["out"], bias=s["bias"], state=s["state"], state_out=s["state_out"])
        return {"out": s["out"], "state_out": s["state_out"]}
    if kind == "conv_grad":
        mb.mb_conv1d_backward(s["x"], s["w"], s["dout"], bias=s["bias"], state=s["state"],
                              dstate_out=s["dstate_out"], grads=s["grads"], ws=s["ws"])
        return dict(s["grads"])
    if kind == "embed":
        mb.mb_embed(s["tokens"], s["table"], s["out"], scale=case["scale"])
        return {"out": s["out"]}
    if kind == "embed_grad":
        mb.mb_embed_backward(s["tokens"], s["dout"], s["dtable"], scale=case["scale"], ws=s["ws"])
        return {"dtable": s["dtable"]}
    if kind == "xent":
        mb.mb_cross_entropy(s["logits"], s["targets"], s["loss"], s["dlogits"], weight=s["weight"], scale=s["scale"])
        return {"loss": s["loss"], "dlogits": s["dlogits"]}
    mb.mb_grad_norm(s["list"], s["norm"], ws=s["ws"])
    mb.mb_grad_clip(s["list"], s["norm"], s["max_norm"], out=s["out_list"])
    return {"norm": s["norm"], **{str(t): flat for t, flat in s["out_flat"].items()}}


def _taps(s):
    """The window followed by the span, 32 bits: [batch, 3 + L, D]."""
    b, _, D = s["x"].shape
    before = torch.zeros(b, 3, D, device=DEV) if s["state"] is None else s["state"].float()
    return torch.cat([before, s["x"].float()], 1)


def _preact(s, u):
    L, w = s["x"].shape[1], s["w"]
    p = u[:, :L] * w[:, 0]
    for k in range(1, 4):
        p += u[:, k:k + L] * w[:, k]
    return p if s["bias"] is None else p + s["bias"]


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "conv":
        u = _taps(s)
        p = _preact(s, u)
        s["out"].copy_(p / (1 + torch.exp(-p)))
        s["state_out"].copy_(u[:, -3:])
        return {"out": s["out"], "state_out": s["state_out"]}
    if kind == "conv_grad":
        L, g, w = s["x"].shape[1], s["grads"], s["w"]
        u = _taps(s)
        p = _preact(s, u)
        sg = 1 / (1 + torch.exp(-p))
        dp = s["dout"].float() * sg * (1 + p * (1 - sg))
        du = torch.zeros_like(u)
        if s["dstate_out"] is not None:
            du[:, -3:] += s["dstate_out"].float()
        for k in range(4):
            du[:, k:k + L] += dp * w[:, k]
            g["dw"][:, k] = (dp * u[:, k:k + L]).sum((0, 1))
        g["dx"].copy_(du[:, 3:])
        if case["bias"]:
            g["dbias"].copy_(dp.sum((0, 1)))
        if case["state"]:
            g["dstate"].copy_(du[:, :3])
        return dict(g)
    if kind == "embed":
        tok = s["tokens"].long()
        valid = (tok >= 0) & (tok < case["V"])
        rows = s["table"][torch.where(valid, tok, 0)].float() * case["scale"]
        s["out"].copy_(torch.where(valid[:, None], rows, 0.0))
        return {"out": s["out"]}
    if kind == "embed_grad":
        tok = s["tokens"].long()
        valid = (tok >= 0) & (tok < case["V"])
        rows = torch.where(valid[:, None], s["dout"].float() * case["scale"], 0.0)
        s["dtable"].zero_()
        s["dtable"].index_add_(0, torch.where(valid, tok, 0), rows)
        return {"dtable": s["dtable"]}
    if kind == "xent":
        l, tgt = s["logits"].float(), s["targets"].long()
        valid = (tgt >= 0) & (tgt < case["V"])
        weight = valid.float() if s["weight"] is None else torch.where(valid, s["weight"], 0.0)
        at = torch.where(valid, tgt, 0)[:, None]
        top = l.amax(1, keepdim=True)
        e = torch.exp(l - top)
        total = e.sum(1, keepdim=True)
        s["loss"].copy_((top + torch.log(total) - l.gather(1, at))[:, 0] * weight)
        e /= total
        e.scatter_add_(1, at, torch.full_like(top, -1.0))
        e *= (weight * s["scale"])[:, None]
        s["dlogits"].copy_(e)
        return {"loss": s["loss"], "dlogits": s["dlogits"]}
    total = torch.zeros(1, device=DEV)
    for t in s["grads"]:
        total += t.float().square().sum()
    torch.sqrt(total, out=s["norm"])
    coef = torch.where(s["norm"] > s["max_norm"], s["max_norm"] / s["norm"], 1.0)
    for t, o in zip(s["grads"], s["out"]):
        o.copy_(t.float() * coef)
    return {"norm": s["norm"], **{str(t): flat for t, flat in s["out_flat"].items()}}


# ---------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    """Each input read once, each output written once."""
    kind = case["kind"]
    size = {"f32": 4, "bf16": 2, "u8": 1, "i32": 4, "i64": 8}
    if kind in ("conv", "conv_grad"):
        es, D = size[case["dtype"]], case["D"]
        t, window = case["batch"] * case["L"] * D, 3 * case["batch"] * D * es
        weights = D * (20 if case["bias"] else 16)
        if kind == "conv":
            return {"bytes": 2 * t * es + window * (2 if case["state"] else 1) + weights, "flops": 12 * t}
        return {"bytes": 3 * t * es + window * (3 if case["state"] else 0) + 2 * weights, "flops": 32 * t}
    if kind == "embed":
        n, V, W = case["n"], case["V"], case["W"]
        return {"bytes": n * size[case["tokens"]] + n * W * size[case["out"]] + min(n, V) * W * size[case["table"]],
                "flops": n * W}
    if kind == "embed_grad":
        n, V, W = case["n"], case["V"], case["W"]
        return {"bytes": n * size[case["tokens"]] + n * W * size[case["out"]] + V * W * 4, "flops": n * W + V * W}
    if kind == "xent":
        n, V = case["n"], case["V"]
        return {"bytes": 2 * n * V * size[case["dtype"]] + n * (size[case["targets"]] + (8 if case["weight"] else 4)),
                "flops": 6 * n * V}
    total = moved = 0
    for shape, big in _model(case):
        n, es = _numel(shape), size[case["proj"]] if big else 4
        total += n
        moved += n * es
        if case["clips"] or case["out"] != "inplace":
            moved += n * (4 if case["out"] == "f32" else es)
    return {"bytes": moved + 4, "flops": 3 * total}


# ---------------------------------------------------------------------------
# the same in 64 bits

def exact(case, seed):
    i = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("conv", "conv_grad"):
        b, L, D = i["x"].shape
        w = i["w"].double()
        u = torch.zeros(b, L + 3, D, device=DEV, dtype=torch.float64)
        u[:, 3:] = i["x"]
        if i["state"] is not None:
            u[:, :3] = i["state"]
        p = torch.zeros(b, L, D, device=DEV, dtype=torch.float64)
        if i["bias"] is not None:
            p += i["bias"].double()
        for j in range(4):   # tap j sees the input of j steps before
            p.addcmul_(u[:, 3 - j:3 - j + L], w[:, 3 - j])
        if kind == "conv":
            return {"out": torch.nn.functional.silu(p), "state_out": u[:, L:].clone()}
        sg = torch.sigmoid(p)
        dp = sg + torch.nn.functional.silu(p) * (1 - sg)
        dp *= i["dout"]
        padded = torch.zeros(b, L + 6, D, device=DEV, dtype=torch.float64)
        padded[:, 3:L + 3] = dp
        # inputs -3 .. L-1: input n feeds the outputs n .. n+3
        du = sum(padded[:, j:j + L + 3] * w[:, 3 - j] for j in range(4))
        if i["dstate_out"] is not None:
            du[:, L:] += i["dstate_out"].double()
        r = dict(dx=du[:, 3:], dw=torch.stack([torch.einsum("btd,btd->d", dp, u[:, k:k + L]) for k in range(4)], 1))
        if case["bias"]:
            r["dbias"] = dp.sum(1).sum(0)
        if case["state"]:
            r["dstate"] = du[:, :3]
        return r
    if kind == "embed":
        tok = i["tokens"].long()
        ok = ((tok >= 0) & (tok < case["V"])).nonzero()[:, 0]
        out = torch.zeros(case["n"], case["W"], device=DEV, dtype=torch.float64)
        out[ok] = i["table"].double().index_select(0, tok[ok]) * case["scale"]
        return {"out": out}
    if kind == "embed_grad":
        # sums of the sorted tokens' rows, as differences of running sums would lose digits: token by token groups
        tok = i["tokens"].long()
        ok = ((tok >= 0) & (tok < case["V"])).nonzero()[:, 0]
        dtable = torch.zeros(case["V"], case["W"], device=DEV, dtype=torch.float64)
        if ok.numel():
            srt, perm = torch.sort(tok[ok], stable=True)
            ids, counts = torch.unique_consecutive(srt, return_counts=True)
            rows = i["dout"][ok[perm]].double()
            dtable[ids] = torch.segment_reduce(rows, "sum", lengths=counts, axis=0) * case["scale"]
        return {"dtable": dtable}
    if kind == "xent":
        n, V = case["n"], case["V"]
        tgt = i["targets"].long()
        weight = torch.ones(n, device=DEV, dtype=torch.float64) if i["weight"] is None else i["weight"].double()
        weight = weight * ((tgt >= 0) & (tgt < V))
        logp = torch.log_softmax(i["logits"].double(), 1)
        hit = torch.arange(V, device=DEV)[None] == tgt[:, None]
        loss = -torch.where(hit, logp, 0.0).sum(1) * weight
        return {"loss": loss, "dlogits": (logp.exp() - hit.double()) * weight[:, None] * i["scale"]}
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in i["flat"].values()))
    coef = i["max_norm"] / norm if norm > i["max_norm"] else 1.0
    if case["out"] != "f32":
        out = {str(t): flat.double() * coef for t, flat in i["flat"].items()}
    else:   # one buffer, in the model's order
        out = {str(torch.float32): torch.cat([t.double().flatten() * coef for t in i["grads"]])}
    return {"norm": torch.tensor([norm], dtype=torch.float64), **out}
