"""Timed cases of the inner step's operators: what a replica that trains between two outer steps asks of the library.

`op`:
  norm     the 2-norm of all gradients and the factor that clips it
  adamw    one AdamW step over all tensors, first and second moments in fp32
  adamw8   the same step with the moments in 8 bits and one scale per 256 values
  lookup   token embeddings: scale * (T_S[x] + T_perp[x]) + PosEmbed[position]
  grad     gradient of the embedding table, summed over the tokens that share a row

Each operator has a plain form here (`own` false: elementary torch operations in fp32) and its call of the library
(`own` true).  Parameters lie in one flat buffer that the plan's tensors are views of, either packed at multiples of two
elements, so that most tensors start at no multiple of 16 bytes, or with every tensor at a multiple of 4096 elements.

Moments in 8 bits: a block is 256 consecutive elements of a tensor.  A block of m is held as e4m3 numbers (4 exponent
bits, 3 mantissa bits, largest value 448) times max|m| / 448, a block of v as those of its square root, s.  A value y
between two e4m3 numbers goes to the upper one where the fraction of the gap that it covers exceeds a threshold that
runs through the unit interval with the step and the element's place (a two-dimensional golden-ratio sequence), so that a
moment whose change per step is smaller than a gap still follows its average.  A root above zero is never held as zero.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List, Tuple

import torch

own = False

CHUNK, BLOCK = 4096, 256
LR, BETA1, BETA2, EPS, DECAY, STEP = 3e-4, 0.9, 0.95, 1e-8, 0.1, 100
MAX_NORM = 1.0
GRAD_SCALE = 0.37
PLACE, TIME = 0xC13FA9A9, 0x91E10DA5               # 2^32 / 1.3247..., 2^32 / 1.3247...^2: steps of the rounding thresholds


def listed() -> List[dict]:
    return [
        # One attention matrix of the 1B model: a call that takes little more than its launches.
        _params("norm 2048x2048", "norm", d=2048, layers=0, ffn=0, vocab=2048, gain=0, grads="f32"),
        # All gradients of the 0.9B model at sizes that are no multiples of anything, bf16 as a mixed-precision backward leaves them.
        _params("norm 0.9B ragged bf16", "norm", d=2050, layers=16, ffn=5630, vocab=32001, gain=2047, grads="bf16"),
        # One matrix: the smallest step.
        _params("adamw 2048x2048", "adamw", d=2048, layers=0, ffn=0, vocab=2048, gain=0, grads="f32"),
        # The 150M model of the experiments, fp32 throughout, clipped.
        _params("adamw 150M", "adamw", d=768, layers=12, ffn=3072, vocab=50304, gain=768, grads="f32", clipped=True),
        # The 0.9B model at odd sizes, packed: bf16 gradients, and the bf16 copy that the next forward pass reads.
        _params("adamw 0.9B ragged bf16", "adamw", d=2050, layers=16, ffn=5630, vocab=32001, gain=2047, grads="bf16",
                clipped=True, copy=True),
        # One of four pipeline stages of the 150M model, moments in 8 bits.
        _params("adamw8 150M stage", "adamw8", d=768, layers=3, ffn=3072, vocab=1, gain=768, grads="f32", packed=False),
        # The 0.9B model, moments in 8 bits, bf16 gradients and copy.
        _params("adamw8 0.9B bf16", "adamw8", d=2048, layers=16, ffn=5632, vocab=32000, gain=2048, grads="bf16",
                packed=False, clipped=True, copy=True),
        # One short prompt: latency.
        _lookup("lookup 37x768", rows=37, seq=1024, d=768, vocab=50304, tables=1, table="f32", out="f32"),
        # A micro-batch of the 1B model: both parts of the split table, bf16 activations.
        _lookup("lookup 16384x2048 split", rows=16384, seq=1024, d=2048, vocab=32000, tables=2, table="f32", out="bf16"),
        # One sequence into the 150M model's table: most rows stay empty, and writing them is most of the work.
        _grad("grad 1024x768", rows=1024, d=768, vocab=50304, grads="f32", out="f32"),
        # A micro-batch of the 1B model; a few tokens are in it a thousand times.
        _grad("grad 16384x2048 bf16", rows=16384, d=2048, vocab=32000, grads="bf16", out="f32"),
        # A large ragged batch with padding, added to the gradient that earlier micro-batches left.
        _grad("grad 65537x2050 accumulated", rows=65537, d=2050, vocab=32001, grads="f32", out="f32", padding=True,
              accumulate=True),
    ]


def _params(name, op, *, d, layers, ffn, vocab, gain, grads, packed=True, clipped=False, copy=False) -> dict:
    return dict(name=name, op=op, d=d, layers=layers, ffn=ffn, vocab=vocab, gain=gain, grads=grads, packed=packed,
                clipped=clipped, copy=copy)


def _lookup(name, *, rows, seq, d, vocab, tables, table, out) -> dict:
    return dict(name=name, op="lookup", rows=rows, seq=seq, d=d, vocab=vocab, tables=tables, table=table, out=out)


def _grad(name, *, rows, d, vocab, grads, out, padding=False, accumulate=False) -> dict:
    return dict(name=name, op="grad", rows=rows, d=d, vocab=vocab, grads=grads, out=out, padding=padding,
                accumulate=accumulate)


def _log_uniform(rng: random.Random, low: float, high: float) -> int:
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng: random.Random) -> dict:
    op = rng.choice(("norm", "adamw", "adamw8", "lookup", "grad"))
    d = _log_uniform(rng, 64, 2050)
    if rng.random() < 0.5:
        d = -(-d // 64) * 64
    if op in ("norm", "adamw", "adamw8"):
        total = _log_uniform(rng, 2e5, 8e8)
        ffn = int(d * rng.choice((2.75, 3, 4))) + rng.choice((0, 0, 1, 2, 30))
        layer = 4 * d * d + 3 * d * ffn
        layers = min(48, total // (2 * layer))
        vocab = max(1, min(50304, (total - layers * layer) // d))
        case = _params("", op, d=d, layers=layers, ffn=ffn, vocab=vocab, gain=rng.choice((d, d, d - 1)),
                       grads=rng.choice(("f32", "bf16")), packed=op != "adamw8", clipped=rng.random() < 0.5,
                       copy=op != "norm" and rng.random() < 0.4)
    elif op == "lookup":
        rows = _log_uniform(rng, 1, 65536)
        case = _lookup("", rows=rows, seq=rng.choice((0, 512, 1024, 2048)), d=d, vocab=_log_uniform(rng, 256, 50304),
                       tables=rng.choice((1, 2)), table=rng.choice(("f32", "f32", "bf16")), out=rng.choice(("f32", "bf16")))
    else:
        rows = _log_uniform(rng, 1, 65536)
        case = _grad("", rows=rows, d=d, vocab=_log_uniform(rng, 256, 50304), grads=rng.choice(("f32", "bf16")),
                     out=rng.choice(("f32", "f32", "bf16")), padding=rng.random() < 0.3, accumulate=rng.random() < 0.3)
    del case["name"]
    return case


def _shapes(case) -> List[Tuple[int, ...]]:
    """Matrices and norm gains of a LLaMA-style decoder with a tied embedding."""
    d, ffn, gain = case["d"], case["ffn"], (case["gain"],)
    layer = [(d, d)] * 4 + [(d, ffn), (d, ffn), (ffn, d), gain, gain]
    return layer * case["layers"] + [(case["vocab"], d), gain]


def _places(case) -> Tuple[List[Tuple[int, int]], int]:
    """(start, elements) of every tensor in the flat buffer, and the buffer's length."""
    at, places = 0, []
    for shape in _shapes(case):
        n = math.prod(shape)
        places.append((at, n))
        step = 2 if case["packed"] else CHUNK
        at += -(-n // step) * step
    return places, at


DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _tokens(n: int, vocab: int, gen) -> torch.Tensor:
    """Token ids with frequencies that fall like 1 / rank, as those of text do: id = floor((vocab + 1)^u) - 1."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1)).floor() - 1).clamp_(0, vocab - 1).to(torch.int32)


def prepare(case: Dict, seed: int) -> Dict:
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def randn(n, std, dtype=torch.float32):
        x = torch.randn(n, generator=gen, device="cuda")
        return x.mul_(std).to(dtype)

    def rand(n):
        return torch.rand(n, generator=gen, device="cuda")

    state = dict(case=case, op=case["op"])
    if own:
        from paper_2601_02360_amd import binding
        state.update(B=binding)
    if case["op"] in ("norm", "adamw", "adamw8"):
        places, n = _places(case)
        real = torch.ones(n, dtype=torch.bool, device="cuda")
        ends = [start for start, _ in places[1:]] + [n]
        for (start, length), end in zip(places, ends):
            real[start + length:end] = False

        def values(x):
            return torch.where(real, x, torch.zeros((), dtype=x.dtype, device="cuda"))

        # heavy-tailed gradients around 1e-3, moments of the size that such gradients leave
        g = randn(n, 1.0)
        g = g.mul_(g.abs()).mul_(1e-3).to(DTYPES[case["grads"]])
        state.update(grads=values(g))
        if case["op"] == "norm":
            state.update(out=torch.empty(2, device="cuda"))
        else:
            state.update(theta=values(randn(n, 0.02)), grad_scale=torch.full((1,), GRAD_SCALE, device="cuda") if case["clipped"] else None,
                         copy=torch.zeros(n, dtype=torch.bfloat16, device="cuda") if case["copy"] else None)
        if case["op"] == "adamw":
            state.update(m=values(randn(n, 3e-4)), v=values((rand(n) * 1e-3 + 3e-4).square_()))
        if case["op"] == "adamw8":
            e4m3 = torch.float8_e4m3fn
            m = values(randn(n, 120.0).clamp_(-448, 448)).to(e4m3)
            v = values(rand(n).mul_(430).add_(1.0)).to(e4m3)
            state.update(m=m, v=v, m_scale=(rand(n // BLOCK) + 0.5) * (1e-3 / 448), v_scale=(rand(n // BLOCK) + 0.5) * (2e-3 / 448))
        if own:
            _bind(state, places)
        return state
    rows, d, vocab = case["rows"], case["d"], case["vocab"]
    ids = _tokens(rows, vocab, gen)
    if case["op"] == "lookup":
        kind = DTYPES[case["table"]]
        state.update(ids=ids, table=randn((vocab, d), 0.02, kind), t_perp=randn((vocab, d), 0.02, kind) if case["tables"] == 2 else None,
                     pos=randn((case["seq"], d), 0.02, kind) if case["seq"] else None, scale=math.sqrt(d),
                     out=torch.empty(rows, d, dtype=DTYPES[case["out"]], device="cuda"))
        return state
    pad = -1
    if case["padding"]:                                      # a tenth of the tokens, the end-of-text token's id
        pad = vocab - 1
        ids = torch.where(rand(rows) < 0.1, torch.full_like(ids, pad), ids)
    kind = DTYPES[case["out"]]
    table = randn((vocab, d), 1e-3, kind) if case["accumulate"] else torch.empty(vocab, d, dtype=kind, device="cuda")
    state.update(ids=ids, pad=pad, grad_out=randn((rows, d), 1e-3, DTYPES[case["grads"]]), table=table, scale=math.sqrt(d))
    if own:
        state.update(workspace=state["B"].embedding_grad_workspace(rows, vocab, d))
    return state


def _bind(state: Dict, places) -> None:
    """The plan and the bound tensors that a training program keeps beside its flat buffers."""
    B = state["B"]
    plan = B.Plan([n for _, n in places], kappa=32)

    def bound(flat):
        return plan.bind([flat[at:at + n] for at, n in places], dtype=flat.dtype)

    state.update(plan=plan, b_grads=bound(state["grads"]))
    if state["op"] == "norm":
        state.update(workspace=B.grad_norm_workspace())
        return
    state.update(b_theta=bound(state["theta"]), b_copy=None if state["copy"] is None else bound(state["copy"]))
    if state["op"] == "adamw":
        state.update(b_m=bound(state["m"]), b_v=bound(state["v"]))


def run(s: Dict):
    return (_OWN if own else _PLAIN)[s["op"]](s)


# ---------------------------------------------------------------- the library's calls

def _own_norm(s):
    s["B"].sparseloco_grad_norm(s["plan"], s["b_grads"], s["out"], s["workspace"], max_norm=MAX_NORM)
    return s["out"]


def _own_adamw(s):
    s["B"].sparseloco_adamw_step(s["plan"], s["b_theta"], s["b_grads"], s["b_m"], s["b_v"], lr=LR, step=STEP,
                                 beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY, grad_scale=s["grad_scale"],
                                 theta_bf16=s["b_copy"])
    return {"theta": s["theta"], "m": s["m"], "v": s["v"], "copy": s["copy"]}


def _own_adamw8(s):
    s["B"].sparseloco_adamw_step_8bit(s["plan"], s["b_theta"], s["b_grads"], s["m"], s["m_scale"], s["v"], s["v_scale"],
                                      lr=LR, step=STEP, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY,
                                      grad_scale=s["grad_scale"], theta_bf16=s["b_copy"])
    return {"theta": s["theta"], "m": s["m"], "m_scale": s["m_scale"], "v": s["v"], "v_scale": s["v_scale"], "copy": s["copy"]}


def _own_lookup(s):
    s["B"].sparseloco_embedding_lookup(s["table"], s["ids"], s["out"], t_perp=s["t_perp"], pos_embed=s["pos"], scale=s["scale"])
    return s["out"]


def _own_grad(s):
    s["B"].sparseloco_embedding_grad(s["grad_out"], s["ids"], s["table"], s["workspace"], scale=s["scale"],
                                     ignore_id=s["pad"], accumulate=s["case"]["accumulate"])
    return s["table"]


_OWN = {"norm": _own_norm, "adamw": _own_adamw, "adamw8": _own_adamw8, "lookup": _own_lookup, "grad": _own_grad}


# ---------------------------------------------------------------- the plain forms

def _plain_norm(s):
    norm = s["grads"].float().square().sum().sqrt()
    factor = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))
    s["out"].copy_(torch.stack([norm, factor]))
    return s["out"]


def _moments(s, m, v):
    """New moments and the change of the parameters but for the decay."""
    g = s["grads"].float()
    if s["grad_scale"] is not None:
        g = g * s["grad_scale"]
    m = m.mul(BETA1).add_(g, alpha=1 - BETA1)
    v = v.mul(BETA2).add_(g.square(), alpha=1 - BETA2)
    root = v.sqrt()
    change = (m / (root / math.sqrt(1 - BETA2 ** STEP) + EPS)).mul_(LR / (1 - BETA1 ** STEP))
    return m, v, root, change


def _apply(s, change):
    s["theta"].mul_(1 - LR * DECAY).sub_(change)
    if s["copy"] is not None:
        s["copy"].copy_(s["theta"])


def _plain_adamw(s):
    m, v, _, change = _moments(s, s["m"], s["v"])
    s["m"].copy_(m)
    s["v"].copy_(v)
    _apply(s, change)
    return {"theta": s["theta"], "m": s["m"], "v": s["v"], "copy": s["copy"]}


def _signed(x: int) -> int:
    return (x + 2 ** 31) % 2 ** 32 - 2 ** 31


def _held(x, offset):
    """Blocks of values as e4m3 numbers and their scales."""
    most = x.abs().amax(1)
    inverse = torch.where(most > 0, 448.0 / most, torch.zeros_like(most))
    y = x * inverse[:, None]
    place = torch.arange(x.numel(), dtype=torch.int32, device="cuda").mul_(_signed(PLACE))
    threshold = (place.add_(_signed(STEP * TIME + offset)) >> 12) & 0xFFFFF
    # times 2^-120 an e4m3 number has its exponent and mantissa in bits 20 to 26 of the fp32 pattern, subnormal ones too
    code = ((y.abs() * 2.0 ** -120).view(torch.int32) + threshold.view_as(x)) >> 20
    return y, code.clamp_(max=126), most / 448.0


def _plain_adamw8(s):
    m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
    root = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1)
    m, _, root, change = _moments(s, m, root.square_())
    y, code, scale = _held(m.view(-1, BLOCK), 0)
    s["m"].copy_((code | (y < 0).to(torch.int32) * 128).to(torch.uint8).view(torch.float8_e4m3fn).view(-1))
    s["m_scale"].copy_(scale)
    y, code, scale = _held(root.view(-1, BLOCK), 2 ** 31)
    s["v"].copy_(torch.where(y > 0, code.clamp(min=1), code).to(torch.uint8).view(torch.float8_e4m3fn).view(-1))
    s["v_scale"].copy_(scale)
    _apply(s, change)
    return {"theta": s["theta"], "m": s["m"], "m_scale": s["m_scale"], "v": s["v"], "v_scale": s["v_scale"], "copy": s["copy"]}


def _plain_lookup(s):
    ids = s["ids"].long()
    x = s["table"][ids].float()
    if s["t_perp"] is not None:
        x = x + s["t_perp"][ids].float()
    x = x * s["scale"]
    if s["pos"] is not None:
        x = x + s["pos"][torch.arange(len(ids), device="cuda") % len(s["pos"])].float()
    return x.to(s["out"].dtype)


def _plain_grad(s):
    ids = s["ids"].long()
    rows = s["grad_out"].float() * s["scale"]
    if s["pad"] >= 0:
        rows = rows * (ids != s["pad"])[:, None]
    total = s["table"].float() if s["case"]["accumulate"] else torch.zeros(s["table"].shape, device="cuda")
    total = total.index_add(0, ids, rows)
    s["table"].copy_(total)
    return s["table"]


_PLAIN = {"norm": _plain_norm, "adamw": _plain_adamw, "adamw8": _plain_adamw8, "lookup": _plain_lookup, "grad": _plain_grad}


# ---------------------------------------------------------------- what a pass cannot do without

def _distinct(rows: int, vocab: int) -> float:
    """Expected number of different tokens among `rows` of _tokens."""
    rank = torch.arange(1, vocab + 1, dtype=torch.float64)
    p = torch.log1p(1 / rank) / math.log(vocab + 1)
    return float((1 - (1 - p) ** rows).sum())


def work(case: Dict) -> Dict:
    size = {"f32": 4, "bf16": 2}
    op = case["op"]
    if op in ("norm", "adamw", "adamw8"):
        n = sum(math.prod(shape) for shape in _shapes(case))
        g = size[case["grads"]]
        if op == "norm":
            return {"bytes": n * g + 8, "flops": 2 * n}
        held = 16 if op == "adamw" else 4 + 16 / BLOCK       # both moments, read and written
        return {"bytes": n * (g + 8 + held + (2 if case["copy"] else 0)), "flops": (16 if op == "adamw" else 30) * n}
    rows, d = case["rows"], case["d"]
    touched = _distinct(rows, case["vocab"]) * d
    if op == "lookup":
        tables = touched * case["tables"] + min(rows, case["seq"]) * d
        return {"bytes": tables * size[case["table"]] + rows * (d * size[case["out"]] + 4),
                "flops": rows * d * (case["tables"] + (1 if case["seq"] else 0))}
    table = (2 * touched if case["accumulate"] else case["vocab"] * d) * size[case["out"]]
    return {"bytes": rows * (d * size[case["grads"]] + 4) + table, "flops": 2 * rows * d}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case: Dict, seed: int):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"norm": _exact_norm, "adamw": _exact_adamw, "adamw8": _exact_adamw, "lookup": _exact_lookup, "grad": _exact_grad}[case["op"]](s)


def _exact_norm(s):
    norm = math.sqrt(sum(float(torch.dot(part, part)) for part in (x.double() for x in s["grads"].split(1 << 26))))
    return torch.tensor([norm, min(1.0, MAX_NORM / norm) if norm else 1.0], dtype=torch.float64)


def _exact_adamw(s):
    eight = s["op"] == "adamw8"
    n = s["theta"].numel()
    names = ["theta", "m", "v"] + (["m_scale", "v_scale"] if eight else [])
    parts: Dict[str, list] = {name: [] for name in names}
    f = GRAD_SCALE_F32 if s["grad_scale"] is not None else 1.0
    for at in range(0, n, 1 << 26):                          # (a multiple of the block)
        cut = slice(at, min(n, at + (1 << 26)))
        blocks = slice(cut.start // BLOCK, -(-cut.stop // BLOCK))
        m, v = s["m"][cut].double(), s["v"][cut].double()
        if eight:
            m = m * s["m_scale"][blocks].double().repeat_interleave(BLOCK)
            v = (v * s["v_scale"][blocks].double().repeat_interleave(BLOCK)) ** 2
        g = s["grads"][cut].double() * f
        m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g * g
        m_hat, v_hat = m / (1 - BETA1 ** STEP), v / (1 - BETA2 ** STEP)
        theta = s["theta"][cut].double()
        parts["theta"].append(theta - LR * DECAY * theta - LR * m_hat / (torch.sqrt(v_hat) + EPS))
        if eight:
            m, m_scale = _exact_held(m, at, 0)
            v, v_scale = _exact_held(torch.sqrt(v), at, 2 ** 31)
            parts["m_scale"].append(m_scale)
            parts["v_scale"].append(v_scale)
        parts["m"].append(m)
        parts["v"].append(v)
    whole = {name: torch.cat(p) for name, p in parts.items()}
    whole["copy"] = None if s["copy"] is None else whole["theta"]
    return whole


GRAD_SCALE_F32 = float(torch.tensor(GRAD_SCALE, dtype=torch.float32))


def _exact_held(x, first: int, offset: int):
    scale = x.abs().reshape(-1, BLOCK).max(dim=1).values / 448
    wide = scale.repeat_interleave(BLOCK)
    a = torch.where(wide > 0, x.abs() / wide, torch.zeros_like(x))
    gap = torch.ldexp(torch.ones_like(a), torch.frexp(a).exponent.clamp(min=-5) - 4)     # 2^(exponent - 3), subnormal below 2^-6
    place = torch.arange(first, first + x.numel(), device=x.device)
    threshold = ((place * PLACE + STEP * TIME + offset) % 2 ** 32).div(2 ** 12, rounding_mode="floor") / 2.0 ** 20
    held = (torch.floor(a / gap + threshold) * gap).clamp(max=448.0)
    if offset:
        held = torch.where((a > 0) & (held == 0), torch.full_like(held, 2.0 ** -9), held)
    return held * torch.sign(x), scale


def _exact_lookup(s):
    ids = s["ids"].long()
    x = torch.index_select(s["table"], 0, ids).double()
    if s["t_perp"] is not None:
        x += torch.index_select(s["t_perp"], 0, ids).double()
    x *= float(torch.tensor(s["scale"], dtype=torch.float32))
    if s["pos"] is not None:
        seq = len(s["pos"])
        x += s["pos"].double().repeat(-(-len(ids) // seq), 1)[:len(ids)]
    return x


def _exact_grad(s):
    keep = (s["ids"] != s["pad"]).nonzero().flatten()
    ids, order = s["ids"][keep].long().sort(stable=True)
    rows = s["grad_out"][keep[order]].double() * float(torch.tensor(s["scale"], dtype=torch.float32))
    total = s["table"].double() if s["case"]["accumulate"] else torch.zeros(s["table"].shape, dtype=torch.float64, device="cuda")
    total.index_put_((ids,), rows, accumulate=True)
    return total
