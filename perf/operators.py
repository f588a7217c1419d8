"""Workloads of the token log probabilities and of the adapters' optimizer step: what is called, on which sizes, and how
much work that is.  Each runs in two forms: the plain one (`own` false), elementary torch operations in 32 bits, and the
library's calls (`own` true).  Kinds of case:

  score   log probabilities of given tokens with entropy, and the k most likely alternatives of each position
  step    the same without alternatives, and the gradient with respect to the logits
  adamw   one AdamW step over many tensors
  norm    the norm of all gradients

Logits are those of a language model: a spread of a few units and a token that stands out on half of the rows; some rows
have no target, and masks ban tokens with minus infinity.  Adapter shapes are those of the LLaMA-7B projections.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 256                     # weights that share one scale of the 8-bit states
BETAS, EPS = (0.9, 0.999), 1e-8
LR, MAX_NORM, LOSS_SCALE = 2e-4, 0.3, 2.0 ** 14
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}
MULT_A, MULT_B, WEYL = 0x6A09E667, 0xBB67AE85, 0x9E3779B9      # fractions of sqrt 2, sqrt 3 and the golden ratio


def _score(name, M, V, dtype, k, entropy=True, pad=0, mask="none"):
    return {"name": name, "kind": "score", "M": M, "V": V, "dtype": dtype, "k": k, "entropy": entropy, "pad": pad,
            "mask": mask}


def _step(name, M, V, dtype, entropy=True, pad=0, mask="none"):
    return {"name": name, "kind": "step", "M": M, "V": V, "dtype": dtype, "entropy": entropy, "pad": pad, "mask": mask}


def _adamw(name, blocks, rank, param, grad, bits, master=False, clip=True, hidden=4096, ffn=11008, odd=0, decay=0.01,
           lr_ratio=1.0):
    return {"name": name, "kind": "adamw", "blocks": blocks, "hidden": hidden, "ffn": ffn, "rank": rank, "param": param,
            "grad": grad, "bits": bits, "master": master, "clip": clip, "odd": odd, "decay": decay,
            "lr_ratio": lr_ratio}


def _norm(name, blocks, rank, grad, hidden=4096, ffn=11008, odd=0):
    return {"name": name, "kind": "norm", "blocks": blocks, "hidden": hidden, "ffn": ffn, "rank": rank, "grad": grad,
            "odd": odd}


def listed():
    return [
        # generation for one sequence: the chosen token's log probability and five alternatives
        _score("score_1x32000", 1, 32000, "f16", 5),
        # a batch of sixteen sequences under a grammar, logits in 32 bits, twenty alternatives
        _score("score_16x32000_f32", 16, 32000, "f32", 20, mask="grammar"),
        # perplexity of a 2048-token sequence: no alternatives, no entropy
        _score("score_2048x32000", 2048, 32000, "f16", 0, entropy=False),
        # scoring of prompts with a large, odd vocabulary in padded rows, some tokens banned
        _score("score_777x128259", 777, 128259, "bf16", 20, pad=61, mask="banned"),
        # policy gradient with an entropy bonus on one 2048-token sequence
        _step("step_2048x32000", 2048, 32000, "f16"),
        # a ragged batch in 32 bits, odd vocabulary (rows at any alignment), no entropy term
        _step("step_333x50257_f32", 333, 50257, "f32", entropy=False),
        # one projection's adapters, no clipping: the latency of a step
        _adamw("adamw_projection", 0, 8, "f16", "f32", 32, clip=False, odd=2),
        # every projection of LLaMA-7B at rank 8: fp16 weights with fp32 masters, clipped, LoRA+ rates
        _adamw("adamw_7b_r8", 32, 8, "f16", "f32", 32, master=True, lr_ratio=4.0),
        # odd sizes: adapters with trained norms and biases beside them, 8-bit states
        _adamw("adamw_odd_8bit", 4, 16, "bf16", "bf16", 8, odd=40),
        # every projection of LLaMA-7B at rank 64 in bf16 with 8-bit states: the largest
        _adamw("adamw_7b_r64_8bit", 32, 64, "bf16", "f32", 8),
        # the norm of the gradients of two blocks, 16-bit, for a log line
        _norm("norm_small", 2, 8, "bf16", odd=5),
        # the norm of all of LLaMA-7B's adapter gradients at rank 16
        _norm("norm_7b_r16", 32, 16, "f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["score", "score", "step", "adamw", "adamw", "norm"])
    if kind in ("score", "step"):
        V = rng.choice([_log_int(rng, 1, 2048), _log_int(rng, 512, 150000), _log_int(rng, 8000, 70000), 32000])
        M = min(_log_int(rng, 1, 2048), max(1, 777 * 128259 // (V if kind == "score" else 2 * V)))
        dtype, pad = rng.choice(["f16", "bf16", "f32"]), rng.choice([0, 0, 8, rng.randint(1, 130)])
        mask = rng.choice(["none", "none", "banned", "grammar", "lowest"])
        if kind == "score":
            c = _score("", M, V, dtype, rng.choice([0, 1, 5, 8, 20, rng.randint(2, 64)]), rng.random() < 0.7, pad, mask)
        else:
            c = _step("", M, V, dtype, rng.random() < 0.6, pad, mask)
    else:
        hidden, ffn = rng.choice([(2048, 5632), (4096, 11008), (5120, 13824)])
        rank, blocks, odd = 8 * rng.randint(1, 8), rng.choice([0, _log_int(rng, 1, 32)]), rng.choice([0, rng.randint(1, 60)])
        odd = odd or (0 if blocks else 3)
        blocks = min(blocks, int(32 * 64 * 4096 / (rank * hidden) / 3))
        if kind == "norm":
            c = _norm("", blocks, rank, rng.choice(["f32", "f32", "bf16", "f16"]), hidden, ffn, odd)
        else:
            param = rng.choice(["f16", "bf16", "bf16", "f32"])
            c = _adamw("", blocks, rank, param, rng.choice(["f32", "f32", param]), rng.choice([8, 32]),
                       param != "f32" and rng.random() < 0.5, rng.random() < 0.7, hidden, ffn, odd,
                       rng.choice([0.0, 0.01, 0.1]), rng.choice([1.0, 4.0]))
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _prepare_logits(c, seed):
    g, M, V, dtype = _generator(seed), c["M"], c["V"], TYPES[c["dtype"]]
    rand = lambda *shape: torch.rand(shape, device="cuda", generator=g)
    full = torch.randn((M, V + c["pad"]), device="cuda", generator=g).mul_(2.5)
    z = full[:, :V]
    rows = torch.arange(M, device="cuda")
    tokens = (rand(M) * V).long().clamp_(max=V - 1)
    z[rows, tokens] += torch.where(rand(M) < 0.5, 14.0, 0.0)          # the model is sure of half of the positions
    if c["mask"] == "banned":           # a tail of unused entries and a few tokens anywhere
        z[:, V - V // 50:] = -math.inf
        z.masked_fill_(rand(M, V) < 0.05, -math.inf)
    elif c["mask"] in ("grammar", "lowest"):        # a few tokens are allowed, the target among them
        low = -math.inf if c["mask"] == "grammar" else -65504.0 if c["dtype"] == "f16" else -3.0e38
        kept = z[rows, tokens]
        z.masked_fill_(rand(M, V) < 1 - 12.0 / max(V, 24), low)
        z[rows, tokens] = kept
        if M > 2:                                                   # ... and in one row none is
            z[0] = low
    tokens = torch.where(rand(M) < 0.1, -1, tokens).int()            # positions of the prompt: nothing to score
    s = {"case": c, "logits": full.to(dtype), "tokens": tokens}
    new = lambda shape, t=torch.float32: torch.empty(shape, dtype=t, device="cuda")
    s["logprob"], s["entropy"] = new(M), new(M) if c["entropy"] else None
    if c["kind"] == "score":
        k = c["k"]
        s["alt_tokens"], s["alt_logprobs"] = (new((M, k), torch.int32), new((M, k))) if k else (None, None)
    else:                               # advantages of a policy gradient, under a loss scale
        s["d_logprob"] = torch.randn(M, device="cuda", generator=g) * (LOSS_SCALE / M)
        s["d_entropy"] = torch.full((M,), 0.01 * LOSS_SCALE / M, device="cuda") if c["entropy"] else None
        s["stats"] = new((M, 4))
        s["dlogits"] = torch.zeros_like(s["logits"])
    return s


def _sizes(c):
    """Number of weights, factor of the learning rate and weight decay of each tensor."""
    h, f, r, ratio, decay = c["hidden"], c["ffn"], c["rank"], c.get("lr_ratio", 1.0), c.get("decay", 0.0)
    pair = lambda a, b: [(r * a, 1.0, decay), (b * r, ratio, decay)]
    block = 4 * pair(h, h) + 2 * pair(h, f) + pair(f, h)
    odd = (h, 1, h // 2 + 1, 257, f, 3, 255, 4 * h + 5)             # norms, biases, single factors
    return (c["blocks"] * block or pair(h, h)) + [(odd[i % 8], 1.0, 0.0) for i in range(c["odd"])]


def _layout(c):
    """Every kind of buffer is one allocation; a tensor begins at a multiple of BLOCK, what lies between stays zero.
    Returns (start, size, factor, decay) of each tensor and the whole length."""
    places, at = [], 0
    for n, ratio, decay in _sizes(c):
        places.append((at, n, ratio, decay))
        at += -(-n // BLOCK) * BLOCK
    return places, at


def _per_block(values, places):
    """One value a tensor -> a column with one value a block."""
    counts = torch.tensor([-(-p[1] // BLOCK) for p in places], device="cuda")
    return torch.repeat_interleave(torch.tensor(values, dtype=torch.float32, device="cuda"), counts)[:, None]


def _prepare_tensors(c, seed):
    g = _generator(seed)
    places, total = _layout(c)
    normal = lambda: torch.randn((total // BLOCK, BLOCK), device="cuda", generator=g)
    inside = torch.zeros(total, device="cuda")
    starts = torch.tensor([p[0] for p in places], device="cuda")
    ends = starts + torch.tensor([p[1] for p in places], device="cuda")
    inside[starts] += 1.0
    edge = ends[ends < total]
    inside.index_add_(0, edge, torch.full((edge.numel(),), -1.0, device="cuda"))
    inside = (inside.cumsum(0, dtype=torch.float64) > 0.5).view(-1, BLOCK)
    spread = _per_block([1e-5 * 10.0 ** (i % 5 / 2.0) for i in range(len(places))], places)     # typical gradient of a tensor
    s = {"case": c, "places": places, "total": total}
    scale = LOSS_SCALE if c["grad"] != "f16" else 1.0
    s["grad_scale"] = 1.0 / scale
    s["grad"] = (normal() * inside * spread * scale).to(TYPES[c["grad"]])
    if c["kind"] == "norm":
        s["norm"] = torch.empty(1, device="cuda")
        return s
    w = normal() * inside * 0.02
    s["param"] = w.to(TYPES[c["param"]])
    s["master"] = w if c["master"] else None
    m = normal() * inside * spread * 0.3
    v = (spread * (0.5 + torch.rand((total // BLOCK, BLOCK), device="cuda", generator=g))).square_() * inside
    if c["bits"] == 8:
        s["m_scale"], s["v_scale"] = _scale_of(m.abs().amax(1)), _scale_of(v.sqrt().amax(1))
        s["m"] = (m / s["m_scale"][:, None].clamp(min=1e-30)).to(torch.float8_e4m3fn)
        s["v"] = (v.sqrt() / s["v_scale"][:, None].clamp(min=1e-30)).to(torch.float8_e4m3fn)
    else:
        s["m"], s["v"] = m, v
    s["ratio"] = _per_block([p[2] for p in places], places)
    s["decay"] = _per_block([p[3] for p in places], places)
    s["taken"], s["seed"] = 10 + seed % 7, seed & 0xFFFF
    if own:
        s["optimizer"] = _optimizer(s)
    return s


def _scale_of(most):
    """The power of two by which a block's values are divided, so that the largest lies in (224, 448]."""
    frac, exp = torch.frexp(most)                                    # most = frac * 2^exp, frac in [0.5, 1)
    return torch.where(most > 0, torch.exp2((exp - 9 + (frac > 0.875)).float()), 0.0)


def _optimizer(s):
    """The plan that a training program makes once, over the tensors' buffers."""
    from paper_2306_08162_amd.device import AdapterOptimizer, OptimTensor
    c, tensors = s["case"], []
    for at, n, ratio, decay in s["places"]:
        part = lambda name: None if s.get(name) is None else s[name].view(-1)[at:at + n]
        scale = lambda name: s[name][at // BLOCK:(at + n + BLOCK - 1) // BLOCK] if c["bits"] == 8 else None
        tensors.append(OptimTensor(part("param"), part("grad"), master=part("master"), exp_avg=part("m"),
                                   exp_avg_sq=part("v"), avg_scale=scale("m_scale"), avg_sq_scale=scale("v_scale"),
                                   lr_scale=ratio, weight_decay=decay))
    return AdapterOptimizer(tensors, lr=LR, betas=BETAS, eps=EPS, max_grad_norm=MAX_NORM if c["clip"] else 0.0,
                            grad_scale=s["grad_scale"], seed=s["seed"], step=s["taken"])


def _gradients(s):
    """The plan over the gradients alone."""
    from paper_2306_08162_amd.device import AdapterOptimizer, OptimTensor
    flat = s["grad"].view(-1)
    return AdapterOptimizer([OptimTensor(None, flat[at:at + n]) for at, n, _, _ in s["places"]], lr=0.0,
                            grad_scale=s["grad_scale"])


def prepare(case, seed):
    if case["kind"] in ("score", "step"):
        s = _prepare_logits(case, seed)
        if own:
            from paper_2306_08162_amd import binding as ql
            s["flag"] = {"f16": ql.QLORA_F16, "bf16": ql.QLORA_BF16, "f32": ql.QLORA_F32}[case["dtype"]]
            nbytes = ql.qlora_token_logprobs_workspace_bytes(case["M"], case["V"], case.get("k", 0), s["flag"])
            s["workspace"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
        return s
    s = _prepare_tensors(case, seed)
    if own and case["kind"] == "norm":
        s["optimizer"] = _gradients(s)
    return s


# ------------------------------------------------------------------------------------------------------ plain forms

def _plain_logprobs(s):
    c = s["case"]
    V = c["V"]
    z = s["logits"][:, :V].float()
    top = z.amax(-1, keepdim=True)
    empty = top == -math.inf                                        # a row that masks every token
    d = z - torch.where(empty, 0.0, top)
    e = torch.exp(d)
    total = torch.where(empty, 1.0, e.sum(-1, keepdim=True))
    log_total = torch.log(total)
    given = (s["tokens"] >= 0) & (s["tokens"] < V)
    at = s["tokens"].clamp(0, V - 1).long()[:, None]
    out = {"logprob": torch.where(given, (d.gather(1, at) - log_total)[:, 0], 0.0)}
    if c["entropy"]:
        out["entropy"] = (log_total - (e * d.clamp(min=-1e30)).sum(-1, keepdim=True) / total)[:, 0]
    return out, d, e, total, log_total, given, at


def _plain_score(s):
    c = s["case"]
    out, d, _, _, log_total, _, _ = _plain_logprobs(s)
    if c["k"]:
        M, V, k = c["M"], c["V"], c["k"]
        # one whole number an entry: the value's order first, then the lower index
        bits = (s["logits"][:, :V].float() + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        key, at = torch.topk(order * 2 ** 31 + (2 ** 31 - 1 - torch.arange(V, device="cuda")), min(k, V), dim=-1)
        lp = d.gather(1, at) - log_total
        masked = s["logits"].gather(1, at) == -math.inf
        out["alt_tokens"] = torch.full((M, k), -1, dtype=torch.int32, device="cuda")
        out["alt_logprobs"] = torch.full((M, k), -math.inf, device="cuda")
        out["alt_tokens"][:, :V] = torch.where(masked, -1, at.int())
        out["alt_logprobs"][:, :V] = torch.where(masked, -math.inf, lp)
    return out


def _plain_step(s):
    out, d, e, total, log_total, given, at = _plain_logprobs(s)
    g = torch.where(given, s["d_logprob"], 0.0)[:, None]
    slope = g
    if s["d_entropy"] is not None:
        slope = g + s["d_entropy"][:, None] * (d.clamp(min=-1e30) - log_total + out["entropy"][:, None])
    dz = -(e / total) * slope
    dz.scatter_add_(1, at, g)
    out["dlogits"] = dz.to(s["logits"].dtype)
    return out


def _mix(x):
    """A 32-bit hash of signed 32-bit words (products wrap; the shifts bring in zeros)."""
    x = (x ^ ((x >> 16) & 0xFFFF)) * MULT_A
    x = (x ^ ((x >> 15) & 0x1FFFF)) * (MULT_B - 2 ** 32)
    return x ^ ((x >> 16) & 0xFFFF)


def _codes(x, scale, r):
    """x / scale in e4m3, rounded up or down with the odds of its place between the two; r: 20 random bits an element."""
    y = (x.abs() / torch.where(scale > 0, scale, 1.0)[:, None]).clamp(max=448.0) * 2.0 ** -120
    code = (y.view(torch.int32) + r) >> 20
    code = torch.where(x < 0, code | 0x80, code)
    return code.to(torch.uint8).view(torch.float8_e4m3fn)


def _plain_norm(s):
    return torch.sqrt(s["grad"].double().square().sum()) * s["grad_scale"]


def _plain_adamw(s):
    c, t = s["case"], s["taken"] + 1
    s["taken"] = t
    out, factor = {}, s["grad_scale"]
    if c["clip"]:       # (the inputs are finite: the step that an infinity would skip does not occur)
        norm = _plain_norm(s)
        out["norm"] = norm.float().reshape(1)
        factor = factor * torch.clamp(MAX_NORM / norm, max=1.0).float()
    g = s["grad"].float() * factor
    b1, b2 = BETAS
    if c["bits"] == 8:
        m = s["m"].float() * s["m_scale"][:, None]
        u = s["v"].float() * s["v_scale"][:, None]
        v = u * u
    else:
        m, v = s["m"], s["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    u = torch.sqrt(v)
    step = (LR / (1 - b1 ** t)) * s["ratio"]
    w = s["master"] if c["master"] else s["param"].float()
    w = w * (1 - LR * s["ratio"] * s["decay"]) - step * (m / (u * (1 - b2 ** t) ** -0.5 + EPS))
    if c["master"]:
        s["master"].copy_(w)
        out["master"] = s["master"]
    s["param"].copy_(w)
    out["param"] = s["param"]
    if c["bits"] == 8:
        key = _mix(torch.full((1,), (s["seed"] + t * WEYL + 2 ** 31) % 2 ** 32 - 2 ** 31, dtype=torch.int32, device="cuda"))
        r = _mix(torch.arange(s["total"], dtype=torch.int32, device="cuda").view(-1, BLOCK) + key)
        s["m_scale"].copy_(_scale_of(m.abs().amax(1)))
        s["v_scale"].copy_(_root_scale_of(v.amax(1)))
        s["m"].copy_(_codes(m, s["m_scale"], (r >> 12) & 0xFFFFF))
        # a second moment above zero keeps a code above zero
        code = _codes(u, s["v_scale"], r & 0xFFFFF).view(torch.uint8)
        s["v"].view(torch.uint8).copy_(torch.maximum(code, (v > 0).to(torch.uint8)))
        out |= {"m_scale": s["m_scale"], "v_scale": s["v_scale"]}
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    out |= {"m": s["m"], "v": s["v"]}
    return out


def _root_scale_of(most):
    """_scale_of(sqrt(most)) without the rounding of the root: sqrt(x) <= 1.75 * 2^k where x <= 3.0625 * 4^k."""
    frac, exp = torch.frexp(most)                                    # most = frac * 2^exp
    half = torch.div(exp - 1, 2, rounding_mode="floor")              # 4^half <= most < 4^(half + 1)
    over = torch.ldexp(frac, exp - 2 * half) > 3.0625
    return torch.where(most > 0, torch.exp2((half - 8 + over).float()), 0.0)


# --------------------------------------------------------------------------------------------------- library's calls

def _own_logprobs(s, k=0, alt_tokens=None, alt_logprobs=None):
    from paper_2306_08162_amd import binding as ql
    c = s["case"]
    stats = s.get("stats")
    ql.qlora_token_logprobs(s["logits"], c["V"] + c["pad"], s["tokens"], s["logprob"], s["entropy"], alt_tokens,
                            alt_logprobs, k, stats, c["M"], c["V"], s["flag"], s["workspace"])
    out = {"logprob": s["logprob"]}
    if c["entropy"]:
        out["entropy"] = s["entropy"]
    return out


def _own_score(s):
    out = _own_logprobs(s, s["case"]["k"], s["alt_tokens"], s["alt_logprobs"])
    if s["case"]["k"]:
        out |= {"alt_tokens": s["alt_tokens"], "alt_logprobs": s["alt_logprobs"]}
    return out


def _own_step(s):
    from paper_2306_08162_amd import binding as ql
    c = s["case"]
    out = _own_logprobs(s)
    ql.qlora_token_logprobs_bwd(s["logits"], c["V"] + c["pad"], s["tokens"], s["stats"], s["d_logprob"], s["d_entropy"],
                                s["dlogits"], c["V"] + c["pad"], c["M"], c["V"], s["flag"])
    out["dlogits"] = s["dlogits"][:, :c["V"]]
    return out


def _own_adamw(s):
    s["optimizer"].step()
    out = {name: s[name] for name in ("param", "master", "m", "v", "m_scale", "v_scale") if s.get(name) is not None}
    if s["case"]["clip"]:
        out["norm"] = s["optimizer"].last_grad_norm
    return out


def run(state):
    kind = state["case"]["kind"]
    if kind == "score":
        return _own_score(state) if own else _plain_score(state)
    if kind == "step":
        return _own_step(state) if own else _plain_step(state)
    if kind == "adamw":
        return _own_adamw(state) if own else _plain_adamw(state)
    if own:
        state["optimizer"].grad_norm(state["norm"])
        return state["norm"]
    return _plain_norm(state).float().reshape(1)


def work(case):
    c = case
    if c["kind"] in ("score", "step"):
        n = c["M"] * c["V"]
        nbytes = n * SIZE[c["dtype"]] + c["M"] * (8 + 4 * c["entropy"] + 8 * c.get("k", 0))
        if c["kind"] == "step":         # the gradient is written; what it reads, the first half has read
            return {"bytes": nbytes + n * SIZE[c["dtype"]] + c["M"] * (4 + 4 * c["entropy"]), "flops": 14 * n}
        return {"bytes": nbytes, "flops": 6 * n}
    n = sum(size for size, _, _ in _sizes(c))
    if c["kind"] == "norm":
        return {"bytes": n * SIZE[c["grad"]], "flops": 2 * n}
    per = SIZE[c["grad"]] + SIZE[c["param"]] + (8 if c["master"] else SIZE[c["param"]])
    per += 16 if c["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * per, "flops": (16 if c["bits"] == 32 else 36) * n + (2 * n if c["clip"] else 0)}


# ------------------------------------------------------------------------------------------------------ in 64 bits

def _exact_logits(s):
    """Row after row block from the definitions: p = softmax(z), H = -sum p ln p."""
    c = s["case"]
    M, V = c["M"], c["V"]
    parts = {"logprob": [], "entropy": [], "dlogits": [], "alt_logprobs": []}
    for at in range(0, M, 128):
        rows = slice(at, min(at + 128, M))
        z, tokens = s["logits"][rows, :V].double(), s["tokens"][rows].long()
        some = (z > -math.inf).any(1)
        logp = torch.log_softmax(torch.where(some[:, None], z, 0.0), 1)
        logp = torch.where(some[:, None], logp, -math.inf)
        p = logp.exp()
        plogp = torch.where(p > 0, p * logp, 0.0)
        H = -plogp.sum(1)
        hit = (torch.arange(V, device="cuda") == tokens[:, None])
        parts["logprob"].append(torch.where(hit, logp, 0.0).sum(1))
        parts["entropy"].append(H)
        if c["kind"] == "step":
            g = s["d_logprob"][rows].double() * hit.any(1)
            dz = g[:, None] * (hit.double() - p)
            if c["entropy"]:
                dz -= s["d_entropy"][rows].double()[:, None] * (plogp + p * H[:, None])
            parts["dlogits"].append(dz)
        elif c["k"]:
            best = torch.sort(logp, 1, descending=True).values[:, :c["k"]]
            parts["alt_logprobs"].append(torch.nn.functional.pad(best, (0, c["k"] - best.shape[1]), value=-math.inf))
    out = {"logprob": torch.cat(parts["logprob"])}
    if c["entropy"]:
        out["entropy"] = torch.cat(parts["entropy"])
    if c["kind"] == "step":
        out["dlogits"] = torch.cat(parts["dlogits"])
    elif c["k"]:
        out |= {"alt_tokens": None, "alt_logprobs": torch.cat(parts["alt_logprobs"])}
    return out


def _hash(x):
    """The hash in 64-bit arithmetic."""
    for multiplier, shift in ((MULT_A, 16), (MULT_B, 15)):
        x = ((x ^ (x >> shift)) * multiplier) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _exact_adamw(s):
    """Tensor after tensor from the definition (states of 8 bits: rounded up or down to them by the same random numbers)."""
    c, t = s["case"], s["taken"] + 1
    b1, b2 = BETAS
    grad = s["grad"].view(-1)
    out, factor = {}, s["grad_scale"]
    if c["clip"]:
        norm = math.sqrt(sum(float(grad[at:at + n].double().pow(2).sum()) for at, n, _, _ in s["places"])) * factor
        out["norm"] = torch.tensor([norm], dtype=torch.float64)
        factor *= min(1.0, MAX_NORM / norm)
    weights = (s["master"] if c["master"] else s["param"]).view(-1)
    got = {k: torch.zeros(s["total"], dtype=torch.float64, device="cuda") for k in ("w", "m", "v")}
    scales = {k: torch.zeros(s["total"] // BLOCK, dtype=torch.float64, device="cuda") for k in ("m", "v")}
    key = _hash(s["seed"] + t * WEYL & 0xFFFFFFFF)
    for at, n, ratio, decay in s["places"]:
        span, end = slice(at, at + n), at + -(-n // BLOCK) * BLOCK
        g = grad[span].double() * factor
        if c["bits"] == 8:
            wide = lambda k: s[k + "_scale"][at // BLOCK:end // BLOCK].double().repeat_interleave(BLOCK)[:n]
            m, v = s["m"].view(-1)[span].double() * wide("m"), (s["v"].view(-1)[span].double() * wide("v")) ** 2
        else:
            m, v = s["m"].view(-1)[span].double(), s["v"].view(-1)[span].double()
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        lr = LR * ratio
        got["w"][span] = weights[span].double() * (1 - lr * decay) - lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + EPS)
        if c["bits"] == 32:
            got["m"][span], got["v"][span] = m, v
            continue
        r = _hash((torch.arange(at, at + n, device="cuda") + key) & 0xFFFFFFFF)
        for name, x, bits in (("m", m, r >> 12), ("v", v.sqrt(), r & 0xFFFFF)):
            most = torch.nn.functional.pad(x.abs(), (0, end - at - n)).view(-1, BLOCK).amax(1)
            scale = torch.exp2(torch.ceil(torch.log2(most.clamp(min=1e-300) / 448.0)))
            y = x.abs() / scale.repeat_interleave(BLOCK)[:n]
            quantum = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)       # distance of the codes around y
            y = torch.floor(y / quantum + bits.double() / 2 ** 20) * quantum
            if name == "v":
                y = torch.where((v > 0) & (y == 0), 2.0 ** -9, y)
            got[name][span] = torch.where(x < 0, -y, y)
            scales[name][at // BLOCK:end // BLOCK] = torch.where(most > 0, scale, 0.0)
    shape = s["grad"].shape
    out |= {"param": got["w"].view(shape), "m": got["m"].view(shape), "v": got["v"].view(shape)}
    if c["master"]:
        out["master"] = got["w"].view(shape)
    if c["bits"] == 8:
        out |= {"m_scale": scales["m"], "v_scale": scales["v"]}
    return out


def exact(case, seed):
    if case["kind"] in ("score", "step"):
        return _exact_logits(_prepare_logits(case, seed))
    c = dict(case)
    s = _prepare_tensors(c, seed)
    if c["kind"] == "norm":
        total = sum(float(s["grad"].view(-1)[at:at + n].double().pow(2).sum()) for at, n, _, _ in s["places"])
        return torch.tensor([math.sqrt(total) * s["grad_scale"]], dtype=torch.float64)
    return _exact_adamw(s)
