"""The operators around the mask, as cases that can be timed: the output head that makes the logits, and what is read off them.

A case's kind says what one pass does:
  head   hidden states (bf16) of the rows to be decoded -> 8-bit blocks with their scales (quantize_blocks) -> the product with
         the head's 8-bit weights, a scale for each 128 x 128 block, written as logits with -inf where the row's mask forbids
         the token (head_logits)
  score  log probabilities of given tokens, the normaliser, the entropy and the top alternatives of each row's distribution
         over the tokens its mask allows (token_logprobs)
  train  the same without alternatives, and then the gradient of the logits (token_logprobs_backward)

A row's mask is that of a place in constrained text: `open` places (inside a string) allow nine tokens of ten, `narrow` ones
(punctuation, keys) a few dozen; "mixed" batches have both, "narrow" ones only the latter, "none" is without a mask.
"""
import math

import torch

own = False

NARROW = 24  # tokens that a narrow place allows, on average


def listed():
    def head(name, **kw):
        return dict({"name": name, "kind": "head", "mask": "mixed", "dtype": "bf16"}, **kw)

    def score(name, **kw):
        return dict({"name": name, "kind": "score", "mask": "mixed", "dtype": "bf16", "tokens": 1, "top": 0, "heat": False}, **kw)

    return [
        # one sequence of a tiny vocabulary: what a launch costs
        head("head-512-k256-n1", V=512, K=256, n=1),
        # eight sequences at places where the grammar leaves a few tokens: most of the weights need not be read
        head("head-narrow-32000-n8", V=32000, K=4096, n=8, mask="narrow"),
        # odd sizes everywhere, fp32 logits
        head("head-50001-k2880-n37", V=50001, K=2880, n=37, dtype="fp32"),
        # a decoding step of a server's batch: bound by reading the weights
        head("head-128256-n64", V=128256, K=4096, n=64),
        # the same with the largest batch
        head("head-128256-n256", V=128256, K=4096, n=256),
        # every position of a prompt scored at once: bound by the products
        head("head-128256-n2048", V=128256, K=4096, n=2048, mask="none"),
        # the greedy token and the likeliest alternatives of one sequence
        score("score-32000-n1", V=32000, n=1, top=20, dtype="fp32"),
        # a batch of constrained rows, rows that begin at any address, a temperature each
        score("score-50001-n48", V=50001, n=48, top=5, heat=True),
        # a server's batch
        score("score-128256-n256", V=128256, n=256, top=20, tokens=2),
        # a prompt's tokens scored
        score("score-128256-n2048", V=128256, n=2048, top=1, mask="none"),
        # a small update of constrained samples
        score("train-50001-n48-fp32", kind="train", V=50001, n=48, dtype="fp32", heat=True, tokens=3),
        # an update over the positions of several long samples
        score("train-128256-n2048", kind="train", V=128256, n=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["head", "head", "score", "train"])
    V = _log(rng, 512, 152064)
    n = _log(rng, 1, 2048)
    case = {"kind": kind, "V": V, "n": n, "mask": rng.choice(["mixed", "mixed", "narrow", "none"]), "dtype": rng.choice(["bf16", "bf16", "fp32"])}
    if kind == "head":
        case["K"] = K = _log(rng, 100, 8192)
        if case["dtype"] == "fp32":
            n = min(n, 1024)
        case["n"] = max(1, min(n, int(2048 * 128256 * 4096 / (V * K))))
    else:
        case["n"] = max(1, min(n, int(1024 * 128256 / V)))
        case["tokens"] = rng.choice([1, 1, 2, 5])
        case["top"] = rng.choice([0, 1, 5, 20, 32]) if kind == "score" else 0
        case["heat"] = rng.random() < 0.5
    return case


def work(case):
    n, V, size = case["n"], case["V"], 2 if case["dtype"] == "bf16" else 4
    allowed = {"none": 1.0, "mixed": 0.7 * 0.9, "narrow": min(1.0, NARROW / V)}[case["mask"]]  # of a row's tokens
    bytes_ = 0.0 if case["mask"] == "none" else n * 4.0 * ((V + 31) // 32)
    if case["kind"] == "head":
        some = 1.0 - (1.0 - min(1.0, NARROW / V)) ** n if case["mask"] == "narrow" else 1.0  # of the vocabulary, allowed by some row
        K = case["K"]
        return {"bytes": bytes_ + some * V * (K + 4.0 * ((K + 127) // 128) / 128) + 2.0 * n * K + size * float(n) * V,
                "flops": 2.0 * n * K * V * allowed}
    bytes_ += size * allowed * n * V + n * (12.0 + 8.0 * case["tokens"] + 8.0 * case["top"])
    if case["kind"] == "train":  # the logits once more, if they are not kept, and the gradient
        return {"bytes": bytes_ + size * float(n) * V, "flops": 12.0 * allowed * n * V}
    return {"bytes": bytes_, "flops": 6.0 * allowed * n * V}


# ------------------------------------------------------------------------------------------------ inputs


def _masks(gen, kind, n, V):
    """Packed masks, int32 [n, ceil(V / 32)], bit t & 31 of word t >> 5; the padding bits are 0."""
    if kind == "none":
        return None
    words = (V + 31) // 32
    out = torch.empty((n, words), dtype=torch.int32, device="cuda")
    weight = (1 << torch.arange(32, device="cuda", dtype=torch.int64))
    opens = torch.rand(n, generator=gen, device="cuda") < (0.7 if kind == "mixed" else 0.0)
    if kind == "mixed":
        opens[0] = True
    share = torch.where(opens, 0.9, min(1.0, NARROW / V))
    for r in range(0, n, 64):
        bits = torch.rand((min(64, n - r), words * 32), generator=gen, device="cuda") < share[r:r + 64, None]
        bits[:, V:] = False
        bits[:, r % V] = True  # no row is left without a token here
        packed = (bits.view(-1, words, 32).to(torch.int64) * weight).sum(-1)
        out[r:r + 64] = torch.where(packed >= 1 << 31, packed - (1 << 32), packed).to(torch.int32)
    return out


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _quantized_weights(gen, V, K, stride):
    """Weights as they are kept: e4m3 bytes in rows of `stride` and a scale for each 128 x 128 block."""
    vb, kb = (V + 127) // 128, (K + 127) // 128
    q = torch.zeros((V, stride), dtype=torch.uint8, device="cuda")
    scales = torch.empty((vb, kb), dtype=torch.float32, device="cuda")
    for r in range(0, V, 8192):
        rows = min(8192, V - r)
        w = torch.zeros((-(-rows // 128) * 128, kb * 128), device="cuda")
        w[:rows, :K] = torch.randn((rows, K), generator=gen, device="cuda") * (2.5 / math.sqrt(K))
        blocks = w.view(-1, 128, kb, 128)
        s = blocks.abs().amax((1, 3)) / 448.0
        scales[r // 128:r // 128 + s.shape[0]] = s
        q[r:r + rows, :K] = (blocks / s[:, None, :, None]).view(-1, kb * 128)[:rows, :K].to(torch.float8_e4m3fn).view(torch.uint8)
    return q, scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 17)
    n, V = case["n"], case["V"]
    state = {"case": case, "mask": _masks(gen, case["mask"], n, V)}
    f32 = dict(dtype=torch.float32, device="cuda")
    if case["kind"] == "head":
        K = case["K"]
        stride, kb = (K + 15) // 16 * 16, (K + 127) // 128
        loud = 1.0 + 7.0 * (torch.rand((1, K), generator=gen, device="cuda") < 0.01)  # a few channels are far larger
        state["hidden"] = (torch.randn((n, K), generator=gen, device="cuda") * loud).to(torch.bfloat16)
        state["weights"], state["weight_scales"] = _quantized_weights(gen, V, K, stride)
        # what a program keeps for every step
        state["q"] = torch.zeros((n, stride), dtype=torch.uint8, device="cuda")
        state["scales"] = torch.zeros((kb, n), **f32)
        state["logits"] = torch.empty((n, V), dtype=_dtype(case), device="cuda")
        return state
    logits = torch.empty((n, V), dtype=_dtype(case), device="cuda")
    for r in range(0, n, 256):
        rows = min(256, n - r)
        x = torch.randn((rows, V), generator=gen, device="cuda") * 2.5
        peaks = torch.randint(0, V, (rows, 8), generator=gen, device="cuda")
        x.scatter_add_(1, peaks, 6.0 + 6.0 * torch.rand((rows, 8), generator=gen, device="cuda"))
        logits[r:r + rows] = x.to(logits.dtype)
    tokens = torch.randint(0, V, (n, case["tokens"]), generator=gen, device="cuda", dtype=torch.int32)
    tokens[:, 0] = (torch.arange(n, device="cuda") // 64 * 64 % V).to(torch.int32)  # one that the mask allows (see _masks)
    state.update(logits=logits, tokens=tokens)
    state["temperature"] = 0.5 + torch.rand(n, generator=gen, device="cuda") if case["heat"] else None
    state["logprobs"] = torch.empty((n, case["tokens"]), **f32)
    state["norm"], state["entropy"] = torch.empty((n, 2), **f32), torch.empty(n, **f32)
    if case["kind"] == "train":
        state["grad_logprobs"] = torch.randn((n, case["tokens"]), generator=gen, device="cuda")
        state["grad_entropy"] = 0.1 * torch.randn(n, generator=gen, device="cuda")
        state["grad_logits"] = torch.empty_like(logits)
    else:
        state["top_ids"] = torch.empty((n, case["top"]), dtype=torch.int32, device="cuda")
        state["top_logprobs"] = torch.empty((n, case["top"]), **f32)
    return state


# ------------------------------------------------------------------------------------------------ one pass


def run(state):
    kind = state["case"]["kind"]
    return (_own if own else _plain)[kind](state)


def _own_head(s):
    import paper_2506_01151_b200 as fmt

    c = s["case"]
    fmt.quantize_blocks(s["hidden"], fmt.BF16, c["n"], c["K"], 1, s["q"], s["scales"], q_stride=s["q"].shape[1])
    fmt.head_logits(s["q"], s["scales"], s["weights"], s["weight_scales"], s["logits"], fmt.BF16 if c["dtype"] == "bf16" else fmt.FP32,
                    c["n"], c["V"], c["K"], mask_dev=s["mask"], hidden_stride=s["q"].shape[1], weight_stride=s["weights"].shape[1])
    return s["logits"]


def _own_score(s):
    import paper_2506_01151_b200 as fmt

    c = s["case"]
    fmt.token_logprobs(s["logits"], fmt.BF16 if c["dtype"] == "bf16" else fmt.FP32, c["n"], c["V"], tokens_dev=s["tokens"], n_tokens=c["tokens"],
                       logprobs_dev=s["logprobs"], norm_dev=s["norm"], entropy_dev=s["entropy"], n_top=c["top"], top_ids_dev=s["top_ids"],
                       top_logprobs_dev=s["top_logprobs"], mask_dev=s["mask"], temperature_dev=s["temperature"])
    return s["logprobs"], s["norm"], s["entropy"], s["top_ids"], s["top_logprobs"]


def _own_train(s):
    import paper_2506_01151_b200 as fmt

    c = s["case"]
    dtype = fmt.BF16 if c["dtype"] == "bf16" else fmt.FP32
    fmt.token_logprobs(s["logits"], dtype, c["n"], c["V"], tokens_dev=s["tokens"], n_tokens=c["tokens"], logprobs_dev=s["logprobs"],
                       norm_dev=s["norm"], entropy_dev=s["entropy"], mask_dev=s["mask"], temperature_dev=s["temperature"])
    fmt.token_logprobs_backward(s["logits"], dtype, c["n"], c["V"], s["norm"], s["grad_logits"], tokens_dev=s["tokens"], n_tokens=c["tokens"],
                                grad_logprobs_dev=s["grad_logprobs"], entropy_dev=s["entropy"], grad_entropy_dev=s["grad_entropy"],
                                mask_dev=s["mask"], temperature_dev=s["temperature"])
    return s["logprobs"], s["norm"], s["entropy"], s["grad_logits"]


def _allowed(mask, r, rows, V):
    """Truth values [rows, V] of the packed masks, or None."""
    if mask is None:
        return None
    shift = torch.arange(32, device=mask.device, dtype=torch.int32)
    return ((mask[r:r + rows, :, None] >> shift) & 1).view(rows, -1)[:, :V].bool()


ROWS = 256  # of a plain form's piece: its values in 32 bits are several times the logits


def _plain_head(s):
    c = s["case"]
    n, V, K = c["n"], c["V"], c["K"]
    kb = (K + 127) // 128
    x = torch.zeros((n, kb * 128), device="cuda")
    x[:, :K] = s["hidden"].float()
    x = x.view(n, kb, 128)
    scale = x.abs().amax(-1)
    scale = scale / torch.full_like(scale, 448.0)  # a quotient in IEEE single precision (by a number, torch multiplies with its reciprocal)
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    x = ((x / scale[..., None]).to(torch.float8_e4m3fn).float() * scale[..., None]).view(n, kb * 128)[:, :K]
    out = s["logits"]
    for v in range(0, V, 32768):
        rows = min(32768, V - v)
        w = s["weights"][v:v + rows, :K].view(torch.float8_e4m3fn).float()
        blocks = s["weight_scales"][v // 128:(v + rows + 127) // 128].repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :K]
        out[:, v:v + rows] = (x @ (w * blocks).t()).to(out.dtype)
    if s["mask"] is not None:
        for r in range(0, n, ROWS):
            allowed = _allowed(s["mask"], r, min(ROWS, n - r), V)
            out[r:r + ROWS] = torch.where(allowed, out[r:r + ROWS], -math.inf)
    return out


def _order(x):
    """Whole numbers in the order of the floats."""
    bits = x.view(torch.int32).to(torch.int64)
    return torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)


def _plain_distribution(s, r, rows):
    """The piece's logits, what is allowed, and (logits - largest) / temperature, ln of the sum, log probabilities, entropy."""
    V = s["case"]["V"]
    x = s["logits"][r:r + rows].float()
    allowed = _allowed(s["mask"], r, rows, V)
    if allowed is not None:
        x = torch.where(allowed, x, -math.inf)
    T = s["temperature"][r:r + rows, None] if s["temperature"] is not None else torch.ones((rows, 1), device="cuda")
    largest = x.amax(-1, keepdim=True)
    d = (x - largest) / T
    p = torch.exp(d)
    ln = torch.log(p.sum(-1, keepdim=True))
    logp = d - ln
    p = torch.exp(logp)
    entropy = -(p * torch.where(p > 0, logp, torch.zeros_like(logp))).sum(-1)
    return x, T, largest, ln, logp, p, entropy


def _plain_score(s):
    c = s["case"]
    n, V = c["n"], c["V"]
    for r in range(0, n, ROWS):
        rows = min(ROWS, n - r)
        x, T, largest, ln, logp, p, entropy = _plain_distribution(s, r, rows)
        s["logprobs"][r:r + rows] = torch.gather(logp, 1, s["tokens"][r:r + rows].long())
        s["norm"][r:r + rows] = torch.cat([largest, ln], 1)
        s["entropy"][r:r + rows] = entropy
        if c["top"]:
            key = _order(x + 0.0) * (1 << 20) - torch.arange(V, device="cuda")  # the lowest index first among equals
            at = torch.topk(key, min(c["top"], V), 1).indices
            got = torch.gather(logp, 1, at)
            k = at.shape[1]
            s["top_ids"][r:r + rows] = -1
            s["top_logprobs"][r:r + rows] = -math.inf
            s["top_ids"][r:r + rows, :k] = torch.where(torch.gather(x, 1, at) == -math.inf, -1, at).to(torch.int32)
            s["top_logprobs"][r:r + rows, :k] = got
    return s["logprobs"], s["norm"], s["entropy"], s["top_ids"], s["top_logprobs"]


def _plain_train(s):
    c = s["case"]
    for r in range(0, c["n"], ROWS):
        rows = min(ROWS, c["n"] - r)
        x, T, largest, ln, logp, p, entropy = _plain_distribution(s, r, rows)
        tokens = s["tokens"][r:r + rows].long()
        got = torch.gather(logp, 1, tokens)
        s["logprobs"][r:r + rows] = got
        s["norm"][r:r + rows] = torch.cat([largest, ln], 1)
        s["entropy"][r:r + rows] = entropy
        g = torch.where(got > -math.inf, s["grad_logprobs"][r:r + rows], torch.zeros_like(got))  # a forbidden token's is a constant
        dx = -p * g.sum(-1, keepdim=True)
        dx -= s["grad_entropy"][r:r + rows, None] * p * torch.where(p > 0, logp + entropy[:, None], torch.zeros_like(p))
        dx.scatter_add_(1, tokens, g)
        s["grad_logits"][r:r + rows] = (dx / T).to(s["grad_logits"].dtype)
    return s["logprobs"], s["norm"], s["entropy"], s["grad_logits"]


_own = {"head": _own_head, "score": _own_score, "train": _own_train}
_plain = {"head": _plain_head, "score": _plain_score, "train": _plain_train}


# ------------------------------------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    n, V = case["n"], case["V"]
    f64 = dict(dtype=torch.float64, device="cuda")

    def bits(r, rows):
        if s["mask"] is None:
            return torch.ones((rows, V), dtype=torch.bool, device="cuda")
        t = torch.arange(V, device="cuda")
        return ((s["mask"][r:r + rows].long()[:, t >> 5] >> (t & 31)) & 1) == 1

    if case["kind"] == "head":
        K = case["K"]
        out = torch.empty((n, V), **f64)
        # 8-bit values and scales are what the definition says, to the bit: quotients in IEEE single precision
        piece = s["hidden"].float()
        x = torch.zeros((n, K), **f64)
        for k in range(0, K, 128):
            b = piece[:, k:k + 128]
            scale = b.abs().max(1, keepdim=True).values
            scale = scale / torch.full_like(scale, 448.0)
            scale[scale == 0] = 1.0
            x[:, k:k + 128] = (b / scale).to(torch.float8_e4m3fn).double() * scale.double()
        for v in range(0, V, 4096):
            rows = min(4096, V - v)
            w = s["weights"][v:v + rows, :K].view(torch.float8_e4m3fn).double()
            for i in range(0, rows, 128):
                ws = s["weight_scales"][(v + i) // 128].double()
                w[i:i + 128] *= ws.repeat_interleave(128)[None, :K]
            out[:, v:v + rows] = x @ w.t()
        for r in range(0, n, 128):
            out[r:r + 128].masked_fill_(~bits(r, min(128, n - r)), -math.inf)
        return out

    logprobs, norm, entropy = torch.empty((n, case["tokens"]), **f64), torch.empty((n, 2), **f64), torch.empty(n, **f64)
    top = case["top"]
    ids = torch.full((n, top), -1, dtype=torch.int32, device="cuda")
    tops = torch.full((n, top), -math.inf, **f64)
    grad = torch.empty((n, V), **f64) if case["kind"] == "train" else None
    for r in range(0, n, 64):
        rows = min(64, n - r)
        ok = bits(r, rows)
        x = s["logits"][r:r + rows].double().masked_fill(~ok, -math.inf)
        T = s["temperature"][r:r + rows].double()[:, None] if case["heat"] else torch.ones((rows, 1), **f64)
        most = x.max(1, keepdim=True).values
        e = torch.exp((x - most) / T)
        total = e.sum(1, keepdim=True)
        p = e / total
        lp = (x - most) / T - torch.log(total)
        at = s["tokens"][r:r + rows].long()
        logprobs[r:r + rows] = torch.gather(lp, 1, at)
        norm[r:r + rows, 0], norm[r:r + rows, 1] = most[:, 0], torch.log(total)[:, 0]
        H = -(p * lp.masked_fill(~ok, 0.0)).sum(1)
        entropy[r:r + rows] = H
        if top:
            order = torch.sort(x, dim=1, descending=True, stable=True)
            k = min(top, V)
            ids[r:r + rows, :k] = order.indices[:, :k].masked_fill(order.values[:, :k] == -math.inf, -1).to(torch.int32)
            tops[r:r + rows, :k] = torch.gather(lp, 1, order.indices[:, :k])
        if grad is not None:
            g = s["grad_logprobs"][r:r + rows].double()
            d = torch.zeros((rows, V), **f64)
            for t in range(case["tokens"]):
                here = at[:, t:t + 1]
                weight = g[:, t:t + 1] * torch.gather(ok, 1, here)
                d -= weight * p
                d.scatter_add_(1, here, weight)
            d -= s["grad_entropy"][r:r + rows].double()[:, None] * p * (lp.masked_fill(~ok, 0.0) + H[:, None])
            grad[r:r + rows] = d / T
    if case["kind"] == "train":
        return logprobs, norm, entropy, grad
    return logprobs, norm, entropy, ids, tops
