"""Log probabilities under the mask and their gradient (fmt_token_logprobs, fmt_token_logprobs_backward) against the formulas in
64 bits, and what the two refuse.

Tolerances, with u = 2^-24 (half a unit of fp32).  d = (x - M) / T takes three roundings: 3 u |d|, and exp turns that into the
same relative error, plus 2 units of its own.  Sums of V terms are made of chains of at most V / 128 additions per thread and a
tree: (V / 128 + 32) u relative for sums of terms of one sign.  So with A = V / 128 + 64 (the rest of the constants included):
  ln p           u (4 |d| + A + 4 dm),       dm = the largest |d| whose exp is not 0 (at most 104)
  entropy        u (A + 4 dm) (2 + H)        (ln S and -t / S are both not negative: nothing cancels)
  gradient       p (u (4 |ln p| + A + 4 dm)) (|sum g| + |g_H| (|ln p| + H + 2)) / T + 4 u sum |g| / T (given tokens)
and half a step of the output's type on top.
"""
import numpy as np
import pytest

import paper_2506_01151_b200 as fmt

U = 2.0 ** -24
gpu = pytest.mark.gpu


def torch_():
    import torch

    return torch


DEV = "cuda:0"


class Inputs:
    """Logits in rows of any stride from any address, packed masks, temperatures, tokens."""

    def __init__(self, n, V, dtype="bf16", mask="mixed", stride=None, offset=0, heat=True, n_tokens=2, seed=0, mask_pad=0, scale=2.5):
        torch = torch_()
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.n, self.V, self.n_tokens = n, V, n_tokens
        self.dtype = fmt.BF16 if dtype == "bf16" else fmt.FP32
        self.type = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.stride = V if stride is None else stride
        self.store = torch.full((offset + max(n, 1) * self.stride + 8,), float("nan"), dtype=self.type, device=DEV)
        self.logits = self.store[offset:].as_strided((n, V), (self.stride, 1))
        self.logits.copy_((torch.randn((n, V), generator=g, device=DEV) * scale).to(self.type))
        self.words = (V + 31) // 32
        self.mask_stride = self.words + mask_pad
        share = {"none": 1.0, "all": 1.0, "mixed": 0.5, "few": min(1.0, 3.0 / V)}[mask]
        self.allow = torch.rand((n, V), generator=g, device=DEV) < share
        self.masked = mask != "none"
        self.temperature = 0.3 + torch.rand(n, generator=g, device=DEV) * 2 if heat else None
        self.tokens = torch.randint(0, V, (n, n_tokens), generator=g, device=DEV, dtype=torch.int32)
        self.g = torch.randn((n, n_tokens), generator=g, device=DEV)
        self.gh = torch.randn(n, generator=g, device=DEV)

    def mask(self):
        """The packed masks; what lies behind a row's words is all ones, and so are the bits beyond V."""
        torch = torch_()
        if not self.masked:
            return None
        bits = torch.ones((self.n, self.mask_stride * 32), dtype=torch.int64, device=DEV)
        bits[:, : self.V] = self.allow.long()
        w = (bits.view(self.n, -1, 32) << torch.arange(32, device=DEV)).sum(-1)
        return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)

    def kw(self, **more):
        return dict(dict(mask_dev=self.mask(), stride_words=self.mask_stride, row_stride=self.stride, temperature_dev=self.temperature), **more)

    def forward(self, n_top=5, stream=None, into=None):
        torch = torch_()
        f = dict(dtype=torch.float32, device=DEV)
        out = into or {
            "logprobs": torch.full((self.n + 1, self.n_tokens), 77.0, **f), "norm": torch.full((self.n + 1, 2), 77.0, **f),
            "entropy": torch.full((self.n + 1,), 77.0, **f), "ids": torch.full((self.n + 1, n_top), 77, dtype=torch.int32, device=DEV),
            "tops": torch.full((self.n + 1, n_top), 77.0, **f), "status": torch.full((self.n + 1,), 77, dtype=torch.int32, device=DEV)}
        fmt.token_logprobs(self.logits, self.dtype, self.n, self.V, tokens_dev=self.tokens, n_tokens=self.n_tokens, logprobs_dev=out["logprobs"],
                           norm_dev=out["norm"], entropy_dev=out["entropy"], n_top=n_top, top_ids_dev=out["ids"], top_logprobs_dev=out["tops"],
                           status_dev=out["status"], stream=stream, **self.kw())
        return out

    def backward(self, out, grad=None, in_place=False, grad_stride=None, with_g=True, with_h=True, stream=None):
        torch = torch_()
        gs = self.stride if in_place else (grad_stride or self.V)
        if in_place:
            grad = self.logits
        elif grad is None:
            self.grad_store = torch.full((self.n * gs + 8,), 77.0, dtype=self.type, device=DEV)
            grad = self.grad_store.as_strided((self.n, self.V), (gs, 1))
        fmt.token_logprobs_backward(self.logits, self.dtype, self.n, self.V, out["norm"], grad, tokens_dev=self.tokens, n_tokens=self.n_tokens,
                                    grad_logprobs_dev=self.g if with_g else None, entropy_dev=out["entropy"],
                                    grad_entropy_dev=self.gh if with_h else None, grad_stride=gs, stream=stream, **self.kw())
        return grad

    def reference(self, n_top=5, with_g=True, with_h=True):
        """Everything in 64 bits from the definition, with the bounds above."""
        torch = torch_()
        n, V = self.n, self.V
        x = self.logits.double()
        allow = self.allow if self.masked else torch.ones_like(self.allow)
        x = torch.where(allow, x, -torch.inf)
        T = self.temperature.double()[:, None] if self.temperature is not None else torch.ones((n, 1), dtype=torch.float64, device=DEV)
        allow = x != -torch.inf
        bad = (~(x < torch.inf)).any(1) | ~((T[:, 0] > 0) & (T[:, 0] < torch.inf))
        M = x.max(1, keepdim=True).values
        none = M[:, 0] == -torch.inf
        d = torch.where(allow, (x - M) / T, -torch.inf)
        S = torch.exp(d).sum(1, keepdim=True)
        lp = torch.where(allow, d - torch.log(S), -torch.inf)
        p = torch.where(allow, torch.exp(lp), 0.0)
        H = -torch.where(p > 0, p * lp, 0.0).sum(1)
        tok = self.tokens.long()
        inside = (tok >= 0) & (tok < V)
        at = tok.clamp(0, V - 1)
        got = torch.where(inside, torch.gather(lp, 1, at), torch.where(tok == -1, 0.0, torch.nan))
        got = torch.where(bad[:, None] & (tok != -1), torch.nan, got)
        order = torch.sort(x + 0.0, dim=1, descending=True, stable=True)
        k = min(n_top, V)
        ids = torch.full((n, n_top), -1, dtype=torch.int64, device=DEV)
        tops = torch.full((n, n_top), -torch.inf, dtype=torch.float64, device=DEV)
        ids[:, :k] = torch.where(order.values[:, :k] == -torch.inf, -1, order.indices[:, :k])
        tops[:, :k] = torch.where(ids[:, :k] >= 0, torch.gather(lp, 1, order.indices[:, :k]), -torch.inf)
        ids[bad], tops[bad] = -1, torch.nan
        norm = torch.cat([M, torch.log(S)], 1)
        norm[bad] = torch.nan
        H = torch.where(bad, torch.nan, torch.where(none, 0.0, H))
        status = torch.where(bad | ((tok < -1) | (tok >= V)).any(1), fmt.ERR_INVALID_ARG, fmt.FMT_OK)
        g = torch.where(inside & (torch.gather(lp, 1, at).float() > -torch.inf), self.g.double() * with_g, 0.0)
        gh = self.gh.double()[:, None] * with_h
        total = g.sum(1, keepdim=True)
        grad = -p * total - gh * p * torch.where(p > 0, lp + H[:, None], 0.0)
        grad.scatter_add_(1, at, g)
        grad = torch.where(allow, torch.where(bad[:, None], torch.nan, grad / T), 0.0)
        A = V / 128 + 64
        dm = torch.where(torch.exp(d) > 1e-45, d.abs(), 0.0).nan_to_num(0, 0, 0).amax(1, keepdim=True).clamp(max=104)
        ad = d.abs().nan_to_num(0, 0, 0)
        tol_lp = U * (4 * ad + A + 4 * dm)
        e = U * (4 * lp.abs().nan_to_num(0, 0, 0) + A + 4 * dm)
        ag = torch.zeros_like(p).scatter_add_(1, at, g.abs())
        tol_grad = (p * e * (g.abs().sum(1, keepdim=True) + gh.abs() * (lp.abs().nan_to_num(0, 0, 0) + H.abs()[:, None] + 2)) + 4 * U * ag) / T
        return {"logprobs": got, "norm": norm, "entropy": H, "ids": ids, "tops": tops, "status": status, "grad": grad,
                "tol": {"logprobs": torch.gather(tol_lp, 1, at), "norm": torch.cat([U * M.abs(), U * (A + 4 * dm)], 1),
                        "entropy": U * (A + 4 * dm[:, 0]) * (2 + H), "tops": torch.gather(tol_lp, 1, ids.clamp(min=0)), "grad": tol_grad}}


def near(got, want, tol, what, half=U):
    torch = torch_()
    if got.dtype == torch.float32:  # what is beyond the type's range (the lowest logit over a temperature below 1) is rounded to an infinity
        want = torch.where(torch.isinf(want.float()), want.float().double(), want)
    got = got.double()
    odd = ~torch.isfinite(want)
    same = torch.where(torch.isnan(want), torch.isnan(got), got == want)
    assert bool(same[odd].all()), (what, "infinities or NaN", torch.nonzero(~same & odd)[:4].tolist())
    err = (got - want).abs()[~odd]
    limit = (tol + half * want.abs() + 1e-40)[~odd]
    assert bool((err <= limit).all()), (what, float((err / limit).max()), float(err.max()))


def check_forward(i, out, n_top=5):
    torch = torch_()
    want = i.reference(n_top)
    n = i.n
    for k in ("logprobs", "norm", "entropy", "tops"):
        near(out[k][:n], want[k], want["tol"][k].nan_to_num(0, 0, 0), k)
        assert bool((out[k][n:] == 77).all()), "behind the last row"
    assert torch.equal(out["ids"][:n].long(), want["ids"]) and torch.equal(out["status"][:n].long(), want["status"])
    assert bool((out["ids"][n:] == 77).all()) and bool((out["status"][n:] == 77).all())
    return want


def check_backward(i, grad, want):
    half = torch_().finfo(i.type).eps / 2
    tiny = 2.0 ** -133 if i.dtype == fmt.BF16 else 2.0 ** -149  # what is left of denormals
    near(grad, want["grad"], want["tol"]["grad"].nan_to_num(0, 0, 0) + tiny, "grad", half)


SHAPES = [(1, 1), (3, 2), (2, 31), (5, 33), (1, 512), (7, 1000), (4, 4099), (37, 50001), (200, 777), (2, 128256), (300, 9001)]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("mask", ["none", "mixed", "few"])
@pytest.mark.parametrize("n,V", SHAPES)
def test_forward_and_gradient(n, V, mask, dtype):
    i = Inputs(n, V, dtype, mask, seed=n * 7 + V, heat=V % 2 == 1)
    out = i.forward()
    want = check_forward(i, out)
    check_backward(i, i.backward(out), want)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5), (5, 1), (7, 9), (8, 16)])
@pytest.mark.parametrize("V", [7, 250, 4099, 20000])
def test_rows_begin_at_any_address(V, offset, pad, dtype):
    i = Inputs(6, V, dtype, "mixed", stride=V + pad, offset=offset, mask_pad=pad % 3, seed=offset + V)
    before = i.store.clone()
    out = i.forward(9)
    want = check_forward(i, out, 9)
    grad = i.backward(out, grad_stride=V + pad)
    check_backward(i, grad, want)
    torch = torch_()
    edge = torch.ones_like(i.grad_store, dtype=torch.bool)
    edge.as_strided((6, V), (V + pad, 1))[:] = False
    assert bool((i.grad_store[edge] == 77).all()), "between the rows"
    assert torch.equal(before.view(torch.uint8), i.store.view(torch.uint8)), "the logits are only read"
    check_backward(i, i.backward(out, in_place=True), want)
    edge = torch.ones_like(i.store, dtype=torch.bool)
    edge[offset:].as_strided((6, V), (V + pad, 1))[:] = False
    assert bool(torch.isnan(i.store[edge]).all()), "between the rows"


@gpu
@pytest.mark.parametrize("V", [40, 6000, 60000])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_that_are_out_of_the_ordinary(V, dtype):
    torch = torch_()
    i = Inputs(17, V, dtype, "mixed", n_tokens=6, seed=V)
    low = torch.finfo(i.type).min
    nan, inf = float("nan"), float("inf")
    x, a = i.logits, i.allow
    a[0] = False                                      # nothing allowed
    a[1] = False; a[1, V - 1] = True                  # one token, the last
    a[2] = True; x[2] = 1.5                           # all alike
    a[3] = True; x[3] = low                           # all the type's lowest value
    x[4] = torch.where(torch.rand(V, device=DEV) < 0.9, torch.full_like(x[4], low), x[4])
    a[5] = True; x[5] = -inf                          # nothing left, and no mask says so
    x[6][~a[6]] = nan                                 # what is not allowed is not looked at
    x[7][~a[7]] = inf
    a[8, 3] = True; x[8, 3] = nan                     # an allowed NaN
    a[9, 4] = True; x[9, 4] = inf
    i.temperature[10], i.temperature[11], i.temperature[12], i.temperature[13] = 0.0, -1.0, nan, inf
    i.tokens[14] = torch.tensor([-1, V, -2, 5, 5, 2 ** 31 - 1], device=DEV, dtype=torch.int32)
    a[14, 5] = True
    i.tokens[15] = 7; a[15, 7] = True                 # one token six times
    a[16] = True; x[16] = torch.where(torch.arange(V, device=DEV) % 2 == 0, 0.0, -0.0).to(i.type)  # 0 and -0 are equal
    out = i.forward(7)
    want = check_forward(i, out, 7)
    assert out["ids"][16].tolist() == list(range(7)) and out["ids"][2].tolist() == list(range(7))
    check_backward(i, i.backward(out), want)


@gpu
@pytest.mark.parametrize("n_top", [1, 2, 31, 32])
@pytest.mark.parametrize("order", ["up", "down", "ties", "one place", "stripes"])
def test_alternatives_wherever_they_lie(order, n_top):
    """The largest logits side by side, far apart, in one thread's part, among many equals."""
    torch = torch_()
    V = 30011
    i = Inputs(3, V, "fp32", "none", heat=False, n_tokens=1, seed=n_top)
    at = torch.arange(V, device=DEV, dtype=torch.float32)
    x = {"up": at / V, "down": -at / V, "ties": (at % 13).floor() - (at % 7 == 3) * 5, "one place": torch.where((at >= 9000) & (at < 9050), 9050 - at, at * 1e-6),
         "stripes": torch.where(at % 1024 == 5, 3 + at / V, at * 1e-6)}[order]
    i.logits[:] = x
    i.logits[1] = x.flip(0)
    i.logits[2] = torch.roll(x, 12345)
    check_forward(i, i.forward(n_top), n_top)
    j = Inputs(3, V, "bf16", "few", heat=False, n_tokens=1, seed=n_top)  # fewer than asked for
    check_forward(j, j.forward(n_top), n_top)


@gpu
@pytest.mark.parametrize("n", [2, 600])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("every,of", [(64, 256), (512, 2048), (1, 4), (3, 97)])
def test_alternatives_crowded_in_some_places(every, of, dtype, n):
    """Thousands of logits that are larger than all others, side by side in stretches of 32 bytes: more than any list holds."""
    torch = torch_()
    V = 40000
    i = Inputs(n, V, dtype, "mixed" if every == 1 else "none", heat=False, n_tokens=1, seed=every)
    unit = torch.arange(V, device=DEV) // (16 if dtype == "bf16" else 8)
    i.logits += torch.where(unit % of < every, 40.0, 0.0).to(i.type)
    for n_top in (20, 32):
        check_forward(i, i.forward(n_top), n_top)


@gpu
@pytest.mark.parametrize("temperature", [1e-30, 1e-9, 1.9e-6, 1e-3, 1e4, 1.5e8, 1e30])
@pytest.mark.parametrize("scale,shift", [(1.0, 0.0), (1.0, -2e11), (1e12, 0.0), (1e20, -1e21), (1e-20, 0.0), (3e37, 0.0)])
def test_extreme_temperatures_and_logits(scale, shift, temperature):
    i = Inputs(3, 5003, "fp32", "mixed", seed=7, scale=scale)
    i.logits += shift
    i.temperature[:] = temperature
    out = i.forward()
    want = check_forward(i, out)
    if scale * 10 / temperature < 1e30 and 1e-20 < temperature:  # (where the gradient, or the exponents' errors, are no numbers of fp32)
        check_backward(i, i.backward(out), want)


@gpu
@pytest.mark.parametrize("mask", ["none", "mixed"])
def test_temperatures_that_are_not_normal_numbers(mask):
    torch = torch_()
    i = Inputs(4, 700, "fp32", mask, seed=2)
    i.temperature[0], i.temperature[1], i.temperature[2] = 1.1754942e-38, 1e-40, 2.0 ** -126  # the first is just below
    i.allow[:, 5] = True
    out = i.forward()
    assert out["status"][:4].tolist() == [fmt.ERR_INVALID_ARG, fmt.ERR_INVALID_ARG, fmt.FMT_OK, fmt.FMT_OK]
    assert bool(torch.isnan(out["logprobs"][:2]).all()) and bool((out["ids"][:2] == -1).all()) and bool(torch.isnan(out["norm"][:2]).all())
    assert float(out["tops"][2, 0]) == 0.0 and not bool(torch.isnan(out["logprobs"][2]).any())


def check_gradient_of_any_size(i, out):
    """The gradient where 1 / T or the gradients that come in are large: a p that fp32 does not hold (below 2^-149) counts as 0, and what is
    left of one that it holds as a denormal is off by half of 2^-149, each times what it is multiplied with."""
    want = i.reference()
    norm, T = want["norm"], i.temperature.double()[:, None]
    lp = ((i.logits.double() - norm[:, :1]) / T - norm[:, 1:]).abs().nan_to_num(0, 0, 0).clamp(max=104)
    H = want["entropy"].abs()[:, None]
    less = 2.0 ** -149 * (i.g.double().abs().sum(1, keepdim=True) + i.gh.double().abs()[:, None] * (lp + H + 2)) / T
    allow = i.allow if i.masked else torch_().ones_like(i.allow)
    want["tol"]["grad"] = want["tol"]["grad"] + torch_().where(allow, less, 0.0)
    grad = i.backward(out)
    check_backward(i, grad, want)
    assert bool((grad[~allow] == 0).all())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("mask", ["none", "mixed", "few"])
@pytest.mark.parametrize("temperature,g,gh", [(2.0 ** -126, 0.5, 1.0), (1e-37, 0.5, 1.0), (1e-37, 0.5, -8.0), (1e-30, 1.0, 1.0), (1e-12, 1.0, 1.0),
                                              (2e-6, 1.0, 1e18), (1.0, 1.0, 1e28), (1.0, 1e33, 1e33), (0.7, 1e30, 0.0), (1e30, 1e33, -1e33)])
def test_gradients_that_are_large(temperature, g, gh, mask, dtype):
    """1 / T, or a gradient by the entropy, that is large: 0 where nothing is allowed or p is 0, and no overflow on the way to a number."""
    torch = torch_()
    i = Inputs(6, 5003, dtype, mask, offset=3, n_tokens=3, seed=11)
    i.temperature[:] = temperature
    if mask != "few":
        i.allow[:, :4] = True
        i.logits[3:, 2] = 20.0  # the likeliest by far
    i.g.clamp_(-1, 1).mul_(g)
    i.gh.clamp_(-1, 1).mul_(gh)
    i.tokens[3:, 0] = 2
    i.tokens[4:, 1] = 2
    check_gradient_of_any_size(i, i.forward())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("by", ["g", "gh"])
def test_gradients_that_are_not_finite_reach_allowed_tokens_only(by, value, dtype):
    torch = torch_()
    i = Inputs(4, 3001, dtype, "mixed", offset=1, seed=12)
    i.allow[:, :8] = True
    i.tokens[:] = torch.tensor([1, 6], dtype=torch.int32, device=DEV)
    i.logits[:, 10:40] = -float("inf")
    out = i.forward()
    getattr(i, by)[1] = value
    grad = i.backward(out)
    off = ~i.allow | (i.logits == -torch.inf)
    assert bool((grad[off] == 0).all())
    assert not bool(torch.isfinite(grad[1][~off[1]]).any())
    assert bool(torch.isfinite(grad[[0, 2, 3]]).all())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("temperature", [1.0, 3.0, 1e8, 1e30, 1e37, 2e38, 3.4e38])
def test_logits_farther_apart_than_the_largest_number(temperature, dtype):
    """x - M may be beyond fp32 where (x - M) / T is not."""
    torch = torch_()
    i = Inputs(5, 4099, dtype, "mixed", offset=1, n_tokens=4, seed=13, scale=1.0)
    i.logits.copy_((i.logits.float().clamp(-3.3, 3.3) * 1e38).to(i.type))
    i.allow[:, :4] = True
    i.logits[:, 0], i.logits[:, 1] = torch.finfo(i.type).max, torch.finfo(i.type).min
    i.tokens[:, 0], i.tokens[:, 1] = 0, 1
    i.temperature[:] = temperature
    out = i.forward()
    check_forward(i, out)
    check_gradient_of_any_size(i, out)


@gpu
@pytest.mark.parametrize("mask", ["none", "all"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_long_rows_of_equal_logits(dtype, mask):
    """As many equal logits as a server's largest batch leaves to one thread block, behind a few that are larger, some for each thread: the
    terms of a thread are all the same then, and a chain of additions would round each of them the same way.  A thread adds up 32 terms
    (17 roundings at most, by pairs), and then those sums, V / 8,192 of them (fp32: half as many terms, twice as many sums); 13 more roundings
    join the threads of a block.  The terms themselves are off by 4 |d| + 4 units (what d takes, and exp), the logarithm by two of its own."""
    torch = torch_()
    V, n, large = 1 << 18, 320, 1024
    i = Inputs(n, V, dtype, mask, heat=False, n_tokens=1, seed=14)
    at = -0.25 - torch.arange(n, device=DEV, dtype=torch.float32) / 128  # (what bf16 makes of it is the input)
    i.logits[:] = at.to(i.type)[:, None]
    i.logits[:, : 8 * large : 8] = 0.0
    norm, entropy = torch.zeros((n, 2), device=DEV), torch.zeros(n, device=DEV)
    fmt.token_logprobs(i.logits, i.dtype, n, V, norm_dev=norm, entropy_dev=entropy, mask_dev=i.mask())
    d = i.logits[:, 1].double()
    S = large + (V - large) * torch.exp(d)
    H = torch.log(S) - (V - large) * d * torch.exp(d) / S
    unit = U * (17 + V / (8192 if dtype == "bf16" else 4096) + 13 + 4 * d.abs() + 4)  # relative, of S and of the sum of p d
    err, limit = (norm[:, 1].double() - torch.log(S)).abs(), unit + 2 * U * torch.log(S)
    assert bool((err <= limit).all()), float((err / limit).max())
    err, limit = (entropy.double() - H).abs(), (2 * unit + 4 * U) * (2 + H)
    assert bool((err <= limit).all()), float((err / limit).max())


@gpu
@pytest.mark.parametrize("n_tokens", [0, 1, 32])
@pytest.mark.parametrize("with_g,with_h", [(True, False), (False, True), (False, False)])
def test_gradients_that_are_not_given(n_tokens, with_g, with_h):
    i = Inputs(5, 3001, "fp32", "mixed", n_tokens=n_tokens, seed=n_tokens)
    out = i.forward(0)
    want = i.reference(0, with_g, with_h)
    check_backward(i, i.backward(out, with_g=with_g, with_h=with_h), want)


@gpu
def test_outputs_that_are_not_asked_for():
    torch = torch_()
    i = Inputs(9, 5003, "bf16", "mixed", n_tokens=1)
    full = i.forward(1)
    ids = torch.full((9,), 77, dtype=torch.int32, device=DEV)
    fmt.token_logprobs(i.logits, i.dtype, 9, i.V, n_top=1, top_ids_dev=ids, **i.kw())
    assert torch.equal(ids, full["ids"][:9, 0])
    lp = torch.full((9, 1), 77.0, device=DEV)
    fmt.token_logprobs(i.logits, i.dtype, 9, i.V, tokens_dev=i.tokens, n_tokens=1, logprobs_dev=lp, n_top=7, **i.kw())
    assert torch.equal(lp, full["logprobs"][:9])
    fmt.token_logprobs(i.logits, i.dtype, 9, i.V, **i.kw())  # nothing asked for
    fmt.token_logprobs(i.logits, i.dtype, 0, i.V, tokens_dev=i.tokens, n_tokens=1, logprobs_dev=lp, **i.kw())
    assert torch.equal(lp, full["logprobs"][:9])


@gpu
def test_gradient_by_differences():
    """Central differences of the 64-bit loss, apart from the formula of the gradient."""
    torch = torch_()
    i = Inputs(2, 60, "fp32", "mixed", n_tokens=3, seed=5)
    i.allow[:, :8] = True
    i.tokens[:] = torch.tensor([[1, 1, 5], [0, -1, 7]], dtype=torch.int32, device=DEV)
    out = i.forward(0)
    grad = i.backward(out).double()
    T, ok = i.temperature.double()[:, None], i.tokens.long() >= 0

    def loss(x):
        lp = torch.log_softmax(torch.where(i.allow, x, -torch.inf) / T, 1)
        p = lp.exp()
        h = -(p * lp.masked_fill(~i.allow, 0)).sum(1)
        return (torch.where(ok, torch.gather(lp, 1, i.tokens.long().clamp(min=0)), 0.0) * i.g.double()).sum(1) + i.gh.double() * h

    x, step = i.logits.double(), 1e-5
    for v in range(60):
        e = torch.zeros_like(x)
        e[:, v] = step
        diff = (loss(x + e) - loss(x - e)) / (2 * step)
        # the third derivative is below 10 here, so the difference is off by less than 10 step^2; the rest are 64-bit roundings
        assert float((grad[:, v] - diff).abs().max()) < 2e-8 + 64 * U * 10, v


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_farther_apart_than_32_bits(dtype):
    torch = torch_()
    stride = (1 << 30) + 7
    i = Inputs(4, 1500, dtype, "mixed", stride=stride, seed=3)
    out = i.forward()
    want = check_forward(i, out)
    check_backward(i, i.backward(out, in_place=True), want)
    del i
    torch.cuda.empty_cache()


@gpu
@pytest.mark.parametrize("masked", [False, True])
def test_the_longest_rows(masked):
    """A row of 2^30 bf16 logits, all alike but for a few: sums, ids and gradients at both ends and in the middle.  A thread of the 2,048
    adds up 2^14 sums of 32 terms: 2^14 + 33 roundings, and 4 |d| + 4 for the terms."""
    torch = torch_()
    V, low, places = 1 << 30, -8.0, [3, 17, (1 << 29) + 5, (1 << 30) - 2]
    values = [9.0, 10.0, 9.5, 8.5]
    x = torch.full((V,), low, dtype=torch.bfloat16, device=DEV)
    x[places] = torch.tensor(values, dtype=torch.bfloat16, device=DEV)
    mask = torch.full((V // 32,), -1, dtype=torch.int32, device=DEV) if masked else None
    if masked:
        mask[1 << 20: 1 << 24] = 0
    tokens = torch.tensor([places + [V - 1, 1 << 25]], dtype=torch.int32, device=DEV)
    lp, norm, H = torch.zeros((1, 6), device=DEV), torch.zeros((1, 2), device=DEV), torch.zeros(1, device=DEV)
    ids, status = torch.zeros((1, 6), dtype=torch.int32, device=DEV), torch.full((1,), 77, dtype=torch.int32, device=DEV)
    kw = dict(tokens_dev=tokens, n_tokens=6, mask_dev=mask)
    fmt.token_logprobs(x, fmt.BF16, 1, V, logprobs_dev=lp, norm_dev=norm, entropy_dev=H, n_top=6, top_ids_dev=ids, status_dev=status, **kw)
    others = V - 4 - (((1 << 24) - (1 << 20)) * 32 if masked else 0)
    d = np.array(values + [low]) - 10.0
    many = np.array([1, 1, 1, 1, others])
    S = (many * np.exp(d)).sum()
    ln = d - np.log(S)
    entropy = -(many * np.exp(ln) * ln).sum()
    off = U * ((1 << 14) + 33 + 4 * 18 + 4)
    assert status.item() == 0 and ids[0].tolist() == [17, (1 << 29) + 5, 3, V - 2, 0, 1]
    assert norm[0, 0].item() == 10.0 and abs(norm[0, 1].item() - np.log(S)) < off + 2 * U * np.log(S)
    gone = masked and (1 << 20) <= (1 << 25) // 32 < (1 << 24)
    want = np.array(list(ln) + [-np.inf if gone else ln[4]])
    got = lp[0].double().cpu().numpy()
    assert got[5] == want[5] if gone else True
    assert (np.abs(got[:5] - want[:5]) < off + 8 * U * np.abs(want[:5])).all()
    assert abs(H.item() - entropy) < (2 * off + 8 * U) * (2 + entropy)
    g, gh = torch.tensor([[0.5, -1.0, 0.25, 2.0, 1.5, 0.75]], device=DEV), torch.tensor([0.7], device=DEV)
    fmt.token_logprobs_backward(x, fmt.BF16, 1, V, norm, x, grad_logprobs_dev=g, entropy_dev=H, grad_entropy_dev=gh, **kw)  # in the logits' place
    gs = g[0].double().cpu().numpy()
    if gone:
        gs[5] = 0.0
    p = np.exp(ln)
    base = -p * gs.sum() - 0.7 * p * (ln + entropy)
    grad = x[places + [V - 1, 1 << 25, 0, (1 << 29) - 1]].double().cpu().numpy()
    more = base[4] if not masked else 0.0
    wants = np.array([base[0] + gs[0], base[1] + gs[1], base[2] + gs[2], base[3] + gs[3], base[4] + gs[4], 0.0 if gone else base[4] + gs[5], base[4], more])
    assert (np.abs(grad - wants) <= 2.0 ** -8 * np.abs(wants) + 2 * off * (1 + gs.sum()) * 4).all(), (grad, wants)
    assert int((x == x[0]).sum()) == others - (1 if gone else 2)  # all that are alike but tokens that were given
    if masked:
        assert int((x == 0).sum()) == V - 4 - others
    del x
    torch.cuda.empty_cache()


@gpu
def test_captured_replayed_and_on_other_streams():
    """Two graphs of the same call with other inputs, replayed at the same time on two streams, several times."""
    torch = torch_()
    ins = [Inputs(n, 40001, "bf16", "mixed", n_tokens=2, seed=n) for n in (3, 150)]
    outs = [i.forward() for i in ins]
    grads = [i.backward(o) for i, o in zip(ins, outs)]
    wants = [check_forward(i, o) for i, o in zip(ins, outs)]
    masks = [i.mask() for i in ins]
    for i, m in zip(ins, masks):
        i.mask = lambda m=m: m
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for i, o, gr, s in zip(ins, outs, grads, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            h = torch.cuda.current_stream().cuda_stream
            i.forward(into=o, stream=h)
            i.backward(o, grad=gr, stream=h)
        graphs.append(g)
    for _ in range(5):
        for o, gr in zip(outs, grads):
            for k in ("logprobs", "norm", "entropy", "tops"):
                o[k].fill_(77.0)
            o["ids"].fill_(77), o["status"].fill_(77), gr.fill_(77.0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for i, o, gr, w in zip(ins, outs, grads, wants):
            check_forward(i, o)
            check_backward(i, gr, w)


@gpu
def test_the_same_call_gives_the_same_bits():
    torch = torch_()
    i = Inputs(64, 50001, "bf16", "mixed", n_tokens=3, seed=1)
    first = i.forward(20)
    grad = i.backward(first).clone()
    for _ in range(3):
        again = i.forward(20)
        assert all(torch.equal(first[k], again[k]) for k in first)
        assert torch.equal(grad, i.backward(again))


def refused(f, *a, **kw):
    with pytest.raises(fmt.FmtError) as e:
        f(*a, **kw)
    assert e.value.code == fmt.ERR_INVALID_ARG
    return str(e.value)


def test_refusals():
    """Every one of these is turned down on the host, before anything reaches a GPU."""
    P = 1 << 20  # never read
    f = lambda **kw: fmt.token_logprobs(**dict(dict(logits_dev=P, dtype=fmt.BF16, rows=2, V=100, norm_dev=P), **kw))
    b = lambda **kw: fmt.token_logprobs_backward(**dict(dict(logits_dev=P, dtype=fmt.BF16, rows=2, V=100, norm_dev=P, grad_logits_dev=P + 4096), **kw))
    for call in (f, b):
        refused(call, logits_dev=None)
        refused(call, dtype=2)
        refused(call, V=0)
        refused(call, V=(1 << 30) + 1)
        refused(call, rows=(1 << 24) + 1)
        refused(call, row_stride=99)
        refused(call, mask_dev=P, stride_words=3)
        refused(call, n_tokens=33, tokens_dev=P)
        refused(call, n_tokens=1)
        refused(call, logits_dev=P + 1)
        refused(call, dtype=fmt.FP32, logits_dev=P + 2)
        refused(call, mask_dev=P + 2)
        refused(call, temperature_dev=P + 1)
        refused(call, n_tokens=1, tokens_dev=P + 3)
        refused(call, norm_dev=P + 2)
    refused(f, n_top=33, top_ids_dev=P)
    refused(f, status_dev=P + 2)
    refused(f, n_top=3, top_ids_dev=P + 1)
    refused(b, norm_dev=None)
    refused(b, grad_logits_dev=None)
    refused(b, grad_stride=99)
    refused(b, grad_entropy_dev=P)
    refused(b, grad_logits_dev=P, row_stride=100, grad_stride=101)
    refused(b, grad_logits_dev=P + 4097)


@gpu
def test_memory_that_the_device_cannot_reach_is_refused():
    torch = torch_()
    i = Inputs(2, 64, "fp32", "mixed", n_tokens=1)
    host = torch.zeros((2, 64))
    norm = torch.zeros((2, 2), device=DEV)
    refused(fmt.token_logprobs, host, fmt.FP32, 2, 64, norm_dev=norm)
    refused(fmt.token_logprobs, i.logits, fmt.FP32, 2, 64, norm_dev=host)
    refused(fmt.token_logprobs, i.logits, fmt.FP32, 2, 64, norm_dev=norm, mask_dev=torch.zeros((2, 2), dtype=torch.int32))
    refused(fmt.token_logprobs_backward, i.logits, fmt.FP32, 2, 64, norm, host)
    status = torch.full((2,), 77, dtype=torch.int32).pin_memory()  # page-locked memory is reached
    fmt.token_logprobs(i.logits, fmt.FP32, 2, 64, norm_dev=norm, status_dev=status)
    torch.cuda.synchronize()
    assert status.tolist() == [0, 0]
