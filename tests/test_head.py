"""The output head: 8-bit blocks with their scales (fmt_quantize_blocks) and the product under the mask (fmt_head_logits), against
the definition in 64 bits; what they refuse; and a decoding loop from hidden states to the next token.

Tolerances.  Scales and 8-bit values are compared bit for bit: their definition is in IEEE single precision.  A logit is a sum of
K products of e4m3 values, each exact in fp32, times two scales for each block of 128.  Sums of 128 products and of the blocks
take at most 128 + blocks additions, the scales three roundings each; every one of them is off by at most 2^-23 (a unit: the
order and the rounding of the additions inside a matrix instruction are not specified) of what has been summed up so far, so
  |logit - exact| <= (128 + blocks + 4) 2^-23 * sum over blocks of xs ws sum |x w|
and half a step of the output's type on top.
"""
import os
import subprocess
import sys

import numpy as np
import pytest

import oracle
import paper_2506_01151_b200 as fmt
import workloads
from helpers import OracleBatch
from test_logprobs import DEV, refused, torch_

gpu = pytest.mark.gpu


def up(a, b):
    return (a + b - 1) // b


def quantized(x, block_rows):
    """The definition, with torch on the device: bytes, scales (as fmt_quantize_blocks lays them out)."""
    torch = torch_()
    rows, cols = x.shape
    f = torch.zeros((up(rows, block_rows) * block_rows, up(cols, 128) * 128), device=x.device)
    f[:rows, :cols] = x.float()
    b = f.view(-1, block_rows, up(cols, 128), 128)
    s = b.abs().amax((1, 3))
    s = s / torch.full_like(s, 448.0)  # (by a number, torch multiplies with its reciprocal on the GPU)
    s = torch.where(s == 0, 1.0, s)
    s = torch.where(torch.isfinite(s), s, torch.nan)
    q = (b / s[:, None, :, None]).clamp(-448, 448).reshape(f.shape)[:rows, :cols].to(torch.float8_e4m3fn).view(torch.uint8)
    return q, (s.t() if block_rows == 1 else s).contiguous()


def normal_nan(q):
    return q.masked_fill((q & 0x7F) == 0x7F, 0x7F)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 128, 0), (3, 129, 7), (128, 256, 0), (130, 500, 12), (257, 4096, 0), (300, 77, 51), (1000, 2880, 16)])
def test_quantize(rows, cols, pad, block_rows, dtype):
    torch = torch_()
    g = torch.Generator(device=DEV)
    g.manual_seed(rows + cols)
    ty = torch.bfloat16 if dtype == "bf16" else torch.float32
    store = torch.full((rows * (cols + pad) + 1,), float("nan"), dtype=ty, device=DEV)
    off = pad % 2
    x = store[off:].as_strided((rows, cols), (cols + pad, 1))
    x.copy_((torch.randn((rows, cols), generator=g, device=DEV) * torch.exp(4 * torch.randn((rows, 1), generator=g, device=DEV))).to(ty))
    x[rows // 2] = 0.0
    x[rows - 1, cols // 2] = 1e4
    x[rows // 3, :] *= 1e-38
    x[rows // 3, 0] = 1e-41
    want, scales = quantized(x, block_rows)
    q = torch.full((rows, cols + pad), 0xAB, dtype=torch.uint8, device=DEV)
    ss = scales.shape[1] + pad
    s = torch.full((scales.shape[0], ss), 77.0, device=DEV)
    fmt.quantize_blocks(x, fmt.BF16 if dtype == "bf16" else fmt.FP32, rows, cols, block_rows, q, s, row_stride=cols + pad, q_stride=cols + pad, scale_stride=ss)
    assert torch.equal(s[:, : scales.shape[1]], scales)
    assert torch.equal(q[:, :cols], want)
    assert bool((q[:, cols:] == 0xAB).all()) and bool((s[:, scales.shape[1]:] == 77).all())


@gpu
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_what_is_not_finite(block_rows):
    torch = torch_()
    x = torch.randn((256, 300), device=DEV)
    x[3, 5], x[140, 290], x[200, 130] = float("nan"), float("inf"), float("-inf")
    want, scales = quantized(x, block_rows)
    q, s = torch.zeros((256, 300), dtype=torch.uint8, device=DEV), torch.zeros_like(scales)
    fmt.quantize_blocks(x, fmt.FP32, 256, 300, block_rows, q, s)
    assert torch.equal(torch.nan_to_num(s, nan=-1.0), torch.nan_to_num(scales, nan=-1.0))
    assert torch.equal(normal_nan(q), normal_nan(want))


class Head:
    def __init__(self, n, V, K, mask="mixed", dtype="bf16", seed=0, pad=0, offset=0, row_pad=0, mask_pad=0, hidden=None):
        torch = torch_()
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.n, self.V, self.K = n, V, K
        self.hs = self.ws = up(K, 16) * 16 + 16 * pad
        kb = up(K, 128)
        hidden = torch.randn((n, K), generator=g, device=DEV) * torch.exp(torch.randn((1, K), generator=g, device=DEV)) if hidden is None else hidden
        weights = torch.randn((V, K), generator=g, device=DEV) * torch.exp(torch.randn((V, 1), generator=g, device=DEV)) / K ** 0.5
        q, s = quantized(hidden, 1)
        # what lies between the rows, behind the last ones and between the scales is NaN
        self.q = torch.full((n, self.hs), 0x7F, dtype=torch.uint8, device=DEV)
        self.q[:, :K] = q
        self.hss = n + pad
        self.s = torch.full((kb, self.hss), float("nan"), device=DEV)
        self.s[:, :n] = s
        q, s = quantized(weights, 128)
        self.w = torch.full((V, self.ws), 0x7F, dtype=torch.uint8, device=DEV)
        self.w[:, :K] = q
        self.wss = kb + pad
        self.wscale = torch.full((up(V, 128), self.wss), float("nan"), device=DEV)
        self.wscale[:, :kb] = s
        self.words, self.dtype = up(V, 32), fmt.BF16 if dtype == "bf16" else fmt.FP32
        self.mask_stride = self.words + mask_pad
        share = {"none": 1.0, "all": 1.0, "mixed": 0.5, "few": min(1.0, 2.0 / V), "empty": 0.0}[mask]
        self.allow = torch.rand((n, V), generator=g, device=DEV) < share
        self.mask = None
        if mask != "none":
            bits = torch.ones((n, self.mask_stride * 32), dtype=torch.int64, device=DEV)
            bits[:, :V] = self.allow.long()
            w = (bits.view(n, -1, 32) << torch.arange(32, device=DEV)).sum(-1)
            self.mask = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)
        ty = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.row_stride = V + row_pad
        self.store = torch.full((offset + n * self.row_stride + 64,), 77.0, dtype=ty, device=DEV)
        self.offset = offset
        self.logits = self.store[offset:].as_strided((n, V), (self.row_stride, 1))

    def call(self, stream=None):
        fmt.head_logits(self.q, self.s, self.w, self.wscale, self.logits, self.dtype, self.n, self.V, self.K, mask_dev=self.mask,
                        hidden_stride=self.hs, hidden_scale_stride=self.hss, weight_stride=self.ws, weight_scale_stride=self.wss,
                        stride_words=self.mask_stride, row_stride=self.row_stride, stream=stream)
        return self.logits

    def check(self):
        torch = torch_()
        K, n, V = self.K, self.n, self.V
        x = self.q[:, :K].view(torch.float8_e4m3fn).double() * self.s[:, :n].t().double().repeat_interleave(128, 1)[:, :K]
        half = torch.finfo(self.logits.dtype).eps / 2
        for v in range(0, V, 16384):
            rows = min(16384, V - v)
            w = self.w[v:v + rows, :K].view(torch.float8_e4m3fn).double()
            w = w * self.wscale[v // 128: up(v + rows, 128), : up(K, 128)].double().repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :K]
            want, most = x @ w.t(), x.abs() @ w.abs().t()
            got, ok = self.logits[:, v:v + rows].double(), self.allow[:, v:v + rows]
            assert bool((got[~ok] == -torch.inf).all()), "not allowed"
            want = torch.where(ok, want, 0.0)
            nan = torch.isnan(want)
            assert torch.equal(torch.isnan(got) & ok, nan)
            err = torch.where(ok & ~nan, (got - want).abs(), 0.0)
            limit = (128 + up(K, 128) + 4) * 2.0 ** -23 * most + half * want.abs() + 1e-40
            limit = torch.where(nan | ~ok, 1.0, limit)
            assert bool((err <= limit).all()), (float((err / limit).max()), torch.nonzero(err > limit)[:4].tolist())
        edge = torch.ones_like(self.store, dtype=torch.bool)
        edge[self.offset:].as_strided((n, V), (self.row_stride, 1))[:] = False
        assert bool((self.store[edge] == 77).all()), "between or behind the rows"


@gpu
@pytest.mark.parametrize("mask", ["none", "mixed", "few"])
@pytest.mark.parametrize("n", [1, 2, 8, 16, 17, 33, 64, 65, 100, 128, 129, 256, 257, 600])
@pytest.mark.parametrize("V,K", [(512, 256), (5000, 640), (33, 130)])
def test_batches(V, K, n, mask):
    h = Head(n, V, K, mask, dtype="fp32" if n % 2 else "bf16", seed=n)
    h.call()
    h.check()


@gpu
@pytest.mark.parametrize("V", [1, 31, 32, 33, 127, 128, 129, 1000, 4737, 20000])
@pytest.mark.parametrize("K", [1, 16, 31, 127, 128, 129, 257, 1000, 4100])
def test_odd_sizes(V, K):
    h = Head(5, V, K, "mixed", dtype="bf16" if K % 2 else "fp32", seed=V + K, pad=K % 3, offset=V % 4, row_pad=V % 5, mask_pad=K % 2)
    h.call()
    h.check()


@gpu
@pytest.mark.parametrize("n", [16, 40, 70, 200])
@pytest.mark.parametrize("V", [1, 33, 100, 200, 4737])
@pytest.mark.parametrize("K", [1, 129, 700])
def test_odd_sizes_of_every_form(K, V, n):
    h = Head(n, V, K, "mixed", dtype="bf16" if K % 2 else "fp32", seed=V + K, pad=K % 3, offset=n % 3, row_pad=V % 5, mask_pad=K % 2)
    h.call()
    h.check()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("offset,row_pad", [(0, 0), (2, 0), (1, 1), (16, 16)])
@pytest.mark.parametrize("n", [20, 100, 300])
def test_rows_begin_at_any_address(n, offset, row_pad, dtype):
    h = Head(n, 3200, 256, "mixed", dtype, seed=n, offset=offset, row_pad=row_pad)
    h.call()
    h.check()


@gpu
@pytest.mark.parametrize("n,V,mask", [(3, 1 << 20, "few"), (3, 1 << 20, "none"), (130, 1 << 20, "few"), (130, 1000001, "mixed"), (700, 1 << 20, "few")])
def test_the_largest_vocabularies(n, V, mask):
    h = Head(n, V, 16, mask, "bf16", seed=n)
    h.call()
    h.check()
    del h
    torch_().cuda.empty_cache()


@gpu
@pytest.mark.parametrize("n", [8, 300])
def test_sparse_masks_of_large_vocabularies(n):
    """From one word in a hundred to every other word in use: the lists of slabs, whole and piecewise."""
    torch = torch_()
    for share in (0.01, 0.1, 0.5, 0.97):
        h = Head(n, 40000, 300, "all", "bf16", seed=int(share * 100))
        g = torch.Generator(device=DEV)
        g.manual_seed(3)
        words = torch.rand(h.words, generator=g, device=DEV) < share
        h.allow = words.repeat_interleave(32)[None, :40000].expand(n, -1).clone()
        h.mask = torch.where(words, -1, 0).to(torch.int32)[None].repeat(n, 1).contiguous()
        h.call()
        h.check()


@gpu
@pytest.mark.parametrize("mask", ["all", "few", "empty"])
@pytest.mark.parametrize("n,V,K,dtype", [(1, 32000, 4096, "bf16"), (8, 128256, 1024, "bf16"), (37, 50001, 2880, "fp32"), (300, 20011, 512, "bf16"), (256, 128256, 256, "bf16"), (1500, 6000, 1030, "bf16")])
def test_large(n, V, K, dtype, mask):
    h = Head(n, V, K, mask, dtype, seed=n + V)
    h.call()
    h.check()


@gpu
def test_long_sums():
    """K of many blocks, values of one sign, so that the sum grows all the way."""
    torch = torch_()
    h = Head(3, 200, 40000, "none", "fp32", hidden=torch.rand((3, 40000), device=DEV))
    h.w &= 0x7F
    h.call()
    h.check()


@gpu
@pytest.mark.parametrize("n", [3, 70, 300])
def test_nan_stays_where_it_belongs(n):
    """A NaN among a row's hidden states or a token's weights makes that row's or that token's logits NaN, and no other."""
    torch = torch_()
    h = Head(n, 1000, 300, "mixed", "fp32", seed=n)
    h.q[2, 299] = 0x7F
    h.s[1, 1] = float("nan")
    h.w[40, 7] = 0x7F
    h.wscale[3, 2] = float("nan")
    h.call()
    h.check()


@gpu
def test_weights_that_no_row_may_use_do_not_matter():
    torch = torch_()
    h = Head(9, 4000, 512, "mixed", "bf16", seed=4)
    dead = torch.zeros(4000, dtype=torch.bool, device=DEV)
    dead[64:96] = dead[1000:1700] = dead[3990:] = True
    h.allow &= ~dead
    bits = torch.zeros((9, h.words * 32), dtype=torch.int64, device=DEV)
    bits[:, :4000] = h.allow.long()
    w = (bits.view(9, -1, 32) << torch.arange(32, device=DEV)).sum(-1)
    h.mask = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)
    h.call()
    first = h.logits.clone()
    h.w[dead] = 0x7F
    h.call()
    h.check()
    assert torch.equal(first, h.logits)


@gpu
def test_logits_farther_apart_than_32_bits():
    torch = torch_()
    h = Head(4, 700, 260, "mixed", "bf16", seed=2, row_pad=(1 << 30) + 3)
    h.call()
    h.check()
    del h
    torch.cuda.empty_cache()


@gpu
def test_captured_replayed_and_on_other_streams():
    torch = torch_()
    hs = [Head(n, 30000, 1000, "mixed", "bf16", seed=n) for n in (4, 200)]
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for h, s in zip(hs, streams):
        h.call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            h.call(torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    for _ in range(5):
        for h in hs:
            h.logits.fill_(5.0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for h in hs:
            h.check()


@gpu
def test_the_same_call_gives_the_same_bits():
    torch = torch_()
    for n in (1, 64, 256):
        h = Head(n, 50001, 1000, "mixed", "fp32", seed=n)
        first = h.call().clone()
        for _ in range(3):
            assert torch.equal(first, h.call())


@gpu
@pytest.mark.parametrize("mask", ["none", "mixed", "few"])
@pytest.mark.parametrize("n", [8, 20, 40, 100, 300])
def test_waits_that_run_out(n, mask):
    """With a limit of few polls, waits run out although nothing is wrong, at other places each time (copies on another stream slow the
    loads down): what comes back is right, or NaN where a token is allowed, and the next call is exact."""
    torch = torch_()
    h = Head(n, 30011, 1000, mask, "bf16" if n % 40 else "fp32", seed=n, row_pad=n % 3)
    right = h.call().clone()
    h.check()
    allow = h.allow if h.mask is not None else torch.ones_like(h.allow)
    block, other = torch.zeros(1 << 28, dtype=torch.uint8, device=DEV), torch.cuda.Stream()
    torch.cuda.synchronize()
    try:
        fmt.head_set_wait_limit(0)
        h.store.fill_(77.0)
        got = h.call()
        assert bool((torch.isnan(got) == allow).all()) and bool((got[~allow] == -torch.inf).all())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            h.call(torch.cuda.current_stream().cuda_stream)
        for polls in (1, 2, 4, 16) * 3:
            fmt.head_set_wait_limit(polls)
            h.store.fill_(77.0)
            with torch.cuda.stream(other):
                for _ in range(4):
                    block.copy_(block.roll(1))
            got = h.call()
            assert bool(((got == right) | (torch.isnan(got) & allow)).all())
            torch.cuda.synchronize()
    finally:
        fmt.head_set_wait_limit()
    h.store.fill_(77.0)
    assert torch.equal(h.call(), right)
    h.check()
    graph.replay()  # a captured call keeps the limit that it was captured with
    assert bool((torch.isnan(h.logits) == allow).all())
    assert torch.equal(h.call(), right)
    fmt.head_set_wait_limit(1 << 31)  # no more than there are otherwise
    assert torch.equal(h.call(), right)
    fmt.head_set_wait_limit()


OTHER_CONTEXTS = """
import ctypes as C, sys
import numpy as np
import paper_2506_01151_b200 as fmt

D = C.CDLL("libcuda.so.1")
def cu(name, *a):
    r = getattr(D, name)(*a)
    assert r == 0, (name, r)
vp = C.c_void_p
D.cuMemAlloc_v2.argtypes = [C.POINTER(vp), C.c_size_t]
D.cuMemcpyHtoD_v2.argtypes = [vp, vp, C.c_size_t]
D.cuMemcpyDtoH_v2.argtypes = [vp, vp, C.c_size_t]
dev, ctx = C.c_int(), vp()
cu("cuInit", 0)
cu("cuDeviceGet", C.byref(dev), 0)

def to_device(a):
    p = vp()
    cu("cuMemAlloc_v2", C.byref(p), a.nbytes)
    cu("cuMemcpyHtoD_v2", p, a.ctypes.data, a.nbytes)
    return p.value

def logits(n, V=300, K=256):  # of ones: e4m3 1.0 is 0x38
    y = to_device(np.zeros((n, V), np.float32))
    fmt.head_logits(to_device(np.full((n, K), 0x38, np.uint8)), to_device(np.ones((2, n), np.float32)), to_device(np.full((V, K), 0x38, np.uint8)),
                    to_device(np.ones((3, 2), np.float32)), y, fmt.FP32, n, V, K)
    got = np.zeros((n, V), np.float32)
    cu("cuCtxSynchronize")
    cu("cuMemcpyDtoH_v2", got.ctypes.data, y, got.nbytes)
    assert (got == K).all(), got

def all_forms():
    for n in (1, 20, 40, 70, 130):
        logits(n)

if sys.argv[1] == "second":
    for _ in range(2):
        cu("cuCtxCreate_v2", C.byref(ctx), 0, dev)
        all_forms()
else:
    for _ in range(2):
        cu("cuDevicePrimaryCtxRetain", C.byref(ctx), dev)
        cu("cuCtxSetCurrent", ctx)
        all_forms()
        cu("cuDevicePrimaryCtxReset_v2", dev)
print("both answered")
"""


@gpu
@pytest.mark.parametrize("how", ["second", "reset"])
def test_another_context_of_the_same_device(how):
    """What a kernel is allowed to use belongs to a context: a process that makes a second one, or resets its device, calls on."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", OTHER_CONTEXTS, how], cwd=root, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "both answered" in r.stdout, r.stdout + r.stderr


def test_refusals():
    """Every one of these is turned down on the host, before anything reaches a GPU."""
    P = 1 << 20  # never read
    q = lambda **kw: fmt.quantize_blocks(**dict(dict(x_dev=P, dtype=fmt.BF16, rows=2, cols=100, block_rows=1, q_dev=P, scales_dev=P), **kw))
    refused(q, x_dev=None)
    refused(q, q_dev=None)
    refused(q, scales_dev=None)
    refused(q, dtype=2)
    refused(q, block_rows=2)
    refused(q, cols=0)
    refused(q, cols=(1 << 20) + 1)
    refused(q, rows=(1 << 24) + 1)
    refused(q, row_stride=99)
    refused(q, q_stride=99)
    refused(q, scale_stride=1)
    refused(q, block_rows=128, cols=129, scale_stride=1)
    refused(q, x_dev=P + 1)
    refused(q, dtype=fmt.FP32, x_dev=P + 2)
    refused(q, scales_dev=P + 2)
    h = lambda **kw: fmt.head_logits(**dict(dict(hidden_dev=P, hidden_scales_dev=P, weight_dev=P, weight_scales_dev=P, logits_dev=P, dtype=fmt.BF16,
                                                 rows=2, V=100, K=256), **kw))
    for name in ("hidden_dev", "hidden_scales_dev", "weight_dev", "weight_scales_dev", "logits_dev"):
        refused(h, **{name: None})
    refused(h, dtype=2)
    refused(h, V=0)
    refused(h, V=(1 << 20) + 1)
    refused(h, K=0)
    refused(h, K=(1 << 20) + 16)
    refused(h, rows=(1 << 24) + 1)
    refused(h, hidden_stride=240)
    refused(h, hidden_stride=264)
    refused(h, weight_stride=240)
    refused(h, weight_stride=264)
    refused(h, K=100, hidden_stride=112)          # weight_stride = K is no multiple of 16
    refused(h, hidden_scale_stride=1)
    refused(h, weight_scale_stride=1)
    refused(h, row_stride=99)
    refused(h, mask_dev=P, stride_words=3)
    refused(h, hidden_dev=P + 8)
    refused(h, weight_dev=P + 8)
    refused(h, hidden_scales_dev=P + 2)
    refused(h, weight_scales_dev=P + 2)
    refused(h, mask_dev=P + 2)
    refused(h, logits_dev=P + 1)
    refused(h, dtype=fmt.FP32, logits_dev=P + 2)


@gpu
def test_memory_that_the_device_cannot_reach_is_refused():
    torch = torch_()
    h = Head(2, 64, 128)
    for name in ("q", "s", "w", "wscale", "mask", "logits"):
        kept = getattr(h, name)
        setattr(h, name, kept.cpu())
        refused(h.call)
        setattr(h, name, kept)
    h.ws = 1 << 40  # more than the copy engine can step
    refused(h.call)
    h.ws = 128
    x, q, s = torch.zeros((2, 64), device=DEV), torch.zeros((2, 64), dtype=torch.uint8, device=DEV), torch.zeros((1, 2), device=DEV)
    refused(fmt.quantize_blocks, x.cpu(), fmt.FP32, 2, 64, 1, q, s)
    refused(fmt.quantize_blocks, x, fmt.FP32, 2, 64, 1, q.cpu(), s)
    refused(fmt.quantize_blocks, x, fmt.FP32, 2, 64, 1, q, s.cpu())
    fmt.quantize_blocks(x, fmt.FP32, 0, 64, 1, q, s)
    fmt.head_logits(h.q, h.s, h.w, h.wscale, h.logits, h.dtype, 0, 64, 128, hidden_scale_stride=2)
    assert bool((h.store == 77).all())


@gpu
def test_steps_back_to_back_on_two_streams():
    """Hidden states -> 8-bit blocks -> masked logits -> log probabilities -> gradient in the logits' place, many steps without a pause on two
    streams at a time (launches overlap: a kernel begins while the one before is still running), against one call after the other."""
    torch = torch_()
    steps, K = 12, 700
    cases = []
    for n, V, mask in ((9, 20011, "few"), (200, 6000, "mixed")):
        h = Head(n, V, K, mask, "bf16", seed=n)
        g = torch.Generator(device=DEV)
        g.manual_seed(n)
        hidden = torch.randn((steps, n, K), generator=g, device=DEV).to(torch.bfloat16)
        cases.append((h, hidden, torch.randint(0, V, (n, 2), generator=g, device=DEV, dtype=torch.int32), torch.randn((n, 2), generator=g, device=DEV),
                      torch.randn(n, generator=g, device=DEV)))

    def outputs():
        f = dict(dtype=torch.float32, device=DEV)
        return [dict(q=torch.zeros((n, h.hs), dtype=torch.uint8, device=DEV), s=torch.zeros((up(K, 128), n), **f),
                     y=torch.zeros((steps, n, h.V), dtype=torch.bfloat16, device=DEV), lp=torch.zeros((steps, n, 2), **f), norm=torch.zeros((steps, n, 2), **f),
                     H=torch.zeros((steps, n), **f), ids=torch.zeros((steps, n, 3), dtype=torch.int32, device=DEV)) for h, *_ in cases for n in [h.n]]

    def step(i, case, o, stream, pause):
        h, hidden, tokens, g, gh = case
        fmt.quantize_blocks(hidden[i], fmt.BF16, h.n, K, 1, o["q"], o["s"], q_stride=h.hs, stream=stream)
        pause()
        fmt.head_logits(o["q"], o["s"], h.w, h.wscale, o["y"][i], fmt.BF16, h.n, h.V, K, mask_dev=h.mask, hidden_stride=h.hs, weight_stride=h.ws,
                        weight_scale_stride=h.wss, stride_words=h.mask_stride, stream=stream)
        pause()
        fmt.token_logprobs(o["y"][i], fmt.BF16, h.n, h.V, tokens_dev=tokens, n_tokens=2, logprobs_dev=o["lp"][i], norm_dev=o["norm"][i], entropy_dev=o["H"][i],
                           n_top=3, top_ids_dev=o["ids"][i], mask_dev=h.mask, stride_words=h.mask_stride, stream=stream)
        pause()
        fmt.token_logprobs_backward(o["y"][i], fmt.BF16, h.n, h.V, o["norm"][i], o["y"][i], tokens_dev=tokens, n_tokens=2, grad_logprobs_dev=g,
                                    entropy_dev=o["H"][i], grad_entropy_dev=gh, mask_dev=h.mask, stride_words=h.mask_stride, stream=stream)
        pause()

    want = outputs()
    for case, o in zip(cases, want):
        for i in range(steps):
            step(i, case, o, 0, torch.cuda.synchronize)
    assert all(len(torch.unique(o["ids"][:, 0, 0])) > 1 for o in want)  # the steps are not alike
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        got = outputs()
        torch.cuda.synchronize()
        for i in range(steps):
            for case, o, s in zip(cases, got, streams):
                step(i, case, o, s.cuda_stream, lambda: None)
        torch.cuda.synchronize()
        for o, w in zip(got, want):
            assert all(torch.equal(o[k].view(torch.uint8), w[k].view(torch.uint8)) for k in w)


@gpu
def test_a_decoding_loop_from_hidden_states_to_the_next_token():
    """Masks from the grammar, logits from the 8-bit head under them, the likeliest token back into the state: every token
    taken is one that the oracle allows, and the distribution is that of the masked logits."""
    torch = torch_()
    w = workloads.build(2, V=6000, batch=6, steps=4)
    g = fmt.Grammar(w.ebnf, w.start, w.vocab, w.eos)
    st = fmt.State(g, w.batch)
    ob = OracleBatch(w)
    K, n, V = 384, w.batch, w.V
    gen = torch.Generator(device=DEV)
    gen.manual_seed(11)
    weights = torch.randn((V, K), generator=gen, device=DEV).to(torch.bfloat16)
    wq, wscale = torch.zeros((V, K), dtype=torch.uint8, device=DEV), torch.zeros((up(V, 128), up(K, 128)), device=DEV)
    fmt.quantize_blocks(weights, fmt.BF16, V, K, 128, wq, wscale)
    hq, hscale = torch.zeros((n, K), dtype=torch.uint8, device=DEV), torch.zeros((up(K, 128), n), device=DEV)
    mask = torch.zeros((n, g.mask_words), dtype=torch.int32, device=DEV)
    logits = torch.zeros((n, V), dtype=torch.bfloat16, device=DEV)
    ids, lp = torch.zeros((n, 1), dtype=torch.int32, device=DEV), torch.zeros((n, 1), device=DEV)
    status = torch.zeros(n, dtype=torch.int32, device=DEV)
    for step in range(12):
        hidden = torch.randn((n, K), generator=gen, device=DEV).to(torch.bfloat16)
        st.fill_mask(mask)
        fmt.quantize_blocks(hidden, fmt.BF16, n, K, 1, hq, hscale)
        fmt.head_logits(hq, hscale, wq, wscale, logits, fmt.BF16, n, V, K, mask_dev=mask)
        fmt.token_logprobs(logits, fmt.BF16, n, V, n_top=1, top_ids_dev=ids, top_logprobs_dev=lp)  # masked already
        with_mask, lp2 = torch.zeros_like(ids), torch.zeros_like(lp)
        fmt.token_logprobs(logits, fmt.BF16, n, V, n_top=1, top_ids_dev=with_mask, top_logprobs_dev=lp2, mask_dev=mask)
        want = np.stack([oracle.bits(ob.mask(b), V) for b in range(n)]).astype(bool)
        got = logits.float().cpu()
        assert np.array_equal((got != -torch.inf).numpy(), want)
        best = [int(np.flatnonzero(got[b].numpy() == got[b].max().item())[0]) if want[b].any() else -1 for b in range(n)]
        assert ids[:, 0].tolist() == best and torch.equal(ids, with_mask) and torch.equal(lp, lp2)
        exact = torch.log_softmax(got.double(), 1).max(1).values
        assert float((lp[:, 0].cpu().double() - exact).abs().max()) < 3.2e-5  # (6000 / 128 + 64 + 4 * 104) 2^-24
        st.advance(ids, status)
        rejected = [ob.advance(b, best[b]) for b in range(n)]
        assert status.tolist() == rejected
        assert all(r in (fmt.FMT_OK, fmt.ERR_FINISHED) for r in rejected)
