"""GPU tests of the MoE layer's operators where they are easiest to get wrong:
lost blocks beside rows that do not exist, strides, slots of no expert, every
store of every kernel, calls that overlap or are captured.

Bounds as in test_gpu_moe: a sum of n fp32 terms is within n 2^-23 of the sum of
their magnitudes, a bf16 result is rounded once (2^-8 of it at most).
"""
import numpy as np
import pytest

from conftest import gpu_available
from oracle import mx4 as omx4
from oracle import route as oroute

pytestmark = pytest.mark.gpu

if not gpu_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

import torch  # noqa: E402

import paper_2606_00079_amd as bm  # noqa: E402
from paper_2606_00079_amd import pipeline  # noqa: E402

DEV = "cuda:0"
U = 2.0 ** -23
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def within(got, want, bound, what):
    """NaN exactly where `want` is, and no farther from it than `bound`."""
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan()), what
    off = ((got - want).abs() - bound)[~want.isnan()]
    assert not (off > 0).any(), (what, float(off.max()), int((off > 0).sum()))


def weights(E, N, K, g, lost=0):
    """Weights in MX4, any codes, scales over a few powers of two; `lost` blocks of
    every expert stand for NaN."""
    codes = torch.randint(0, 256, (E, N, K // 2), dtype=torch.uint8, device=DEV)
    scales = g.integers(118, 124, (E, N, K // 32), dtype=np.uint8)
    for e in range(E):
        scales[e, g.integers(0, N, lost), g.integers(0, K // 32, lost)] = 255
    return codes, torch.from_numpy(scales).to(DEV)


def values(codes, scales):
    v = torch.tensor(omx4.GRID, dtype=torch.float64, device=DEV)
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    s = torch.where(scales == 255, torch.nan, 2.0 ** (scales.double() - 127))
    return v[c & 7] * (1 - 2 * (c >> 3)) * s.repeat_interleave(32, -1)


def offsets_of(E, S, tail, g, head=0):
    load = np.exp(0.7 * g.standard_normal(E)) * (g.random(E) > 0.1)
    load[0] += 1e-3
    n = g.multinomial(S - tail - head, load / load.sum())
    return (head + np.r_[0, np.cumsum(n)]).astype(np.int32)


def exact(codes, scales, X, off, rows=None, glu=False, grad=False):
    """(y, bound of an fp32 result) in 64 bits, a loop over the experts; a slot whose
    row does not exist, or that has no expert, is 0."""
    S = len(X) if rows is None else len(rows)
    r = torch.arange(S, device=DEV) if rows is None else rows.long()
    there = (r >= 0) & (r < len(X))
    x = X.double()[torch.where(there, r, 0)]
    width = codes.shape[2] * 2 if grad else codes.shape[1]
    y = torch.zeros((S, width), dtype=torch.float64, device=DEV)
    size = torch.zeros_like(y)
    for e in range(len(off) - 1):
        w = values(codes[e], scales[e])
        w = w if grad else w.t().contiguous()
        at = slice(int(off[e]), int(off[e + 1]))
        y[at], size[at] = x[at] @ w, x[at].abs() @ w.abs()
    size = size * ((x.shape[1] + 16) * U)
    if glu:
        N = y.shape[1] // 2
        g, u, eg, eu = y[:, :N], y[:, N:], size[:, :N], size[:, N:]
        s = g / (1 + torch.exp(-g))
        y = s * u
        size = 1.1 * eg * (u.abs() + eu) + s.abs() * eu + y.abs() * 2.0 ** -20
    y[~there], size[~there] = 0, 0
    return y, size + 1e-38


def product(form, codes, scales, X, **kw):
    """The result, and the tokens as the product saw them."""
    if form == "mx4":
        q = bm.mx4_quantize(X)
        return bm.mx4_product_q(codes, scales, *q, **kw), bm.mx4_dequantize(*q)
    return bm.mx4_product(codes, scales, X, **kw), X


def taken(kernel, call):
    """What `call` returns; it must have gone to `kernel`, in one launch."""
    bm.timing(True)
    try:
        out = call()
        assert bm.kernel_time(kernel)[1] == 1, kernel
    finally:
        bm.timing(False)
    return out


# form, kernel, E, N (2 N with glu), K, S
FORWARD = [
    ("bf16", "mx4_rows", 6, 250, 1056, 9), ("mx4", "mx4_rows", 6, 250, 1056, 9),
    ("bf16", "mx4_few", 90, 1550, 1312, 300), ("mx4", "mx4_few", 90, 1550, 1312, 300),
    ("bf16", "mx4_few", 40, 1550, 2080, 800), ("mx4", "mx4_few", 40, 1550, 2080, 800),
    ("bf16", "mx4_tile", 5, 2048, 288, 9000), ("bf16", "mx4_tile", 4, 2048, 512, 9000),
    ("mx4", "mx4_tile", 5, 2048, 288, 9000), ("mx4", "mx4_tile", 4, 2048, 1024, 9000),
]


@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("case", FORWARD)
def test_rows_that_do_not_exist_beside_lost_blocks(case, glu):
    """0 for such a slot, whatever kernel takes the call: not 0 times NaN."""
    form, kernel, E, N, K, S = case
    g = np.random.default_rng([E, N, K, S, glu])
    codes, scales = weights(E, N, K, g, lost=3)
    off = offsets_of(E, S, S // 50, g)
    T = S // 2 + 1
    X = torch.randn(T, K, device=DEV).to(torch.bfloat16)
    rows = g.integers(0, T, S).astype(np.int32)
    rows[::3], rows[1::5], rows[2::7] = -1, T, T + 1000
    rows = torch.from_numpy(rows).to(DEV)
    got, x = taken(kernel, lambda: product(form, codes, scales, X, offsets=torch.from_numpy(off).to(DEV), rows=rows,
                                           glu=glu, dtype=torch.float32))
    want, bound = exact(codes, scales, x, off, rows, glu)
    assert want.isnan().any()
    within(got, want, bound, case)


# form, kernel, E, N, K, S
BACKWARD = [
    ("grad", "mx4_grad_few", 6, 256, 1056, 9), ("grad", "mx4_grad_few", 90, 1552, 480, 1300),
    ("grad", "mx4_grad_tile", 5, 296, 2112, 9000), ("grad", "mx4_grad_tile", 2, 264, 4096, 9000),
]


@pytest.mark.parametrize("case", FORWARD + BACKWARD)
def test_slots_before_the_first_expert_and_after_the_last(case):
    """The slots of some of the experts only: the others' are 0, not left as they were."""
    form, kernel, E, N, K, S = case
    g = np.random.default_rng([E, N, K, S, 5])
    codes, scales = weights(E, N, K, g, lost=2)
    off = offsets_of(E, S, S // 9 + 1, g, head=S // 7 + 2)
    kw = {"offsets": torch.from_numpy(off).to(DEV), "dtype": torch.float32}
    X = torch.randn(S, N if form == "grad" else K, device=DEV).to(torch.bfloat16)
    if form == "grad":
        kw["out"] = torch.full((S, K), torch.nan, device=DEV)
        got = taken(kernel, lambda: bm.mx4_product_grad(codes, scales, X, **kw))
    else:
        kw["out"] = torch.full((S, N), torch.nan, device=DEV)
        got, X = taken(kernel, lambda: product(form, codes, scales, X, **kw))
    want, bound = exact(codes, scales, X, off, grad=form == "grad")
    within(got, want, bound, case)
    assert (got[:off[0]] == 0).all() and (got[off[-1]:] == 0).all()


@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("E,N,K,S", [(6, 250, 1056, 9), (90, 1550, 1312, 300), (4, 2048, 1024, 9000)])
def test_slots_of_no_rows_at_all(E, N, K, S, glu):
    """No token of these experts is here: zeros, in either form."""
    g = np.random.default_rng([E, N, K, S])
    codes, scales = weights(E, N, K, g, lost=2)
    kw = {"offsets": torch.from_numpy(offsets_of(E, S, 3, g)).to(DEV), "glu": glu,
          "rows": torch.full((S,), -1, dtype=torch.int32, device=DEV)}
    none = torch.zeros(0, K, dtype=torch.bfloat16, device=DEV)
    for form in ("bf16", "mx4"):
        out = torch.full((S, N // 2 if glu else N), torch.nan, device=DEV)
        got, _ = product(form, codes, scales, none, dtype=torch.float32, out=out, **kw)
        assert (got == 0).all(), form


def test_more_tiles_than_a_launch_takes():
    """The small tiles that cost least here would be more than 2^23 workgroups: the
    resident large ones take the call instead."""
    g = np.random.default_rng(17)
    S, T, first = (1 << 27) + 77, 64, (1 << 26) + 3
    codes, scales = weights(2, 1, 32, g)
    X = torch.randn(T, 32, device=DEV).to(torch.bfloat16)
    rows = torch.randint(0, T, (S,), dtype=torch.int32, device=DEV)
    off = torch.tensor([0, first, S], dtype=torch.int32, device=DEV)
    got = taken("mx4_tile", lambda: bm.mx4_product(codes, scales, X, offsets=off, rows=rows))
    w = values(codes, scales)[:, 0]
    table, size = X.double() @ w.t().contiguous(), X.double().abs() @ w.t().contiguous().abs()
    for e, at in ((0, slice(0, first)), (1, slice(first, S))):
        r = rows[at].long()
        want = table[:, e][r]
        within(got[at, 0], want, size[:, e][r] * 48 * U + 2.0 ** -8 * want.abs(), ("forward", e))
    del got, rows, r, want
    S, first = (1 << 28) + 40, (1 << 27) + 9
    codes, scales = weights(2, 8, 32, g)
    dY = torch.randn(1 << 20, 8, device=DEV).to(torch.bfloat16).repeat(257, 1)[:S]
    off = torch.tensor([0, first, S], dtype=torch.int32, device=DEV)
    got = taken("mx4_grad_tile", lambda: bm.mx4_product_grad(codes, scales, dY, offsets=off))
    w = values(codes, scales)
    cuts = sorted({0, first, S, *range(0, S, 1 << 24)})
    for lo, hi in zip(cuts, cuts[1:]):
        e, d = int(lo >= first), dY[lo:hi].double()
        want = d @ w[e]
        within(got[lo:hi], want, d.abs() @ w[e].abs() * 24 * U + 2.0 ** -8 * want.abs(), ("gradient", lo))


# Every way that a kernel stores and takes its slots: N a multiple of 256 (whole tiles, 16-byte stores) or not, K a
# multiple of 512 (scales 16 bytes a row) or not.  form, kernel, E, N (2 N with glu), K, S
STORED = [
    ("bf16", "mx4_rows", 6, 256, 1056, 9), ("mx4", "mx4_rows", 6, 256, 1056, 9),
    ("bf16", "mx4_few", 90, 1536, 1312, 300), ("mx4", "mx4_few", 90, 1536, 1312, 300),
    ("bf16", "mx4_few", 40, 1536, 2080, 800), ("mx4", "mx4_few", 200, 2048, 96, 3500),
    ("bf16", "mx4_tile", 5, 2048, 288, 9000), ("bf16", "mx4_tile", 4, 2048, 512, 9000),
    ("bf16", "mx4_tile", 3, 1794, 1536, 9001), ("mx4", "mx4_tile", 5, 2048, 288, 9000),
    ("mx4", "mx4_tile", 4, 2048, 1024, 9000), ("mx4", "mx4_tile", 4, 2050, 1024, 9000),
    ("bf16", "mx4_tile", 130, 1024, 800, 9000), ("mx4", "mx4_tile", 130, 1024, 1024, 9000),
]


@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("case", STORED)
def test_every_store_of_the_products(case, glu):
    """bf16 and fp32 results, rows given (some do not exist) and not, strided tokens, lost blocks, a tail."""
    form, kernel, E, N, K, S = case
    g = np.random.default_rng([E, N, K, S, glu, 3])
    codes, scales = weights(E, N, K, g, lost=1)
    off = offsets_of(E, S, S // 40, g)
    rows = g.integers(0, S // 2, S).astype(np.int32)
    rows[::9], rows[4::13] = -5, S
    wide = torch.randn(S, K + 64, device=DEV).to(torch.bfloat16)
    tokens = wide[:, 32:32 + K]
    for X, r in ((tokens, None), (tokens[:S // 2], torch.from_numpy(rows).to(DEV)), (tokens[::2], None)):
        o = off if r is not None else np.minimum(off, len(X)).astype(np.int32)
        kw = {"offsets": torch.from_numpy(o).to(DEV), "rows": r, "glu": glu}
        n = len(X) if r is None else S
        full = n == S  # (fewer slots may go to another kernel)
        X = X.contiguous() if form == "mx4" else X
        results = []
        for dtype in DT.values():
            call = lambda: product(form, codes, scales, X, dtype=dtype, **kw)  # noqa: E731
            y, x = taken(kernel, call) if full else call()
            results.append(y)
        want, bound = exact(codes, scales, x, o, r, glu)
        for y in results:
            assert y.shape == want.shape
            within(y, want, bound + (2.0 ** -8 * want.abs() if y.dtype == torch.bfloat16 else 0), (case, glu, y.dtype))


@pytest.mark.parametrize("case", [
    ("mx4_grad_few", 6, 256, 1024, 9), ("mx4_grad_few", 90, 1552, 512, 1300), ("mx4_grad_few", 40, 1552, 480, 300),
    ("mx4_grad_tile", 5, 296, 2048, 9000), ("mx4_grad_tile", 2, 264, 4096, 9000), ("mx4_grad_tile", 130, 800, 1024, 9001),
    ("mx4_grad_tile", 5, 296, 2112, 9000), ("mx4_grad_tile", 1, 160, 1056, 50000)])
def test_every_store_of_the_gradient(case):
    kernel, E, N, K, S = case
    g = np.random.default_rng([E, N, K, S, 4])
    codes, scales = weights(E, N, K, g, lost=1)
    off = offsets_of(E, S, S // 40, g)
    wide = torch.randn(S, N + 24, device=DEV).to(torch.bfloat16)
    dY = wide[:, 8:8 + N]
    for dtype in DT.values():
        got = taken(kernel, lambda: bm.mx4_product_grad(codes, scales, dY, offsets=torch.from_numpy(off).to(DEV),
                                                        dtype=dtype))
        want, bound = exact(codes, scales, dY, off, grad=True)
        within(got, want, bound + (2.0 ** -8 * want.abs() if dtype == torch.bfloat16 else 0), (case, dtype))


@pytest.mark.parametrize("case", [("bf16", "mx4_rows", 256, 512, 9), ("bf16", "mx4_tile", 2048, 512, 6000),
                                  ("mx4", "mx4_tile", 2048, 1024, 6000), ("mx4", "mx4_tile", 2048, 544, 9000)])
def test_one_expert_without_offsets(case):
    form, kernel, N, K, S = case
    g = np.random.default_rng([N, K, S])
    codes, scales = weights(1, N, K, g)
    X = torch.randn(S, K, device=DEV).to(torch.bfloat16)
    got, x = taken(kernel, lambda: product(form, codes, scales, X))
    want, bound = exact(codes, scales, x, [0, S])
    within(got, want, bound + 2.0 ** -8 * want.abs(), case)
    if kernel == "mx4_tile":
        d = torch.randn(S, N, device=DEV).to(torch.bfloat16)
        back = taken("mx4_grad_tile", lambda: bm.mx4_product_grad(codes, scales, d))
        want, bound = exact(codes, scales, d, [0, S], grad=True)
        within(back, want, bound + 2.0 ** -8 * want.abs(), (case, "grad"))


def test_large_tiles_past_32_bits():
    """Codes of more than 2^32 bytes, tokens past 2^31 entries."""
    E, N, K, S = 33, 16384, 16384, 3000
    codes = torch.zeros((E, N, K // 2), dtype=torch.uint8, device=DEV)
    scales = torch.full((E, N, K // 32), 120, dtype=torch.uint8, device=DEV)
    codes[E - 1] = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device=DEV)
    assert codes.numel() > 1 << 32
    T = (1 << 17) + 700
    X = torch.zeros((T, K), dtype=torch.bfloat16, device=DEV)
    X[-600:] = torch.randn(600, K, device=DEV).to(torch.bfloat16)
    rows = torch.randint(T - 600, T, (S,), dtype=torch.int32, device=DEV)
    off = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    off[E] = S
    w64, x = values(codes[E - 1], scales[E - 1]), X[-600:].double()
    table, size = x @ w64.t().contiguous(), x.abs() @ w64.abs().t().contiguous() * (K + 16) * U
    at = (rows - (T - 600)).long()
    got = taken("mx4_tile", lambda: bm.mx4_product(codes, scales, X, offsets=off, rows=rows))
    within(got, table[at], size[at] + 2.0 ** -8 * table[at].abs(), "far")
    q = bm.mx4_quantize(X)
    x = bm.mx4_dequantize(q[0][-600:].contiguous(), q[1][-600:].contiguous()).double()
    table, size = x @ w64.t().contiguous(), x.abs() @ w64.abs().t().contiguous() * (K + 16) * U
    got = taken("mx4_tile", lambda: bm.mx4_product_q(codes, scales, *q, offsets=off, rows=rows))
    within(got, table[at], size[at] + 2.0 ** -8 * table[at].abs(), "far in MX4")
    del table, size, q, X, x, got
    d = torch.randn(S, N, device=DEV).to(torch.bfloat16)
    back = taken("mx4_grad_tile", lambda: bm.mx4_product_grad(codes, scales, d, offsets=off, dtype=torch.float32))
    within(back, d.double() @ w64, d.double().abs() @ w64.abs() * (N + 16) * U, "far gradient")


def gated(kernel, tokens, times=1):
    """silu(times x) of every x of tokens as the product with glu gives it (times 1 or 6), in fp32."""
    E, N, K, S = {"mx4_rows": (6, 16, 1056, 9), "mx4_few": (90, 776, 1312, 300), "mx4_tile": (4, 1024, 1024, 9000)}[kernel]
    out = []
    for part in tokens.split(S):
        codes = torch.zeros((E, 2 * N, K // 2), dtype=torch.uint8, device=DEV)
        codes[:, :N, 0], codes[:, N:, 0] = {1: 0x02, 6: 0x07}[times], 0x20  # (entry 0 of gate rows, entry 1 of up rows)
        scales = torch.full((E, 2 * N, K // 32), 127, dtype=torch.uint8, device=DEV)
        x = torch.zeros((S, K), dtype=torch.bfloat16, device=DEV)
        x[:len(part), 0], x[:, 1] = part, 1
        off = torch.linspace(0, S, E + 1, device=DEV).round().to(torch.int32)
        y = taken(kernel, lambda: bm.mx4_product(codes, scales, x, offsets=off, glu=True, dtype=torch.float32))
        assert torch.equal(y.nan_to_num(7.0), y[:, :1].expand_as(y).nan_to_num(7.0))
        out.append(y[:len(part), 0].clone())
    return torch.cat(out)


@pytest.mark.parametrize("kernel", ["mx4_rows", "mx4_few", "mx4_tile"])
def test_silu_of_exact_gates(kernel):
    """2^-21 of itself: an ulp (2^-23) each of exponential and reciprocal, half of one of their operands' rounding and
    of the product.  Without the exponent's rounding put back it is |v| 2^-24, 2^-18 at 64."""
    v = torch.cat((torch.linspace(-86, 86, 500), torch.linspace(-8, 8, 200), torch.tensor([0.0, -0.0, 3e38, 1e-38, -200.0])))
    v = v.to(DEV).to(torch.bfloat16)
    want = v.double() / (1 + torch.exp(-v.double()))
    within(gated(kernel, v), want, want.abs() * 2.0 ** -21 + 2.0 ** -126, kernel)
    got = gated(kernel, torch.tensor([1e38, -1e38, torch.nan], device=DEV).to(torch.bfloat16), times=6)
    assert got[0] == torch.inf and got[1:].isnan().all()  # (gates past fp32: silu(-inf) is inf / inf)


# ----------------------------------------------------------------- router
def grow_scratch():
    """A call of another operator that needs more of the library's scratch than any before."""
    logits = torch.randn(1 << 18, 512, device=DEV)
    k, T, E = 1, *logits.shape
    new = lambda n, dt: torch.empty(n, dtype=dt, device=DEV)  # noqa: E731
    i, f = torch.int32, torch.float32
    out = [new(T * k, i), new(T * k, f), new(E + 1, i), new(E + 1, i), new(T * k, i), new(T * k, i), new(T, f), new(2, f)]
    st = bm.lib().bitsmoe_route(logits.data_ptr(), bm.F32, T, E, E, k, None, 1, *(t.data_ptr() for t in out),
                                torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert st == 0
    return out


def equal(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


def test_a_captured_router_of_many_rows_outlives_the_scratch():
    g = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn(3000, 96, generator=g, device=DEV)
    bm.route(x, 4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = bm.route(x, 4)
    for turn in range(4):
        x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        if turn == 1:
            grow_scratch()
        graph.replay()
        want = bm.route(x, 4)
        torch.cuda.synchronize()
        assert equal(r, want), turn


def test_routers_of_many_rows_on_two_streams():
    g = torch.Generator(device=DEV).manual_seed(5)
    xs = [torch.randn(20000, 64, generator=g, device=DEV) for _ in range(2)]
    want = [bm.route(x, 6) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[], []]
    for _ in range(20):
        for x, s, into in zip(xs, streams, got):
            with torch.cuda.stream(s):
                into.append(bm.route(x, 6))
    torch.cuda.synchronize()
    for w, several in zip(want, got):
        assert all(equal(r, w) for r in several)


def test_the_call_without_a_workspace():
    """The same results out of the library's scratch; refused under capture, which it leaves as it was."""
    x = torch.randn(3000, 96, device=DEV)
    T, E, k = 3000, 96, 4
    want = bm.route(x, k)
    out = [torch.empty_like(t) for t in (want.experts, want.weights, want.counts, want.offsets, want.rows, want.slots,
                                         want.lse, want.losses)]
    args = [x.data_ptr(), bm.F32, T, E, E, k, None, 1, *(t.data_ptr() for t in out)]
    assert bm.lib().bitsmoe_route(*args, torch.cuda.current_stream().cuda_stream) == 0
    assert equal(out, (want.experts, want.weights, want.counts, want.offsets, want.rows, want.slots, want.lse,
                       want.losses))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st = bm.lib().bitsmoe_route(*args, torch.cuda.current_stream().cuda_stream)
        text = bm.lib().bitsmoe_last_error()
        r = bm.route(x, k)
    assert st == 1 and b"capture" in text
    graph.replay()
    torch.cuda.synchronize()
    assert equal(r, want)


@pytest.mark.parametrize("T,E,k", [(32769, 24, 3), (70001, 8, 2)])
def test_route_of_more_rows_than_the_longest_256_runs(T, E, k):
    """Whole numbers against a stable sort, sums against 64 bits."""
    g = torch.Generator(device=DEV).manual_seed(T)
    x = torch.randn(T, E, generator=g, device=DEV)
    valid = torch.rand(T, generator=g, device=DEV) < 0.9
    r = bm.route(x, k, valid=valid)
    p = torch.softmax(x.double(), 1) * valid[:, None]
    top = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]  # (ties: the lowest index)
    ex = torch.where(valid[:, None], top, -1)
    assert torch.equal(r.experts.long(), ex)
    w = x.double().gather(1, ex.clamp(min=0))
    w = torch.softmax(w, 1) * valid[:, None]
    within(r.weights, w, w * (k + 70) * U, "weights")
    bucket = torch.where(ex < 0, E, ex).flatten()
    order = torch.sort(bucket, stable=True).indices
    counts = torch.bincount(bucket, minlength=E + 1)[:E]
    n = int(valid.sum())
    assert torch.equal(r.counts.long(), torch.cat((counts, valid.sum()[None])))
    assert torch.equal(r.offsets[1:].long(), counts.cumsum(0)) and int(r.offsets[0]) == 0
    assert torch.equal(r.rows.long(), order // k)
    assert torch.equal(r.slots.flatten()[order].long(), torch.arange(T * k, device=DEV))
    lse = torch.logsumexp(x.double(), 1)
    z = (lse[valid] ** 2).mean()
    balance = E / (k * n * n) * (counts * p.sum(0)).sum()
    # a sum over the rows: at most 128 of a run, 32 parts of the runs, and as many again
    within(r.losses, torch.stack((balance, z)), torch.stack((balance, z)) * 2000 * U, "losses")


# ---------------------------------------------------------------- joining
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,S,d", [(1, 1, 3000, 8), (4, 2, 6, 16), (300, 8, 2400, 72), (300, 8, 7000, 40), (512, 8, 100, 64),
                                     (0, 2, 37, 64), (700, 6, 4200, 264), (16384, 1, 20000, 24),
                                     (2049, 8, 17000, 40), (16385, 1, 1200000, 8), (900, 8, 5, 8),
                                     (66000, 1, 33, 8)])
def test_gradient_of_rows_that_no_slot_names(T, k, S, d, dtype):
    """0, whatever the memory held, for few slots and for many."""
    g = np.random.default_rng([T, k, S, d])
    n = T * k
    at = np.r_[g.permutation(S), -1 - g.integers(0, 9, max(n, 1)), S + g.integers(0, 9, max(n, 1))][:max(2 * n, S)]
    slots = g.permutation(at)[:n].reshape(T, k).astype(np.int32)  # (a row once at most; some name none)
    Z = torch.randn(S, d, device=DEV).to(DT[dtype])
    dY = torch.randn(T, d, device=DEV).to(DT[dtype])
    w = torch.randn(T, k, device=DEV)
    want, wdw = oroute.combine_grad(Z.double().cpu().numpy(), slots, w.double().cpu().numpy(), dY.double().cpu().numpy())
    mags = oroute.combine_grad(Z.double().abs().cpu().numpy(), slots, w.double().cpu().numpy(),
                               dY.double().abs().cpu().numpy())[1]
    want, wdw, mags = (torch.from_numpy(x).to(DEV) for x in (want, wdw, mags))
    unnamed = torch.ones(S, dtype=torch.bool, device=DEV)
    unnamed[torch.from_numpy(slots[(slots >= 0) & (slots < S)].astype(np.int64)).to(DEV)] = False
    slots = torch.from_numpy(slots).to(DEV)
    bound = want.abs() * (U + (2.0 ** -8 if dtype == "bf16" else 0))
    p = lambda t: t.data_ptr() if t is not None and t.numel() else None  # noqa: E731
    # what the workspace holds does not matter: nothing of use, places of slots, places of slots that name the row
    works = [torch.full((S,), -1, device=DEV), torch.randint(0, max(n, 1), (S,), device=DEV),
             torch.arange(S, device=DEV) % max(n, 1), torch.full((S,), 0x7FFFFFFF, device=DEV)]
    if n <= 16384:
        works.append(None)
    for work in works:
        work = None if work is None else work.to(torch.int32)
        dz, dw = torch.full((S, d), torch.nan, device=DEV).to(DT[dtype]), torch.full((T, k), torch.nan, device=DEV)
        st = bm.lib().bitsmoe_combine_grad_all(p(Z), bm.BF16 if dtype == "bf16" else bm.F32, S, p(slots), p(w), p(dY), T,
                                               k, d, p(dz), p(dw), p(work), torch.cuda.current_stream().cuda_stream)
        assert st == 0, bm.lib().bitsmoe_last_error()
        within(dz, want, bound, "dz")
        assert (dz[unnamed] == 0).all()
        within(dw, wdw, mags * (d + 16) * U, "dw")
    junk = torch.full((S, d), torch.nan, device=DEV).to(DT[dtype])
    del junk  # (its memory is what a new tensor of this size gets)
    dz, dw = bm.combine_grad(Z, slots, w, dY)
    within(dz, want, bound, "dz of the binding")
    within(dw, wdw, mags * (d + 16) * U, "dw of the binding")


# --------------------------------------------------------------- together
def experts_of(E, N, K, **ones):
    """Experts whose weights are 0 but for the entries given: {(e, row, column): value}."""
    w = {"gate": torch.zeros(E, N, K), "up": torch.zeros(E, N, K), "down": torch.zeros(E, K, N)}
    for name, at in ones.items():
        for i, v in at.items():
            w[name][i] = v
    return pipeline.mx4_experts(*(w[n].to(DEV) for n in ("gate", "up", "down")))


def test_training_and_serving_give_one_answer():
    """Gate and up are not rounded before silu(g) u: 257 x 257 = 66049 is 66048 in bf16; of 257 rounded first, 65536."""
    ex = experts_of(1, 32, 32, gate={(0, 0, 0): 1, (0, 0, 1): 1}, up={(0, 0, 0): 1, (0, 0, 1): 1}, down={(0, 5, 0): 1})
    x = torch.zeros(3, 32, device=DEV)
    x[:, 0], x[:, 1] = 256, 1
    logits = torch.zeros(3, 1, device=DEV)
    for quantize in (False, True):
        if quantize:
            x[:, 0], x[:, 1] = 4, 0.5  # (both in the format, with one scale) 4.5 x 4.5 silu's sigma: not exact
        y, _ = pipeline.mx4_layer(x.to(torch.bfloat16), logits, ex, 1, quantize_tokens=quantize)
        yt, _, saved = pipeline.mx4_layer(x.to(torch.bfloat16), logits, ex, 1, quantize_tokens=quantize, train=True)
        assert torch.equal(y, yt)
        if not quantize:
            assert (y[:, 5] == 66048).all() and (saved.up[:, 0] == 257).all()


def test_gradient_of_a_token_is_rounded_after_its_slots_are_summed():
    """One expert's part of dx is 256 + 1, the other's -256: 1, where 257 rounded first would leave 0."""
    # gate = 64 (its sigmoid is 1 in fp32), up = 0: d(up) = 64 dh, d(gate) = 0
    ex = experts_of(2, 32, 32, gate={(0, 0, 1): 1, (0, 1, 1): 1, (1, 0, 1): 1}, up={(0, 0, 0): 1, (0, 1, 0): 1, (1, 0, 0): 1},
                    down={(0, 0, 0): 1, (0, 1, 1): 1, (1, 0, 0): -1})
    x = torch.zeros(1, 32, device=DEV)
    x[0, 1] = 64
    _, _, saved = pipeline.mx4_layer(x.to(torch.bfloat16), torch.zeros(1, 2, device=DEV), ex, 2, train=True)
    dy = torch.zeros(1, 32, device=DEV)
    dy[0, 0], dy[0, 1] = 8, 2.0 ** -5  # (both weights are 1/2)
    dx, _ = pipeline.mx4_layer_grad(saved, ex, dy.to(torch.bfloat16))
    assert dx.dtype == torch.bfloat16 and dx[0, 0] == 1 and (dx[0, 1:] == 0).all()


@pytest.mark.parametrize("T,E,k,N,K", [(60, 12, 3, 96, 160), (3000, 4, 2, 512, 1024)])
@pytest.mark.parametrize("quantize", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_layer_stage_by_stage(T, E, k, N, K, quantize, renorm):
    """Every stage of a short batch and of a long one (the large tiles, the router's three launches) in 64 bits from
    what the stage before it gave; tokens in 4 bits as the oracle rounds them."""
    g = torch.Generator(device=DEV).manual_seed(T + 2 * quantize + renorm)
    randn = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    ex = pipeline.mx4_experts(randn(E, N, K) / K ** 0.5, randn(E, N, K) / K ** 0.5, randn(E, K, N) / N ** 0.5)
    x, logits, dy = randn(T, K).to(torch.bfloat16), randn(T, E), randn(T, K).to(torch.bfloat16)
    valid = torch.rand(T, generator=g, device=DEV) < 0.9
    dl = torch.tensor([0.3, 0.1], device=DEV)

    def seen(v):
        if not quantize:
            return v
        return torch.from_numpy(omx4.dequantize(*omx4.quantize(v.double().cpu().numpy()))).to(DEV)

    bf16 = lambda want, bound: bound + 2.0 ** -8 * want.abs()  # noqa: E731
    y, r = pipeline.mx4_layer(x, logits, ex, k, valid=valid, renorm=renorm, quantize_tokens=quantize)
    yt, rt, saved = pipeline.mx4_layer(x, logits, ex, k, valid=valid, renorm=renorm, quantize_tokens=quantize, train=True)
    assert equal(r, rt)
    off = r.offsets.cpu().numpy()
    top = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(r.experts.long(), torch.where(valid[:, None], top, -1))

    def joined(z, zb, got, what):
        """y of rows z [S][K], each known to zb."""
        w = r.weights.double()[:, :, None]
        at = r.slots.long()
        want, size = (w * z[at]).sum(1), (w * zb[at]).sum(1) + (k + 2) * U * (w * z[at].abs()).sum(1)
        within(got, want, size + 2.0 ** -8 * (want.abs() + size), what)

    # serving: h is what the product gives by itself
    call = {"offsets": r.offsets, "rows": r.rows, "glu": True}
    h, _ = product("mx4" if quantize else "bf16", ex.up_codes, ex.up_scales, x, **call)
    want, bound = exact(ex.up_codes, ex.up_scales, seen(x), off, r.rows, True)
    within(h, want, bf16(want, bound), "h")
    z, zb = exact(ex.down_codes, ex.down_scales, seen(h), off)
    joined(z, bf16(z, zb), y, "y")
    # training
    want, bound = exact(ex.up_codes, ex.up_scales, seen(x), off, r.rows)
    within(saved.up, want, bound, "gate and up")
    gate, up = saved.up.chunk(2, dim=1)
    h = (torch.nn.functional.silu(gate) * up).to(torch.bfloat16)
    z, zb = exact(ex.down_codes, ex.down_scales, seen(h), off)
    within(saved.z, z, bf16(z, zb), "z")
    joined(saved.z.double(), torch.zeros_like(z), yt, "y in training")
    dx, dlogits = pipeline.mx4_layer_grad(saved, ex, dy, dlosses=dl)
    dz, dw = bm.combine_grad(saved.z, r.slots, r.weights, dy)
    assert torch.equal(dlogits, bm.route_grad(logits, r, dweights=dw, dlosses=dl, renorm=renorm))
    want = (dy.double()[:, None] * r.weights.double()[:, :, None]).flatten(0, 1)
    within(dz[r.slots.flatten().long()], want, 2.0 ** -8 * want.abs() + 1e-38, "dz")
    dh = exact(ex.down_codes, ex.down_scales, dz, off, grad=True)[0]
    gate, up = gate.double(), up.double()
    sig = torch.sigmoid(gate)
    dup = torch.cat((dh * up * sig * (1 + gate * (1 - sig)), dh * gate * sig), 1)
    part = exact(ex.up_codes, ex.up_scales, dup, off, grad=True)[0]
    want = part[r.slots.long()].sum(1)
    # two roundings to bf16 (of dup's entries, whose errors add up like the entries, and of the sum), 2^-9 each at most
    assert (dx.double() - want).norm() < 2.0 ** -7 * want.norm()


def test_layer_and_gradients_of_many_rows_in_a_graph():
    T, E, k, N, K = 6000, 8, 4, 64, 96
    g = torch.Generator(device=DEV).manual_seed(8)
    randn = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    ex = pipeline.mx4_experts(randn(E, N, K) / 10, randn(E, N, K) / 10, randn(E, K, N) / 8)
    x, logits, dy = randn(T, K).to(torch.bfloat16), randn(T, E), randn(T, K).to(torch.bfloat16)
    dl = torch.tensor([0.3, 0.1], device=DEV)

    def step():
        y, r, saved = pipeline.mx4_layer(x, logits, ex, k, train=True)
        return (y, *r, *pipeline.mx4_layer_grad(saved, ex, dy, dlosses=dl))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for turn in range(4):
        for t in (x, logits, dy):
            t.copy_(randn(*t.shape))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert equal(out, want), turn
