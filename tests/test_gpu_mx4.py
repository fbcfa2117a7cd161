"""4-bit matrices and their products on the GPU against the 64-bit oracle.

Quantisation is exact arithmetic: values are equal, not near.  A product's fp32 sum over K takes one
rounding per k-step of 64 and a few more, each at most 2^-23 of the sum of magnitudes that has been
added (the matrix instruction may truncate): (K/64 + 8) 2^-23 of |a||w| + |bias|; tanh does not
enlarge it and adds two roundings of 2^-23; bf16 outputs add 2^-8 of the value.
"""

import numpy as np
import pytest
import torch

from gpu_common import say
from oracle import mx4
from paper_2111_05188_amd import tp

pytestmark = pytest.mark.gpu

BOTH = [torch.float32, torch.bfloat16]
EPS = 2.0 ** -23


def matrix(rows, K, dtype, seed, layout="rows"):
    """A matrix of spread magnitudes in one of the layouts a caller may have."""
    g = torch.Generator("cuda").manual_seed(seed)
    new = lambda *s: (torch.randn(*s, generator=g, device="cuda")  # noqa: E731
                      * torch.exp2(torch.randint(-6, 7, s, generator=g, device="cuda").float())).to(dtype)
    if layout == "rows":
        return new(rows, K)
    if layout == "pitch":                       # aligned rows with something behind them
        return new(rows, -(-K // 32) * 32 + 32)[:, :K]
    if layout == "odd":                         # neither base nor pitch aligned
        return new(rows, K + 3)[:, 1:K + 1]
    if layout == "turned":
        return new(K, rows).t()
    if layout == "turned-odd":
        return new(K, rows + 3)[:, 1:rows + 1].t()
    raise KeyError(layout)


def host(t):
    return t.double().cpu().numpy()


def back(m, dtype=torch.float32):
    y = torch.full((m.rows, m.K), 7.0, dtype=dtype, device="cuda")
    tp.mx4_dequantize(m, y)
    torch.cuda.synchronize()
    return host(y)


SHAPES = [(1, 1), (1, 31), (2, 32), (3, 33), (31, 64), (32, 65), (33, 128), (5, 301), (64, 1001),
          (130, 256), (257, 96), (1000, 40)]


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("layout", ["rows", "pitch", "odd", "turned", "turned-odd"])
@pytest.mark.parametrize("shape", SHAPES)
def test_quantize(shape, layout, dtype):
    say(f"[mx4] quantize {shape} {layout} {dtype}")
    x = matrix(*shape, dtype, sum(shape), layout)
    m = tp.Mx4T.empty(*shape)
    m.data.fill_(0xEE)                          # stale bytes do not matter
    tp.mx4_quantize(x, m)
    want = mx4.values(host(x))
    assert np.array_equal(back(m), want)
    assert np.array_equal(back(m, torch.bfloat16), want)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", SHAPES + [(17, 8), (50, 9), (9, 2047), (100, 63)])
def test_dequantize_to_rows_of_any_pitch(shape, dtype):
    """Rows one after the other, rows of a pitch, rows that begin anywhere: the same values, and
    nothing else is written."""
    rows, K = shape
    m = tp.mx4_quantize(matrix(rows, K, dtype, 7))
    want = mx4.values(host(matrix(rows, K, dtype, 7)))
    for pitch, begin in ((K, 0), (K, 1), (K + 1, 0), (K + 5, 3), (-(-K // 8) * 8, 0)):
        flat = torch.full((rows * pitch + 16,), 7.0, dtype=dtype, device="cuda")
        y = flat[begin:].as_strided((rows, K), (pitch, 1), begin)
        tp.mx4_dequantize(m, y)
        torch.cuda.synchronize()
        assert np.array_equal(host(y), want), (pitch, begin)
        y.fill_(7.0)
        assert (flat == 7.0).all(), (pitch, begin)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("layout", ["rows", "turned"])
def test_ties_and_special_blocks(layout, dtype):
    x = np.zeros((40, 96), np.float32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.96875, 4.0])
    for r in range(20):
        x[r, :11] = ties * 2.0 ** (r - 10)
        x[r, 32:43] = -ties * 2.0 ** (10 - r)
    x[20, 3], x[21, 40], x[22, 95], x[23, 0] = np.nan, np.inf, -np.inf, -np.nan
    x[24, :3] = 3e38, 1e38, -2e38
    x[25, :4] = 2.0 ** -126, -1.5 * 2.0 ** -126, 2.0 ** -127, 2.0 ** -133
    x[26, :2] = 2.0 ** -133, -2.0 ** -130
    x[27, 0] = 2.0 ** -124
    x[28] = -0.0
    t = torch.from_numpy(x).cuda().to(dtype)
    want = mx4.values(host(t))
    if layout == "turned":
        t = t.t().contiguous().t()
    got = back(tp.mx4_quantize(t))
    assert np.array_equal(got, want, equal_nan=True)


def check(got, a, w, bias, act, dtype, K):
    want, mass = mx4.product(a, w, bias, act)
    tol = (K / 64 + 8) * EPS * mass + (2 * EPS if act == "tanh" else 0.0)
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * np.abs(want)
    nan = np.isnan(want)
    assert np.array_equal(nan, np.isnan(got))
    err = np.abs(np.where(nan, 0, got - want))
    tol = np.where(nan, 0, tol)
    assert (err <= tol).all(), (err.max(), (err / np.maximum(tol, 1e-300)).max())


PRODUCTS = [(1, 1, 1), (1, 5, 31), (2, 100, 64), (16, 33, 65), (31, 64, 301), (33, 1, 128),
            (64, 192, 1001), (70, 100, 512), (129, 257, 320), (300, 100, 1024), (257, 96, 1025),
            (40, 40, 1600), (513, 130, 200), (1030, 70, 1001)]


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", PRODUCTS)
def test_matmul(shape, dtype):
    M, N, K = shape
    say(f"[mx4] matmul {shape} {dtype}")
    a, w = matrix(M, K, torch.float32, 1), matrix(N, K, torch.bfloat16, 2)
    bias = torch.randn(N, generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    act = tp.TP_ACT_TANH if (M + N) % 2 else tp.TP_ACT_NONE
    qa, qw = tp.mx4_quantize(a), tp.mx4_quantize(w)
    va, vw = mx4.values(host(a)), mx4.values(host(w))
    wide = torch.full((M, N + 5), 7.0, dtype=dtype, device="cuda")
    y = wide[:, :N]
    tp.mx4_matmul(qa, qw, y, bias=bias, act=act)
    torch.cuda.synchronize()
    check(host(y), va, vw, host(bias), "tanh" if act else None, dtype, K)
    assert (wide[:, N:] == 7.0).all()           # nothing past the rows
    z = torch.full((M, N), 7.0, dtype=dtype, device="cuda")
    tp.mx4_matmul(qa, qw, z)
    torch.cuda.synchronize()
    check(host(z), va, vw, None, None, dtype, K)


@pytest.mark.parametrize("xdtype,dtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16),
                                          (torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("layout", ["rows", "pitch", "odd"])
@pytest.mark.parametrize("shape", PRODUCTS)
def test_linear(shape, layout, xdtype, dtype):
    M, N, K = shape
    say(f"[mx4] linear {shape} {layout} {xdtype} {dtype}")
    x, w = matrix(M, K, xdtype, 4, layout), matrix(N, K, torch.float32, 5)
    bias = torch.randn(N, generator=torch.Generator("cuda").manual_seed(6), device="cuda")
    act = tp.TP_ACT_TANH if (M + N) % 2 else tp.TP_ACT_NONE
    qw = tp.mx4_quantize(w)
    y = torch.full((M, N), 7.0, dtype=dtype, device="cuda")
    tp.mx4_linear(x, qw, y, bias=bias, act=act)
    torch.cuda.synchronize()
    check(host(y), mx4.values(host(x)), mx4.values(host(w)), host(bias), "tanh" if act else None,
          dtype, K)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("xdtype", [torch.float32, torch.bfloat16, None])
@pytest.mark.parametrize("M,N,K", [(33000, 1536, 1001), (33000, 1001, 301), (16400, 1100, 512),
                                   (16400, 1536, 40)])
def test_many_rows(M, N, K, xdtype, dtype):
    """Rows enough that a workgroup passes many tiles of W: several pieces of y's columns, whole
    and partial, from starting points of each workgroup's own.  Every row is one of 300, whose
    results a small call gives; x in memory, or (None) in 4 bits."""
    say(f"[mx4] many rows {M, N, K} {xdtype} {dtype}")
    base, w = matrix(300, K, xdtype or torch.float32, 25), matrix(N, K, torch.float32, 26)
    bias = torch.randn(N, generator=torch.Generator("cuda").manual_seed(27), device="cuda")
    pick = torch.randint(0, 300, (M,), generator=torch.Generator("cuda").manual_seed(28),
                         device="cuda")
    x = torch.zeros(M, -(-K // 32) * 32, dtype=base.dtype, device="cuda")[:, :K]
    x.copy_(base[pick])
    qw, small = tp.mx4_quantize(w), torch.empty(300, N, dtype=dtype, device="cuda")
    wide = torch.full((M, N + 8), 7.0, dtype=dtype, device="cuda")
    for rows, y in ((base, small), (x, wide[:, :N])):
        if xdtype is None:
            tp.mx4_matmul(tp.mx4_quantize(rows), qw, y, bias=bias)
        else:
            tp.mx4_linear(rows, qw, y, bias=bias)
    torch.cuda.synchronize()
    check(host(small), mx4.values(host(base)), mx4.values(host(w)), host(bias), None, dtype, K)
    assert torch.equal(wide[:, :N], small[pick]) and (wide[:, N:] == 7.0).all()


@pytest.mark.parametrize("M,N,K", [(96, 64, 20000), (5, 7, 65537), (1, 1, 4097), (200, 1001, 3001)])
def test_long_sums(M, N, K):
    """The long axis is split over workgroups and joined in a fixed order."""
    a, w = matrix(M, K, torch.bfloat16, 7, "turned"), matrix(N, K, torch.bfloat16, 8, "turned")
    qa, qw = tp.mx4_quantize(a), tp.mx4_quantize(w)
    bias = torch.randn(N, generator=torch.Generator("cuda").manual_seed(9), device="cuda")
    y = torch.empty(M, N, device="cuda")
    work = tp.mx4_workspace(M, N, K)
    work.fill_(0xEE)
    tp.mx4_matmul(qa, qw, y, bias=bias, act=tp.TP_ACT_TANH, work=work)
    z = torch.empty_like(y)
    tp.mx4_matmul(qa, qw, z, bias=bias, act=tp.TP_ACT_TANH, work=work)
    torch.cuda.synchronize()
    check(host(y), mx4.values(host(a)), mx4.values(host(w)), host(bias), "tanh", torch.float32, K)
    assert torch.equal(y, z)


@pytest.mark.parametrize("M", [3, 40, 700])
def test_nan_stays_in_its_row(M):
    """NaN and infinity in x: that row is NaN, every other one as without them; in w: its column."""
    N, K = 70, 301
    x, w = matrix(M, K, torch.bfloat16, 10), matrix(N, K, torch.float32, 11)
    y0, y = (torch.empty(M, N, device="cuda") for _ in range(2))
    tp.mx4_linear(x, tp.mx4_quantize(w), y0)
    x[1, 300], x[2, 5] = float("nan"), float("inf")
    tp.mx4_linear(x, tp.mx4_quantize(w), y)
    torch.cuda.synchronize()
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[1:3] = False
    assert torch.isnan(y[1:3]).all() and torch.equal(y[keep], y0[keep])
    w[69, 0] = float("inf")
    tp.mx4_linear(x, tp.mx4_quantize(w), y)
    torch.cuda.synchronize()
    assert torch.isnan(y[:, 69]).all() and torch.equal(y[keep][:, :69], y0[keep][:, :69])


def test_what_lies_behind_the_rows_does_not_matter():
    """Rows of 1,001 in a pitch of 1,024: NaN in the padding is not looked at."""
    x = matrix(50, 1001, torch.bfloat16, 12, "pitch")
    w = tp.mx4_quantize(matrix(64, 1001, torch.float32, 13))
    y, z = (torch.empty(50, 64, device="cuda") for _ in range(2))
    tp.mx4_linear(x, w, y)
    x.as_strided((50, x.stride(0) - 1001), (x.stride(0), 1), 1001)[:49].fill_(float("nan"))
    tp.mx4_linear(x, w, z)
    torch.cuda.synchronize()
    assert torch.isfinite(y).all() and torch.equal(y, z)


def test_repeated_rows_and_one_row():
    """A row repeated by a stride of 0; one row with any pitch."""
    w = tp.mx4_quantize(matrix(40, 96, torch.float32, 14))
    one = matrix(1, 96, torch.float32, 15)
    y, z = torch.empty(33, 40, device="cuda"), torch.empty(1, 40, device="cuda")
    tp.mx4_linear(one, w, z)
    m = tp.mx4_quantize(one.expand(33, 96))
    tp.mx4_matmul(m, w, y)
    torch.cuda.synchronize()
    assert torch.equal(y, z.expand(33, 40))


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("K", [1, 31, 301, 1001])
def test_one_row_goes_to_4_bits_on_the_way(K, dtype):
    """A row's pitch means nothing to a single one: with an aligned base, x of any length goes to 4
    bits inside the product, so the workspace stays as it was."""
    w = matrix(192, K, torch.float32, 22)
    x, qw = matrix(1, K, dtype, 23), tp.mx4_quantize(w)
    work = tp.mx4_workspace(1, 192, K).fill_(0xEE)
    y, z = torch.empty(1, 192, device="cuda"), torch.empty(2, 192, device="cuda")
    tp.mx4_linear(x, qw, y, work=work)
    tp.mx4_linear(x.repeat(2, 1), qw, z)
    torch.cuda.synchronize()
    assert (work == 0xEE).all() and torch.equal(y, z[:1])
    assert np.array_equal(back(tp.mx4_quantize(x)), mx4.values(host(x)))
    check(host(y), mx4.values(host(x)), mx4.values(host(w)), None, None, torch.float32, K)


def test_rows_past_four_gigabytes():
    """Source and output rows whose offsets pass 32 bits."""
    K, N, M = 64, 32, 9
    w = tp.mx4_quantize(matrix(N, K, torch.float32, 16))
    x = matrix(M, K, torch.bfloat16, 17)
    y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    tp.mx4_linear(x, w, y)
    st = 300_000_008
    big = torch.empty((M - 1) * st + K, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((M, K), (st, 1))
    far.copy_(x)
    out = torch.empty((M - 1) * st + N, dtype=torch.bfloat16, device="cuda").as_strided((M, N), (st, 1))
    tp.mx4_linear(far, w, out)
    torch.cuda.synchronize()
    assert torch.equal(out.contiguous(), y)


def test_the_most_rows():
    """2^27 rows of odd length, one after the other, and back."""
    rows, K = 1 << 27, 9
    one = matrix(1, K, torch.bfloat16, 24)
    m = tp.mx4_quantize(one.expand(rows, K))
    y = torch.full((rows, K), 7.0, dtype=torch.bfloat16, device="cuda")
    tp.mx4_dequantize(m, y)
    want = torch.from_numpy(mx4.values(host(one))).cuda().bfloat16()
    torch.cuda.synchronize()
    assert (y == want).all()


def test_streams_and_graph_replays():
    """On a stream of its own, and captured in a HIP graph and replayed on new inputs."""
    M, N, K = 300, 100, 301
    x, w = matrix(M, K, torch.bfloat16, 18), matrix(N, K, torch.float32, 19)
    q, a = tp.Mx4T.empty(N, K), tp.Mx4T.empty(M, K)
    y, z, work = torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda"), tp.mx4_workspace(M, N, K)
    back_x = torch.empty(M, K, device="cuda")

    def calls():
        tp.mx4_quantize(w, q)
        tp.mx4_linear(x, q, y, work=work)
        tp.mx4_quantize(x, a)
        tp.mx4_matmul(a, q, z, work=work)
        tp.mx4_dequantize(a, back_x)

    calls()
    torch.cuda.synchronize()
    first = [t.clone() for t in (y, z, back_x)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        calls()
    s.synchronize()
    for p, t in zip(first, (y, z, back_x)):
        assert torch.equal(p, t)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for k in range(3):
        x.copy_(matrix(M, K, torch.bfloat16, 30 + k))
        w.copy_(matrix(N, K, torch.float32, 40 + k))
        calls()
        want = [t.clone() for t in (y, z, back_x)]
        for t in (y, z, back_x):
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for p, t in zip(want, (y, z, back_x)):
            assert torch.equal(p, t)


def test_memory_of_a_call_on_another_stream():
    """What a call on a stream allocates itself is not handed out again before it has run: the
    current stream's next memory is filled with other bytes while the call waits for its turn."""
    M, N, K = 500, 100, 1601
    x, w = matrix(M, K, torch.float32, 20, "odd"), matrix(N, K, torch.float32, 21)
    qa, qw = tp.mx4_quantize(x), tp.mx4_quantize(w)
    want, back_x = torch.empty(M, N, device="cuda"), torch.empty(M, K, device="cuda")
    tp.mx4_linear(x, qw, want)
    tp.mx4_dequantize(qa, back_x)
    torch.cuda.synchronize()
    nb = tp.mx4_workspace(M, N, K).numel()
    s = torch.cuda.Stream()
    for call in (lambda y: tp.mx4_linear(x, qw, y, stream=s),
                 lambda y: tp.mx4_matmul(qa, qw, y, stream=s),
                 lambda y: tp.mx4_matmul(tp.mx4_quantize(x, stream=s), qw, y, stream=s)):
        y = torch.empty(M, N, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            torch.cuda._sleep(500_000_000)     # a fifth of a second
        call(y)
        assert not s.query()
        others = [torch.full((n,), 0xEE, dtype=torch.uint8, device="cuda")
                  for n in (nb, nb, tp.mx4_bytes(M, K))]
        torch.cuda.current_stream().synchronize()
        s.synchronize()
        del others
        assert torch.equal(y, want)


def test_refusals():
    x = torch.zeros(4, 64, device="cuda")
    w = tp.mx4_quantize(torch.zeros(5, 64, device="cuda"))
    y = torch.empty(4, 5, device="cuda")
    with pytest.raises(tp.TPError) as e:
        tp.mx4_quantize(torch.zeros(4, 64, 2, device="cuda")[:, :, 0])
    assert e.value.code == tp.TP_EUNSUPPORTED
    with pytest.raises(tp.TPError) as e:
        tp.mx4_linear(x, w, y, work=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == tp.TP_EINVAL and "workspace" in str(e.value)
    with pytest.raises(tp.TPError):
        tp.mx4_linear(x, w, y, act=9)
    with pytest.raises(AssertionError):
        tp.mx4_linear(x[:, :32], w, y)
    with pytest.raises(tp.TPError) as e:
        tp.mx4_matmul(tp.mx4_quantize(x[:, :32]), w, y)
    assert "elements a row" in str(e.value)
