"""GPU checks of the token operators against plain implementations: codes and factors bit for bit, products against 64-bit
arithmetic with bounds derived from the roundings of the definition."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
F64 = torch.float64


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _acts(seed, *shape, dtype=torch.float32, pad=0, offset=0):
    g = _gen(seed)
    wide = torch.randn(*shape[:-1], shape[-1] + pad + offset, generator=g, device="cuda")
    wide = torch.where(torch.rand(wide.shape[-1], generator=g, device="cuda") < 0.05, 20 * wide, wide).to(dtype)
    return wide[..., offset:offset + shape[-1]]


def _codes(seed, *shape):
    return torch.randint(-128, 128, shape, generator=_gen(seed), device="cuda").to(torch.int8)


def plain_quantize(x):
    """The definition in numpy, whose fp32 division is IEEE and whose rint is half to even."""
    v = x.detach().float().cpu().numpy()
    with np.errstate(all="ignore"):
        m = np.abs(v).max(-1)
        s = np.where(m == 0, np.float32(1), np.maximum(m / np.float32(127), np.float32(2.0 ** -126))).astype(np.float32)
        bad = ~np.isfinite(m)
        z = np.clip(np.rint(v / s[..., None]), -128, 127)
        z[bad] = 0
        s[bad] = np.nan
    return z.astype(np.int8), s


# ------------------------------------------------------------------------------------------------ codes
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (3, 64), (5, 100), (2, 3, 1024), (300, 257), (1, 4096), (9, 5000), (2, 20000), (2, 40001)], ids=str)
def test_quantize_tokens_bit_exact(q8, dtype, shape):
    x = _acts(1, *shape, dtype=TYPES[dtype])
    z, s = q8.q8_quantize_tokens(x)
    zr, sr = plain_quantize(x)
    assert z.shape == x.shape and s.shape == x.shape[:-1]
    assert np.array_equal(s.cpu().numpy(), sr)
    assert np.array_equal(z.cpu().numpy(), zr)
    for out, t in ((q8.Q8_F32, torch.float32), (q8.Q8_F16, torch.float16), (q8.Q8_BF16, torch.bfloat16)):
        r = q8.q8_dequantize_tokens(z, s, out)
        assert r.dtype == t and torch.equal(r, (z.float() * s[..., None]).to(t))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("C,pad,offset", [(64, 16, 0), (64, 1, 0), (100, 3, 1), (256, 0, 8), (129, 7, 5), (1000, 24, 3)])
def test_strided_rows_and_what_lies_between(q8, dtype, C, pad, offset):
    x = _acts(2, 13, C, dtype=TYPES[dtype], pad=pad, offset=offset)
    wide = torch.full((13, C + 11), 77, dtype=torch.int8, device="cuda")
    scale = torch.empty(13, device="cuda")
    z, s = q8.q8_quantize_tokens(x, out=wide[:, 5:5 + C], scale=scale)
    zr, sr = plain_quantize(x)
    assert np.array_equal(z.cpu().numpy(), zr) and np.array_equal(scale.cpu().numpy(), sr)
    assert bool((wide[:, :5] == 77).all()) and bool((wide[:, 5 + C:] == 77).all())
    back = torch.full((13, C + 9), 3.0, dtype=TYPES[dtype], device="cuda")
    q8.q8_dequantize_tokens(z, s, out=back[:, 4:4 + C])
    assert torch.equal(back[:, 4:4 + C], (z.float() * s[:, None]).to(TYPES[dtype]))
    assert bool((back[:, :4] == 3).all()) and bool((back[:, 4 + C:] == 3).all())


@pytest.mark.parametrize("C", [48, 515, 9000])
def test_extreme_rows(q8, C):
    x = _acts(3, 16, C)
    x[0] = 0
    x[1, C // 2] = float("inf")
    x[2, C - 1] = float("nan")
    x[3, 0] = -float("inf")
    x[4] *= 2.0 ** 120
    x[5] *= 2.0 ** -140          # subnormal values
    x[6] = 0
    x[6, 3] = 2.0 ** -149        # the least one alone
    x[7] = 3.4028234663852886e38
    x[8] *= 2.0 ** -62           # both sides of the factor at which a division replaces the multiplication
    x[9] *= 2.0 ** -70
    x[10] = torch.arange(C, device="cuda") % 255 - 127.0   # ties: factor 1, codes as they are ...
    x[11] = (torch.arange(C, device="cuda") % 255 - 127.0) / 2
    x[11, 0] = 127               # ... and halves
    x[12] = -0.0
    z, s = q8.q8_quantize_tokens(x)
    zr, sr = plain_quantize(x)
    assert np.array_equal(s.cpu().numpy(), sr, equal_nan=True)
    assert np.array_equal(z.cpu().numpy(), zr)
    assert bool(torch.isnan(q8.q8_dequantize_tokens(z, s)[1:4]).all())


def test_no_tokens_and_offsets_past_32_bits(q8):
    z, s = q8.q8_quantize_tokens(torch.empty(0, 64, device="cuda"))
    assert z.shape == (0, 64) and s.shape == (0,)
    assert q8.q8_dequantize_tokens(z, s).shape == (0, 64)
    assert q8.q8_linear(z, _codes(1, 32, 64), torch.ones(32, device="cuda"), x_scale=s).shape == (0, 32)
    # rows 2^31 elements apart
    big = torch.empty(3 << 30, dtype=torch.float16, device="cuda")
    x = big.as_strided((2, 100), (1 << 31, 1))
    x.copy_(_acts(4, 2, 100, dtype=torch.float16))
    z, s = q8.q8_quantize_tokens(x)
    zr, sr = plain_quantize(x)
    assert np.array_equal(z.cpu().numpy(), zr) and np.array_equal(s.cpu().numpy(), sr)
    w, ws = _codes(5, 24, 100), torch.rand(24, device="cuda")
    assert torch.equal(q8.q8_linear(x, w, ws), q8.q8_linear(x.contiguous(), w, ws))
    y = big.as_strided((2, 24), (1 << 31, 1), 128)
    q8.q8_linear(z, w, ws, x_scale=s, out=y)
    assert torch.equal(y, q8.q8_linear(z, w, ws, x_scale=s, out_type=q8.Q8_F16))


# ------------------------------------------------------------------------------------------------ product
def check_linear(y, z, s, w, ws, bias):
    """y against the 64-bit product.  The definition rounds float(acc), its two products and the sum with the bias to fp32,
    half a step (2^-24) each, and the result to y's type; subnormal results are off by half a least step."""
    exact = torch.outer(s.to(F64), ws.to(F64)) * (z.to(F64) @ w.to(F64).t())
    total = exact if bias is None else exact + bias.to(F64)
    info = torch.finfo(y.dtype)
    tol = 3 * 2.0 ** -24 * exact.abs() * 1.000001 + (2.0 ** -24 * total.abs() if bias is not None else 0)
    tol = tol + (total.abs() + tol) * (info.eps / 2 if y.dtype != torch.float32 else 0) + info.smallest_normal * info.eps
    if y.dtype == torch.float16:
        # the last fp16 number is 2^16 - 2^5; from half a step above it on, 2^16 - 2^4, values round to infinity
        bound = tol - total.abs() * info.eps / 2
        gone = torch.isinf(y)
        assert bool((gone == (total.abs() >= 65520))[(total.abs() - 65520).abs() > bound].all())
        assert bool((torch.sign(y.to(F64)) == torch.sign(total))[gone].all())
        y, total = torch.where(gone, 0, y), torch.where(gone, 0, total)
    assert bool(((y.to(F64) - total).abs() <= tol).all()), float(((y.to(F64) - total).abs() / tol).max())


LINEAR = [  # M, C, K
    (1, 1, 1), (1, 64, 16), (1, 4096, 512), (2, 100, 33), (7, 333, 17), (8, 256, 64), (9, 256, 64), (16, 640, 48), (17, 1000, 100),
    (31, 2048, 130), (33, 96, 257), (64, 512, 512), (65, 128, 128), (127, 777, 255), (128, 1024, 256), (129, 1032, 1000),
    (200, 320, 264), (257, 64, 520), (384, 2064, 136), (1000, 176, 80), (3, 20000, 40), (40, 12000, 24), (300, 5000, 300),
]


@pytest.mark.parametrize("M,C,K", LINEAR)
def test_linear_codes(q8, M, C, K):
    for out, pad, bias in ((q8.Q8_F32, 0, True), (q8.Q8_BF16, 16, False), (q8.Q8_F16, 5, True)):
        zw = _codes(10 + M, M, C + pad)
        wide = _codes(11 + K, K, C + pad)
        z, w = zw[:, :C], wide[:, :C]
        g = _gen(12 + C)
        s, ws = torch.rand(M, generator=g, device="cuda") + 0.1, (torch.rand(K, generator=g, device="cuda") + 0.1) / (1000 * C ** 0.5)
        b = torch.randn(K, generator=g, device="cuda") if bias else None
        y = q8.q8_linear(z, w, ws, x_scale=s, bias=b, out_type=out)
        check_linear(y, z, s, w, ws, b)
        none = torch.empty(0, dtype=torch.uint8, device="cuda")
        assert torch.equal(q8.q8_linear(z, w, ws, x_scale=s, bias=b, out_type=out, workspace=none), y)   # the result without scratch
        wide_y = torch.full((M, K + 7), 9.0, dtype=y.dtype, device="cuda")
        q8.q8_linear(z, w, ws, x_scale=s, bias=b, out=wide_y[:, 3:3 + K])
        assert torch.equal(wide_y[:, 3:3 + K], y) and bool((wide_y[:, :3] == 9).all()) and bool((wide_y[:, 3 + K:] == 9).all())
    q8.q8_read_status()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("M,C,K", LINEAR)
def test_linear_of_activations_is_that_of_their_codes(q8, M, C, K, dtype):
    x = _acts(20 + M, M, C, dtype=TYPES[dtype], pad=C % 3)
    w, ws = _codes(21, K, C), torch.rand(K, device="cuda") / 1000
    z, s = q8.q8_quantize_tokens(x)
    y = q8.q8_linear(x, w, ws, out_type=q8.Q8_F32)
    check_linear(y, z, s, w, ws, None)
    assert torch.equal(y, q8.q8_linear(z, w, ws, x_scale=s, out_type=q8.Q8_F32))
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    assert torch.equal(y, q8.q8_linear(x, w, ws, out_type=q8.Q8_F32, workspace=none))
    # a token's result is its own, whatever is beside it
    t = M // 2
    assert torch.equal(q8.q8_linear(x[t:t + 1], w, ws, out_type=q8.Q8_F32), y[t:t + 1])
    q8.q8_read_status()


@pytest.mark.parametrize("M", [1, 5, 24, 150, 600])
@pytest.mark.parametrize("C", [131071, 131056])
def test_longest_reduction_at_its_extremes(q8, M, C):
    z = torch.full((M, C), -128, dtype=torch.int8, device="cuda")
    w = torch.full((20, C), -128, dtype=torch.int8, device="cuda")
    w[3] = 127
    ones = torch.ones(M, device="cuda")
    y = q8.q8_linear(z, w, torch.ones(20, device="cuda"), x_scale=ones, out_type=q8.Q8_F32)
    check_linear(y, z, ones, w, torch.ones(20, device="cuda"), None)
    assert float(y[0, 0]) == float(np.float32(128 * 128 * C)) and float(y[-1, 3]) == -float(np.float32(128 * 127 * C))


@pytest.mark.parametrize("M", [4, 20, 300])
def test_bad_tokens_do_not_spread(q8, M):
    x = _acts(30, M, 320)
    w, ws = _codes(31, 96, 320), torch.rand(96, device="cuda")
    good = q8.q8_linear(x, w, ws)
    x[1, 7], x[3, 319] = float("nan"), float("inf")
    y = q8.q8_linear(x, w, ws)
    assert bool(torch.isnan(y[1]).all()) and bool(torch.isnan(y[3]).all())
    keep = [t for t in range(M) if t not in (1, 3)]
    assert torch.equal(y[keep], good[keep])


def test_linear_leading_dimensions_views_and_broadcasts(q8):
    x = _acts(32, 3, 5, 64, dtype=torch.bfloat16)
    w, ws = _codes(33, 40, 64), torch.rand(40, device="cuda")
    y = q8.q8_linear(x, w, ws)
    assert y.shape == (3, 5, 40) and torch.equal(y.view(15, 40), q8.q8_linear(x.reshape(15, 64), w, ws))
    assert torch.equal(q8.q8_linear(x[1, 2], w, ws), y[1, 2])
    for bad in (x.transpose(0, 1), x[..., ::2].expand(3, 5, 32), x[0, 0].expand(4, 64), x.double(), x.cpu()):
        with pytest.raises(TypeError):
            q8.q8_linear(bad, w[:, :bad.shape[-1]], ws)
    with pytest.raises(TypeError):
        q8.q8_linear(x, w, ws[:39])
    with pytest.raises(TypeError):
        q8.q8_linear(x, w, ws, bias=torch.zeros(40, dtype=torch.float16, device="cuda"))
    with pytest.raises(q8.Q8Error):
        q8.q8_linear(x, w, ws, x_scale=torch.ones(15, device="cuda"))


@pytest.mark.parametrize("M,C,K", [(1, 1024, 256), (24, 1024, 256), (300, 1024, 512), (40, 1001, 130)])
def test_linear_on_another_stream_and_replayed(q8, M, C, K):
    x = _acts(40, M, C, dtype=torch.bfloat16)
    w, ws = _codes(41, K, C), torch.rand(K, device="cuda")
    want = q8.q8_linear(x, w, ws)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = q8.q8_linear(x, w, ws)
    torch.cuda.current_stream().wait_stream(other)
    assert torch.equal(got, want)
    graph, y = torch.cuda.CUDAGraph(), torch.empty_like(want)
    with torch.cuda.graph(graph):
        z, s = q8.q8_quantize_tokens(x)
        q8.q8_linear(z, w, ws, x_scale=s, out=y)
        y2 = q8.q8_linear(x, w, ws)
    for seed in (42, 43):
        x.copy_(_acts(seed, M, C, dtype=torch.bfloat16))
        graph.replay()
        want = q8.q8_linear(x, w, ws)
        assert torch.equal(y, want) and torch.equal(y2, want)
    q8.q8_read_status()


# ------------------------------------------------------------------------------------------------ experts
def _experts(seed, C, I, E):
    g = _gen(seed)
    w = lambda *s: torch.randn(*s, generator=g, device="cuda").mul_(32).round_().clamp_(-127, 127).to(torch.int8)  # noqa: E731
    u = lambda *s, n: (0.5 + torch.rand(*s, generator=g, device="cuda")) / (32 * n ** 0.5)  # noqa: E731
    return (torch.randn(E, C, generator=g, device="cuda") / C ** 0.5, w(E, 2 * I, C), u(E, 2 * I, n=C), w(E, C, I), u(E, C, n=I))


def plain_moe(x, router, wgu, sgu, wd, sd, k, renorm):
    """The definition in 64 bits, and how far 32-bit arithmetic on 22 bits of each row may be from it.

    x and h are held to 2^-22 of their row's largest at the worst (a code of 24 bits is off by half a step of 2^-23, its factor
    by two roundings), so a sum is off by that times the sum of the weights' magnitudes; sums are exact; scaling, the gate
    (expf within 2 ulp, a sum, a division, two products) and the probabilities are a few roundings of 2^-24 each."""
    T, C = x.shape
    I = wd.shape[-1]
    v = x.to(F64)
    logits = v @ router.to(F64).t()
    y, tol = torch.zeros(T, C, dtype=F64, device="cuda"), torch.zeros(T, C, dtype=F64, device="cuda")
    ids, probs = [], []
    step, u = 2.0 ** -22, 2.0 ** -24
    for t in range(T):
        row = logits[t].tolist()
        chosen = sorted(range(len(row)), key=lambda e: (-row[e], e))[:k]
        soft = torch.softmax(logits[t, chosen] if renorm else logits[t], -1)
        p = soft.tolist() if renorm else [float(soft[e]) for e in chosen]
        ids.append(chosen)
        probs.append(p)
        for j, e in enumerate(chosen):
            a = wgu[e].to(F64)
            gu = (a @ v[t]) * sgu[e].to(F64)
            dgu = step * v[t].abs().max() * a.abs().sum(-1) * sgu[e].to(F64) + 4 * u * gu.abs()
            g, up = gu[:I], gu[I:]
            h = g * torch.sigmoid(g) * up
            dh = 1.1 * dgu[:I] * (up.abs() + dgu[I:]) + (g * torch.sigmoid(g)).abs() * dgu[I:] + 16 * u * h.abs()
            dh = dh + step * (h.abs().max() + dh.max())
            b = wd[e].to(F64)
            out = (b @ h) * sd[e].to(F64)
            y[t] += p[j] * out
            tol[t] += p[j] * ((b.abs() @ dh) * sd[e].to(F64) + 40 * u * out.abs())
    return y, tol, torch.tensor(ids, dtype=torch.int32, device="cuda"), torch.tensor(probs, dtype=F64, device="cuda")


def check_moe(got, want):
    y, ids, probs = got
    ry, tol, rids, rprobs = want
    assert torch.equal(ids, rids)
    assert bool(((probs.to(F64) - rprobs).abs() <= 32 * 2.0 ** -24 * rprobs + 2.0 ** -140).all())
    info = torch.finfo(y.dtype)
    tol = tol + (ry.abs() + tol) * info.eps / 2 + info.smallest_normal * info.eps
    assert bool(((y.to(F64) - ry).abs() <= tol).all()), float(((y.to(F64) - ry).abs() / tol).max())


MOE = [  # T, C, I, E, k
    (1, 64, 32, 4, 2), (1, 1, 1, 1, 1), (1, 2048, 768, 8, 8), (2, 33, 7, 1, 1), (3, 100, 36, 5, 2), (5, 1000, 520, 17, 2), (16, 256, 128, 16, 4),
    (2, 1024, 2048, 3, 2), (16, 48, 16, 1, 1), (12, 96, 80, 2, 2), (17, 128, 64, 8, 3), (40, 80, 48, 6, 2), (4, 32, 16, 1024, 32), (7, 333, 250, 40, 5),
    (1, 5000, 96, 3, 1), (3, 64, 5008, 2, 1), (9, 512, 256, 64, 6), (16, 20000, 48, 2, 2), (16, 16, 9000, 2, 1),
]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("T,C,I,E,k", MOE)
def test_moe(q8, T, C, I, E, k, dtype):
    x = _acts(50 + T, T, C, dtype=TYPES[dtype], pad=T % 3, offset=T % 2)
    experts = _experts(51, C, I, E)
    for renorm in (True, False):
        got = q8.q8_moe(x, *experts, k, renormalize=renorm)
        check_moe(got, plain_moe(x, *experts, k, renorm))
    wide = torch.full((T, C + 5), 2.0, dtype=x.dtype, device="cuda")
    q8.q8_moe(x, *experts, k, renormalize=False, out=wide[:, 2:2 + C])
    assert torch.equal(wide[:, 2:2 + C], got[0]) and bool((wide[:, :2] == 2).all()) and bool((wide[:, 2 + C:] == 2).all())
    t = T // 2   # a token's result is its own, whatever is beside it
    alone = q8.q8_moe(x[t], *experts, k, renormalize=False)
    assert all(torch.equal(a, b[t]) for a, b in zip(alone, got))
    q8.q8_read_status()


def test_moe_ties_and_bad_tokens(q8):
    T, C, I, E, k = 6, 160, 64, 12, 3
    x = _acts(60, T, C)
    router, *rest = _experts(61, C, I, E)
    router[5], router[9], router[2] = router[7], router[7], router[1]   # equal logits: the lower index first
    x[0] = 0                                                             # all of them equal
    good = q8.q8_moe(x, router, *rest, k)
    check_moe(good, plain_moe(x, router, *rest, k, True))
    assert good[1][0].tolist() == [0, 1, 2] and bool((good[0][0] == 0).all())
    x[2, 11], x[4, 0] = float("nan"), -float("inf")
    y, ids, probs = q8.q8_moe(x, router, *rest, k)
    keep = [0, 1, 3, 5]
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip((y, ids, probs), good))
    assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[4]).all())
    assert bool(((ids >= 0) & (ids < E)).all()) and ids[2].tolist() == [0, 1, 2]
    router[0, 3] = float("nan")        # an expert that nothing can choose
    ids = q8.q8_moe(x, router, *rest, k)[1]
    assert bool((ids[[1, 3, 5]] != 0).all())


@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** -30, 2.0 ** 40])
def test_moe_of_small_and_large_activations(q8, scale):
    x = _acts(62, 3, 256) * scale
    experts = _experts(63, 256, 96, 4)
    y, ids, probs = q8.q8_moe(x, *experts, 2)
    ry, tol, rids, _ = plain_moe(x, *experts, 2, True)
    assert torch.equal(ids, rids)
    assert bool(((y.to(F64) - ry).abs() <= tol + ry.abs() * 2.0 ** -24 + 2.0 ** -126).all())


def test_moe_on_another_stream_and_replayed(q8):
    T, C, I, E, k = 4, 512, 256, 16, 4
    x = _acts(64, T, C, dtype=torch.bfloat16)
    experts = _experts(65, C, I, E)
    graph = torch.cuda.CUDAGraph()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    want = q8.q8_moe(x, *experts, k)
    with torch.cuda.stream(other):
        got = q8.q8_moe(x, *experts, k)
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.graph(graph):
        out = q8.q8_moe(x, *experts, k)
        twice = q8.q8_moe(out[0], *experts, k)
    for seed in (66, 67):
        x.copy_(_acts(seed, T, C, dtype=torch.bfloat16))
        graph.replay()
        want = q8.q8_moe(x, *experts, k)
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert all(torch.equal(a, b) for a, b in zip(twice, q8.q8_moe(want[0], *experts, k)))
    q8.q8_read_status()


def test_moe_workspace_contents_do_not_matter(q8):
    x = _acts(68, 5, 128)
    experts = _experts(69, 128, 64, 8)
    d = q8.q8_moe_desc(0, 0, 5, 128, 64, 8, 2, q8.Q8_F32, 1, 0)
    n = q8.q8_moe_workspace_bytes(d)
    want = q8.q8_moe(x, *experts, 2)
    for fill in (0, 255, 127):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        for _ in range(2):
            assert all(torch.equal(a, b) for a, b in zip(q8.q8_moe(x, *experts, 2, workspace=ws), want))
    with pytest.raises(q8.Q8Error):
        q8.q8_moe(x, *experts, 2, workspace=ws[:n - 1])


# ------------------------------------------------------------------------------------------------ edges between the kernels
@pytest.mark.parametrize("C,K", [(512, 384), (1001, 130), (136, 1027)])
def test_linear_rows_do_not_depend_on_the_batch(q8, C, K):
    """Sums are exact, so a token's results are the same bits in every batch, whichever kernel takes it."""
    z, s = q8.q8_quantize_tokens(_acts(80, 300, C))
    w, ws, bias = _codes(81, K, C), torch.rand(K, device="cuda"), torch.randn(K, generator=_gen(82), device="cuda")
    want = q8.q8_linear(z, w, ws, x_scale=s, bias=bias, out_type=q8.Q8_F32)
    check_linear(want, z, s, w, ws, bias)
    for M in (1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 24, 31, 33, 63, 65, 127, 129, 192, 255, 256, 257, 288):
        assert torch.equal(q8.q8_linear(z[:M], w, ws, x_scale=s[:M], bias=bias, out_type=q8.Q8_F32), want[:M]), M
    empty = torch.empty(0, dtype=torch.uint8, device="cuda")
    assert torch.equal(q8.q8_linear(z, w, ws, x_scale=s, bias=bias, out_type=q8.Q8_F32, workspace=empty), want)
    q8.q8_read_status()


@pytest.mark.parametrize("M", [1, 12, 40, 300])
@pytest.mark.parametrize("at,ld", [(1, 513), (8, 520), (16, 528), (3, 512)])
def test_linear_from_any_address(q8, M, at, ld):
    C, K = 500, 260
    flat = _codes(83, at + K * ld)
    w = flat[at:].view(K, ld)[:, :C]
    x = _codes(84, at + M * ld)[at:].view(M, ld)[:, :C]
    s, ws = torch.rand(M, device="cuda"), torch.rand(K, device="cuda")
    y = torch.zeros(at + M * ld, dtype=torch.float16, device="cuda")[at:].view(M, ld)[:, :K]
    q8.q8_linear(x, w, ws, x_scale=s, out=y)
    assert torch.equal(y, q8.q8_linear(x.contiguous(), w.contiguous(), ws, x_scale=s, out_type=q8.Q8_F16))
    check_linear(y, x, s, w, ws, None)


@pytest.mark.parametrize("T,C,I,E,k", [(3, 256, 128, 6, 2), (16, 264, 72, 5, 2), (1, 130, 34, 4, 4)])
def test_moe_from_any_address(q8, T, C, I, E, k):
    x = _acts(85, T, C, dtype=torch.float16)
    router, wgu, sgu, wd, sd = _experts(86, C, I, E)
    want = q8.q8_moe(x, router, wgu, sgu, wd, sd, k)
    check_moe(want, plain_moe(x, router, wgu, sgu, wd, sd, k, True))
    for a, b in ((1, 0), (0, 1), (8, 8), (24, 3)):
        gu = torch.empty(wgu.numel() + a, dtype=torch.int8, device="cuda")[a:].view(wgu.shape).copy_(wgu)
        down = torch.empty(wd.numel() + b, dtype=torch.int8, device="cuda")[b:].view(wd.shape).copy_(wd)
        r = torch.empty(router.numel() + 1, device="cuda")[1:].view(router.shape).copy_(router)
        assert all(torch.equal(p, q) for p, q in zip(q8.q8_moe(x, r, gu, sgu, down, sd, k), want))


@pytest.mark.parametrize("T,k,E", [(20, 20, 32), (33, 32, 40), (16, 16, 16), (9, 32, 32)])
def test_moe_of_many_chosen_experts(q8, T, k, E):
    C, I = 96, 40
    x, experts = _acts(87, T, C), _experts(88, C, I, E)
    for renorm in (True, False):
        check_moe(q8.q8_moe(x, *experts, k, renormalize=renorm), plain_moe(x, *experts, k, renorm))


def test_moe_where_one_expert_takes_all(q8):
    """Every token chooses the same two experts, others none: sixteen tokens of an item, and experts with nothing to do."""
    T, C, I, E, k = 16, 320, 200, 48, 2
    x = _acts(89, T, C).abs()
    router, *rest = _experts(90, C, I, E)
    router[:] = -router.abs()
    router[17] = 1.0
    router[40] = 2.0
    got = q8.q8_moe(x, router, *rest, k)
    assert got[1].tolist() == [[40, 17]] * T
    check_moe(got, plain_moe(x, router, *rest, k, True))


def test_calls_on_two_streams_at_once(q8):
    """Each call with a workspace of its own; results as one after the other."""
    T, C, I, E, k = 5, 512, 320, 24, 4
    xs = [_acts(91 + i, T, C, dtype=torch.bfloat16) for i in range(2)]
    experts = _experts(93, C, I, E)
    w, ws = _codes(94, 640, C), torch.rand(640, device="cuda")
    want = [(q8.q8_moe(x, *experts, k), q8.q8_linear(x, w, ws)) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, (x, stream) in enumerate(zip(xs, streams)):
            with torch.cuda.stream(stream):
                got[i].append((q8.q8_moe(x, *experts, k), q8.q8_linear(x, w, ws)))
    torch.cuda.synchronize()
    for i in range(2):
        for moe, y in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(moe, want[i][0])) and torch.equal(y, want[i][1])
    q8.q8_read_status()


def test_two_graphs_share_a_workspace(q8):
    T, C, I, E, k = 3, 256, 192, 8, 2
    x, experts = _acts(95, T, C), _experts(96, C, I, E)
    w, ws = _codes(97, 2048, C), torch.rand(2048, device="cuda")
    d = q8.q8_moe_desc(0, 0, T, C, I, E, k, q8.Q8_F32, 1, 0)
    space = torch.empty(max(q8.q8_moe_workspace_bytes(d), 8 << 20), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = q8.q8_moe(x, *experts, k, workspace=space)
            outs.append((*y, q8.q8_linear(y[0], w, ws, workspace=space)))
        graphs.append(g)
    for seed in (98, 99):
        x.copy_(_acts(seed, T, C))
        for g in graphs:
            g.replay()
        want = q8.q8_moe(x, *experts, k)
        want = (*want, q8.q8_linear(want[0], w, ws))
        for o in outs:
            assert all(torch.equal(a, b) for a, b in zip(o, want))


def test_weights_past_32_bits(q8):
    C, K = 8192, 300000
    w = torch.empty(K, C, dtype=torch.int8, device="cuda")
    w.random_(-128, 128, generator=_gen(110))
    ws = torch.rand(K, generator=_gen(111), device="cuda")
    for M in (1, 12, 40, 300):
        x = _acts(112 + M, M, C, dtype=torch.float16)
        y = q8.q8_linear(x, w, ws)
        for at in (0, 262143, K - 260):
            assert torch.equal(y[:, at:at + 260], q8.q8_linear(x, w[at:at + 260], ws[at:at + 260])), (M, at)
    del w
    C, I, E, k = 4096, 2100, 160, 2
    g = _gen(113)
    wgu = torch.empty(E, 2 * I, C, dtype=torch.int8, device="cuda").random_(-128, 128, generator=g)
    wd = torch.empty(E, C, I, dtype=torch.int8, device="cuda").random_(-128, 128, generator=g)
    sgu, sd = torch.rand(E, 2 * I, generator=g, device="cuda") / 4096, torch.rand(E, C, generator=g, device="cuda") / 4096
    router = torch.zeros(E, C, device="cuda")
    router[E - 1], router[E - 2], router[0] = 1.0 / C, 0.99 / C, 0.98 / C
    for T in (1, 3, 6):
        x = _acts(114, T, C).abs()
        got = q8.q8_moe(x, router, wgu, sgu, wd, sd, k)
        assert got[1].tolist() == [[E - 1, E - 2]] * T
        check_moe(got, plain_moe(x, router, wgu, sgu, wd, sd, k, True))
    q8.q8_read_status()


@pytest.mark.parametrize("T", [1, 6])
def test_moe_of_bad_weights_ends(q8, T):
    """Every NaN is a value like others: also the one of all ones, in a factor, and nobody waits for what is behind it."""
    C, I, E, k = 128, 80, 4, 2
    x = _acts(120, T, C)
    router, wgu, sgu, wd, sd = _experts(121, C, I, E)
    router[:] = 0
    router[1], router[2] = 1e-3 * x.sum(0), 1e-3 * x.sum(0)
    want = q8.q8_moe(x, router, wgu, sgu, wd, sd, E, renormalize=True)
    ones = torch.full((1,), -1, dtype=torch.int32, device="cuda").view(torch.float32)
    bad = sd.clone()
    bad[1, 5], bad[2, 7], bad[3, 127] = ones[0], float("inf"), float("nan")
    y = q8.q8_moe(x, router, wgu, sgu, wd, bad, E)[0]
    gone = torch.zeros(C, dtype=torch.bool, device="cuda")
    gone[[5, 7, 127]] = True
    assert bool((~torch.isfinite(y[:, gone])).all()) and torch.equal(y[:, ~gone], want[0][:, ~gone])
    for value in (ones[0], float("nan"), float("inf")):
        bad = sgu.clone()
        bad[2, 3] = value
        y = q8.q8_moe(x, router, wgu, bad, wd, sd, E)[0]
        assert bool(torch.isnan(y).all())
    q8.q8_read_status()


def test_moe_without_tokens(q8):
    router, *rest = _experts(122, 64, 32, 4)
    y, ids, probs = q8.q8_moe(torch.empty(0, 64, device="cuda"), router, *rest, 2)
    assert y.shape == (0, 64) and ids.shape == (0, 2) and probs.shape == (0, 2)


# ------------------------------------------------------------------------------------------------ as they are used
def test_prepared_layers(q8):
    from paper_1805_08691_b200 import pipeline
    T, C, I, E, k = 5, 200, 72, 6, 2
    x = _acts(100, T, C, dtype=torch.bfloat16)
    w, bias = _acts(101, 130, C, dtype=torch.bfloat16), torch.randn(130, generator=_gen(102), device="cuda")
    layer = pipeline.prepare_linear(w, bias, q8.Q8_F32)
    zr, sr = plain_quantize(w)
    assert np.array_equal(layer.w_q.cpu().numpy(), zr) and np.array_equal(layer.w_scale.cpu().numpy(), sr)
    z, s = q8.q8_quantize_tokens(x)
    check_linear(layer(x), z, s, layer.w_q, layer.w_scale, bias)
    assert torch.equal(layer(z, s), layer(x))
    g = _gen(103)
    router, gate_up, down = (torch.randn(*n, generator=g, device="cuda") for n in ((E, C), (E, 2 * I, C), (E, C, I)))
    experts = pipeline.prepare_experts(router / C ** 0.5, gate_up.half(), down.half(), k, renormalize=False)
    zr, sr = plain_quantize(down.half())
    assert np.array_equal(experts.w_down.cpu().numpy(), zr) and np.array_equal(experts.s_down.cpu().numpy(), sr)
    check_moe(experts(x), plain_moe(x, experts.router, experts.w_gate_up, experts.s_gate_up, experts.w_down, experts.s_down, k, False))


def test_a_layer_of_all_of_them(q8):
    """Projection of the activations, its result through the experts, a projection of codes shared by two products."""
    T, C = 6, 256
    x = _acts(70, T, C, dtype=torch.bfloat16)
    w1, s1 = _codes(71, C, C), torch.full((C,), 1e-4, device="cuda")
    experts = _experts(72, C, 128, 8)
    a = q8.q8_linear(x, w1, s1)
    y, ids, probs = q8.q8_moe(a, *experts, 2)
    z, s = q8.q8_quantize_tokens(y)
    q = q8.q8_linear(z, w1, s1, x_scale=s, out_type=q8.Q8_F32)
    v = q8.q8_linear(z[:, :128], w1[:64, :128], s1[:64], x_scale=s, out_type=q8.Q8_F32)
    za, sa = plain_quantize(x)
    check_linear(a, torch.from_numpy(za).cuda(), torch.from_numpy(sa).cuda(), w1, s1, None)
    check_moe((y, ids, probs), plain_moe(a, *experts, 2, True))
    zr, sr = plain_quantize(y)
    assert np.array_equal(z.cpu().numpy(), zr) and np.array_equal(s.cpu().numpy(), sr)
    check_linear(q, z, s, w1, s1, None)
    check_linear(v, z[:, :128], s, w1[:64, :128], s1[:64], None)
