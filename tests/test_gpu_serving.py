"""Serving operators on the GPU against the definitions in 64 bits: the 8-bit integer product with a scale for each token and
channel, the 4-bit cache and attention over it.

Tolerances are bounds, derived beside each: u(t) = finfo(t).eps / 2 is the half step of a type."""
import math

import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def u(t):
    return torch.finfo(t).eps / 2


@pytest.fixture(scope="module")
def hb():
    from paper_1804_01526_b200 import binding
    yield binding
    assert binding.device_status() == 0


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


# ----------------------------------------------------------------------------- 8-bit integers


def int8_reference(x):
    """(q, scale) of rows, in 64 bits on the host."""
    x = x.double().cpu().numpy()
    top = np.abs(x).max(axis=1, initial=0)
    s = (top / 127).astype(np.float32)
    q = np.where(s[:, None] > 0, np.rint(x / np.where(s > 0, s, 1).astype(np.float64)[:, None]), 0)
    return np.clip(q, -127, 127).astype(np.int8), s


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,k", [(1, 1), (3, 7), (5, 16), (2, 129), (33, 1000), (4, 2049), (2, 9001), (1, 70000)])
def test_int8_quantize_rows(hb, dtype, rows, k):
    x = normal(gen(rows + k), rows, k).mul_(3).to(dtype)
    x[0, k // 2] = 0
    r = hb.int8_quantize(x)
    q, s = int8_reference(x)
    assert r.q.shape == (rows, max(16, -(-k // 16) * 16)) and r.k == k
    assert np.array_equal(r.scale.cpu().numpy(), s)
    assert np.array_equal(r.q[:, :k].cpu().numpy(), q)
    assert not r.q[:, k:].any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k,cols", [(1, 1), (7, 3), (128, 32), (129, 33), (1000, 65), (300, 200)])
def test_int8_quantize_columns_are_the_rows_of_the_transpose(hb, dtype, k, cols):
    x = normal(gen(k + cols), k, cols + 3).to(dtype)[:, 1:cols + 1]           # rows further apart than they are long, and unaligned
    r, t = hb.int8_quantize(x, 0), hb.int8_quantize(x.t().contiguous(), 1)
    assert torch.equal(r.q, t.q) and torch.equal(r.scale, t.scale) and r.k == k
    q, s = int8_reference(x.t())
    assert np.array_equal(r.q[:, :k].cpu().numpy(), q)


@pytest.mark.parametrize("dtype", DTYPES)
def test_int8_quantize_ties_zero_rows_and_scales_at_the_ends(hb, dtype):
    half = torch.arange(-127, 127, device="cuda").float() + 0.5
    rows = [torch.cat([torch.tensor([127.0], device="cuda"), half]),                                   # scale 1: every value a tie, to even
            torch.zeros(255, device="cuda"),
            torch.cat([torch.tensor([127.0 * 2.0 ** -20], device="cuda"), half * 2.0 ** -20]),
            torch.cat([torch.tensor([3.0], device="cuda"), torch.linspace(-3, 3, 254, device="cuda")])]
    if dtype == torch.float32:
        rows.append(torch.linspace(-1.0e-41, 1.0e-41, 255, device="cuda"))                             # a scale that is no normal number
        rows.append(torch.linspace(-1.0, 1.0, 255, device="cuda") * 3.0e38)
        rows.append(torch.linspace(-2.0e-44, 2.0e-44, 255, device="cuda"))                             # the scale rounds to zero
    x = torch.stack(rows).to(dtype)
    r = hb.int8_quantize(x)
    q, s = int8_reference(x)
    assert np.array_equal(r.scale.cpu().numpy(), s) and np.array_equal(r.q[:, :255].cpu().numpy(), q)
    assert torch.equal(r.q[0, 1:255].int() % 2, torch.zeros(254, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k", [257, 500, 1016, 1023, 1031, 1279, 1280, 4097, 5113, 9001, 10239, 16367, 16377])
@pytest.mark.parametrize("first", [0, 1, 3, 5])
def test_int8_quantize_rows_that_start_anywhere(hb, dtype, k, first):
    """Rows off 16-byte borders by every number of elements, around the lengths that each number of threads holds: the result is that of a copy
    whose rows start on borders; so are tiny rows, whose division takes another way."""
    g = gen(k + first)
    x = normal(g, 9, k + 7).to(dtype)
    x[3] *= 1e-38 if dtype != torch.float16 else 1e-6
    x[4] = 0
    view = x[:, first:first + k]
    place = torch.zeros(9, (k + 15) // 16 * 16, dtype=dtype, device="cuda")
    place[:, :k] = view
    got, want = hb.int8_quantize(view), hb.int8_quantize(place[:, :k])
    assert torch.equal(got.scale, want.scale) and torch.equal(got.q, want.q)
    assert not got.q[:, k:].any()


def test_int8_quantize_views_and_out(hb):
    x = normal(gen(1), 40, 530).bfloat16()
    for v in (x[:, :512], x[:, 1:514], x[::3, 5:6], x[7:8]):
        q, s = int8_reference(v)
        r = hb.int8_quantize(v)
        assert np.array_equal(r.q[:, :v.shape[1]].cpu().numpy(), q) and np.array_equal(r.scale.cpu().numpy(), s)
    out = hb.Int8Rows(torch.full((40, 544), 77, dtype=torch.int8, device="cuda"), torch.empty(40, device="cuda"), 530)
    assert hb.int8_quantize(x, out=out) is out
    assert not out.q[:, 530:].any() and np.array_equal(out.q[:, :530].cpu().numpy(), int8_reference(x)[0])
    assert torch.equal(out.dequantize(), out.q[:, :530].float() * out.scale[:, None])
    empty = hb.int8_quantize(x[:0])
    assert empty.q.shape == (0, 544) and empty.scale.shape == (0,)


def test_int8_rows_with_infinities_and_nan_stay_by_themselves(hb):
    x = normal(gen(2), 4, 64)
    x[1, 3], x[2, 5] = math.inf, math.nan
    w = hb.int8_quantize(normal(gen(3), 24, 64))
    y, clean = hb.int8_gemm(x, w), hb.int8_gemm(x[[0, 3]].contiguous(), w)
    assert torch.equal(y[[0, 3]], clean)
    assert not torch.isfinite(y[1:3]).any()


def check_product(hb, x, w, bias, y):
    """The sum is exact; converting it, scaling by the token and scaling by the channel with the bias added are a rounding to FP32 each, the
    result's type one more (binary16 may be subnormal: half its smallest step)."""
    qa, sa = int8_reference(x)
    acc = torch.from_numpy(qa).cuda().double() @ w.q[:, :w.k].double().t()
    prod = acc * torch.from_numpy(sa).cuda().double()[:, None] * w.scale.double()
    ref = prod + (bias.double() if bias is not None else 0)
    tol = 3 * u(torch.float32) * prod.abs() + (u(y.dtype) + 2 * u(torch.float32)) * ref.abs()
    tol += 2.0 ** -25 if y.dtype == torch.float16 else 1e-44
    assert (y.double() - ref).abs().le(tol).all(), ((y.double() - ref).abs() / tol).max()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 64, 256), (1, 1000, 777), (2, 130, 33), (7, 129, 4096), (16, 256, 512), (17, 300, 1000), (33, 128, 2000),
                                   (64, 512, 640), (65, 200, 128), (100, 77, 9000), (128, 128, 128), (129, 257, 515), (300, 1111, 200), (513, 640, 1024),
                                   (2048, 1536, 64), (1, 20000, 48), (20000, 16, 48)])
def test_int8_gemm(hb, dtype, M, N, K):
    g = gen(M * 7 + N * 3 + K)
    x = (normal(g, M, K) * torch.exp(normal(g, M, 1))).to(dtype)
    w = hb.int8_quantize(normal(g, N, K) * torch.exp(normal(g, N, 1)))
    bias = normal(g, N) if (M + N + K) % 2 else None
    y = hb.int8_gemm(x, w, bias=bias)
    assert y.dtype == dtype and y.shape == (M, N)
    check_product(hb, x, w, bias, y)
    again = hb.int8_gemm(hb.int8_quantize(x), w, bias=bias, dtype=dtype)       # converted before: the same numbers
    assert torch.equal(y, again)


def test_int8_gemm_largest_sums_are_exact(hb):
    """K = 131071 of largest magnitude in both operands: the sum is 127 * 127 * K, close to 2^31."""
    K = 131071
    w = hb.Int8Rows(torch.zeros(16, K + 1, dtype=torch.int8, device="cuda"), torch.ones(16, device="cuda"), K)
    w.q[::2, :K], w.q[1::2, :K] = 127, -128
    x = torch.full((9, K), 127.0, device="cuda")
    y = hb.int8_gemm(x, w)
    expect = torch.tensor([127.0 * 127 * K, -127.0 * 128 * K] * 8, dtype=torch.float64, device="cuda").float()
    assert torch.equal(y, expect.expand(9, 16))
    x8 = hb.Int8Rows(torch.full((130, K + 1), -128, dtype=torch.int8, device="cuda"), torch.ones(130, device="cuda"), K)
    y = hb.int8_gemm(x8, w)
    assert torch.equal(y, torch.tensor([-127.0 * 128 * K, 128.0 * 128 * K] * 8, dtype=torch.float64, device="cuda").float().expand(130, 16))


@pytest.mark.parametrize("M", [1, 20, 200])
def test_int8_gemm_views_types_and_what_lies_behind(hb, M):
    g = gen(M)
    K, N = 200, 96
    wide = normal(g, M, K + 9)
    x = wide[:, 3:3 + K]                                                       # unaligned rows of a larger matrix
    w = hb.int8_quantize(normal(g, N, K))
    w.q[:, K:] = 99                                                            # bytes behind the contraction are not read
    bias = normal(g, N)
    full = torch.full((M + 2, N + 7), 42.0, device="cuda")
    out = full[1:M + 1, 2:N + 2]
    assert hb.int8_gemm(x, w, bias=bias, out=out) is out
    check_product(hb, x, w, bias, out)
    rest = full.clone()
    rest[1:M + 1, 2:N + 2] = 42.0
    assert (rest == 42.0).all()
    for t in (torch.bfloat16, torch.float16):
        check_product(hb, x, w, bias, hb.int8_gemm(x, w, bias=bias, dtype=t))
    assert hb.int8_gemm(hb.int8_quantize(x), w).dtype == torch.float32
    rows = hb.Int8Rows(w.q[5:40], w.scale[5:40], K)                            # some of the channels
    assert torch.equal(hb.int8_gemm(x, rows), hb.int8_gemm(x, w)[:, 5:40])


@pytest.mark.parametrize("M,N,K", [(1, 40, 30000), (3, 100, 13000), (3, 24, 14400), (2, 5000, 96), (4, 33, 30000)])
def test_int8_gemm_few_tokens_long_contractions(hb, M, N, K):
    """Tokens that fit the one-launch kernel's shared memory and ones that do not."""
    g = gen(K)
    x, w = normal(g, M, K).bfloat16(), hb.int8_quantize(normal(g, N, K))
    check_product(hb, x, w, None, hb.int8_gemm(x, w))


@pytest.mark.parametrize("M", [2, 9, 200])
def test_int8_gemm_of_part_of_a_larger_matrix(hb, M):
    """Channels and contraction are a window of wider weights, up to its last byte."""
    g = gen(M + 50)
    big = hb.int8_quantize(normal(g, 64, 512))
    w = hb.Int8Rows(big.q[16:, 256:], big.scale[16:], 250)
    x = normal(g, M, 250)
    check_product(hb, x, w, None, hb.int8_gemm(x, w))


def test_int8_runs_in_a_graph_and_on_another_stream(hb):
    g = gen(77)
    for M, N, K in ((1, 256, 512), (20, 300, 500), (2048, 1536, 256)):
        x, w = normal(g, M, K).half(), hb.int8_quantize(normal(g, N, K))
        want = hb.int8_gemm(x, w)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            y = hb.int8_gemm(x, w)
        side.synchronize()
        assert torch.equal(y, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = hb.int8_gemm(x, w)
        x.copy_(normal(g, M, K))
        graph.replay()
        assert torch.equal(y, hb.int8_gemm(x, w))


def test_int8_linear_keeps_its_scales(hb):
    """A module given another type keeps FP32 scales; its product is the function's."""
    from paper_1804_01526_b200.serving import Int8Linear
    g = gen(5)
    layer = Int8Linear(normal(g, 96, 40), normal(g, 40)).half()
    assert layer.weight_scale.dtype == layer.bias.dtype == torch.float32 and layer.weight_q.dtype == torch.int8
    x = normal(g, 2, 3, 96).half()
    y = layer(x)
    assert y.shape == (2, 3, 40) and y.dtype == torch.float16 and not y.requires_grad
    check_product(hb, x.view(6, 96), hb.Int8Rows(layer.weight_q, layer.weight_scale, 96), layer.bias, y.view(6, 40))
    again = Int8Linear(torch.zeros(96, 40, device="cuda"), torch.zeros(40, device="cuda"))
    again.load_state_dict(layer.state_dict())
    assert torch.equal(again(x), y)


def test_int8_linear_takes_any_order(hb):
    """Weights and tokens that are views of other tensors, transposed, broadcast or empty; a wrong extent is refused."""
    from paper_1804_01526_b200.serving import Int8Linear
    g = gen(6)
    w, b = normal(g, 40, 96), normal(g, 40)
    layer = Int8Linear(w.t(), b)
    same = Int8Linear(w.t().contiguous(), b)
    assert torch.equal(layer.weight_q, same.weight_q) and torch.equal(layer.weight_scale, same.weight_scale)
    x = normal(g, 96, 5, 7)
    for view in (x.permute(1, 2, 0), x[:, 0].t(), x[:, 0, 0], x[:, 0, :1].t().expand(4, 96), x.permute(2, 1, 0)[:, ::2], x[:1, 0, 0].expand(2, 96)):
        y = layer(view)
        assert y.shape == (*view.shape[:-1], 40)
        assert torch.equal(y, layer(view.contiguous()))
    assert layer(x.permute(1, 2, 0)[:, :0]).shape == (5, 0, 40)
    for bad in (x.permute(1, 2, 0)[..., :48], normal(g, 4, 192), x[0, 0, 0]):
        with pytest.raises(ValueError):
            layer(bad)
    nothing = Int8Linear(torch.zeros(0, 40, device="cuda"), b)
    assert torch.equal(nothing(torch.zeros(3, 0, device="cuda")), b.expand(3, 40))


def test_int8_gemm_of_nothing(hb):
    w = hb.int8_quantize(normal(gen(0), 8, 32))
    assert hb.int8_gemm(torch.empty(0, 32, device="cuda"), w).shape == (0, 8)
    assert hb.int8_gemm(normal(gen(1), 3, 32), hb.int8_quantize(torch.empty(0, 32, device="cuda"))).shape == (3, 0)
    no_terms = hb.Int8Rows(torch.zeros(8, 16, dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda"), 0)
    bias = normal(gen(2), 8)
    x = torch.empty(3, 0, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(hb.int8_gemm(x, no_terms, bias=bias), bias.bfloat16().expand(3, 8))
    assert not hb.int8_gemm(x, no_terms).any()


def test_int8_refusals(hb):
    x, w = normal(gen(0), 4, 32), hb.int8_quantize(normal(gen(1), 8, 32))
    for bad in (lambda: hb.int8_gemm(x.double(), w), lambda: hb.int8_gemm(x[:, :30], w), lambda: hb.int8_gemm(x.t(), w), lambda: hb.int8_gemm(x, w, bias=x[0, :8].double()),
                lambda: hb.int8_gemm(x, w, bias=x[0, :7]), lambda: hb.int8_gemm(x, w, out=torch.empty(4, 9, device="cuda")),
                lambda: hb.int8_gemm(x, w, out=torch.empty(4, 8)), lambda: hb.int8_gemm(x, hb.Int8Rows(w.q.cpu(), w.scale, 32)),
                lambda: hb.int8_gemm(x, hb.Int8Rows(w.q.float(), w.scale, 32)), lambda: hb.int8_gemm(x, hb.Int8Rows(w.q, w.scale[:7], 32)),
                lambda: hb.int8_gemm(x, hb.Int8Rows(w.q, w.scale, 33)), lambda: hb.int8_quantize(x, 2), lambda: hb.int8_quantize(x.long()),
                lambda: hb.int8_gemm(x, w, out=torch.empty(4, 8, device="cuda"), dtype=torch.float16), lambda: hb.int8_quantize(x[0])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(hb.HbfpError) as e:                                     # a pitch that is no multiple of 16
        hb.int8_gemm(x[:, :20].contiguous(), hb.Int8Rows(torch.zeros(8, 20, dtype=torch.int8, device="cuda"), w.scale, 20))
    assert e.value.code == hb.ERR_ALIGNMENT
    with pytest.raises(hb.HbfpError) as e:
        hb.int8_gemm(torch.zeros(1, 131072, device="cuda"), hb.Int8Rows(torch.zeros(1, 131072, dtype=torch.int8, device="cuda"), w.scale[:1], 131072))
    assert e.value.code == hb.ERR_UNSUPPORTED


# ----------------------------------------------------------------------------- the cache


def unpack(m, e):
    """The values (float64) of the cache's arrays, by the documented layout."""
    words = m.contiguous().view(torch.int32).long()
    place = torch.tensor([4 * (i // 2) + 16 * (i % 2) for i in range(8)], device=m.device)
    q = ((words[..., None] >> place) & 15) - 8
    q = q.flatten(-2).unflatten(-1, (-1, 32))
    return (q.double() * torch.exp2(e.double())[..., None]).flatten(-2)


def pages_of(lengths, page, g, spare=3):
    """A page table for sequences of these lengths, pages in random order, -1 behind each sequence's last page."""
    per = [-(-max(n, 0) // page) for n in lengths]
    order = torch.randperm(sum(per) + spare, generator=g, device="cuda").int()
    table = torch.full((len(lengths), max(max(per), 1)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, c in enumerate(per):
        table[b, :c] = order[at:at + c]
        at += c
    return table, sum(per) + spare


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,D,page", [(1, 64, 16), (3, 96, 32), (2, 128, 64), (2, 256, 16)])
def test_append_is_the_librarys_4_bit_format(hb, dtype, heads, D, page):
    """Mantissas and exponents equal the oracle's conversion with 4 bits and blocks of 32; other rows stay as they were."""
    g = gen(D + heads)
    lengths, n = [n0 + 5 for n0 in (0, 13, 16, 31, 77)], 5
    table, pages = pages_of(lengths, page, g)
    cache = hb.kv4_alloc(pages, heads, page, D)
    for t in (cache.k_mant, cache.k_exps, cache.v_mant, cache.v_exps):
        t.fill_(0x5A)
    x = (normal(g, len(lengths) * n, 2, heads, D) * torch.exp(3 * normal(g, 1, 2, heads, 1))).to(dtype)
    x[2, :, :, :32] = 0                                                        # an all-zero block
    k, v = x[:, 0], x[:, 1]                                                    # rows of a fused tensor
    hb.kv4_append(cache, k, v, table, i32(lengths))
    written = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
    for src, m, e in ((k, cache.k_mant, cache.k_exps), (v, cache.v_mant, cache.v_exps)):
        q, s = oracle.quantize(np.ascontiguousarray(src.float().cpu().numpy().reshape(-1, D)), 1, oracle.Format(mant_bits=4, block=32))
        want = (q.reshape(-1, D // 32, 32) * np.exp2(s.astype(np.float64))[..., None]).reshape(len(lengths), n, heads, D)
        for b, L in enumerate(lengths):
            for i in range(n):
                p = L - n + i
                pg, r = int(table[b, p // page]), p % page
                written[pg, r] = True
                assert np.array_equal(e[pg, :, r].cpu().numpy(), s.reshape(len(lengths), n, heads, D // 32)[b, i])
                assert np.array_equal(unpack(m[pg, :, r], e[pg, :, r]).cpu().numpy(), want[b, i])
        assert (m.transpose(1, 2)[~written] == 0x5A).all() and (e.transpose(1, 2)[~written] == 0x5A).all()
    rk, rv = hb.kv4_read(cache, n, table, i32(lengths))
    assert torch.equal(rv.double().cpu(), torch.from_numpy(want.reshape(-1, heads, D)))


def test_append_largest_values_saturate(hb):
    cache = hb.kv4_alloc(1, 1, 16, 64)
    k = torch.zeros(1, 1, 64, device="cuda")
    k[0, 0, :4] = torch.tensor([3.0e38, 7 * 2.0 ** 120, -3.0e38, 2.0 ** 120], device="cuda")
    k[0, 0, 32:34] = torch.tensor([1e-44, 0.0], device="cuda")
    hb.kv4_append(cache, k, k, i32([[0]]), i32([1]))
    r, _ = hb.kv4_read(cache, 1, i32([[0]]), i32([1]))
    top = 7 * 2.0 ** 120
    assert r[0, 0, :4].tolist() == [top, top, -top, 2.0 ** 120] and not r[0, 0, 4:].any()


def test_append_ragged_starts_padding_and_short_sequences(hb):
    """Sequences of 0, 1, 4 and 2 new tokens, one of them longer than its length (its first rows have no position), two rows behind the last."""
    g = gen(5)
    lengths, starts, page, heads, D = [40, 1, 2, 18], [0, 0, 1, 5, 7], 16, 2, 64
    table, pages = pages_of(lengths, page, g)
    cache = hb.kv4_alloc(pages, heads, page, D)
    for t in (cache.k_mant, cache.k_exps, cache.v_mant, cache.v_exps):
        t.zero_()
    k, v = normal(g, 9, heads, D), normal(g, 9, heads, D)
    hb.kv4_append(cache, k, v, table, i32(lengths), starts=i32(starts))
    back = unpack(cache.k_mant, cache.k_exps).transpose(1, 2)                  # [pages][page][heads][D]
    used = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
    for b, row, p in ((1, 0, 0), (2, 3, 0), (2, 4, 1), (3, 5, 16), (3, 6, 17)):
        pg = int(table[b, p // page])
        used[pg, p % page] = True
        step = torch.exp2(cache.k_exps[pg, :, p % page].double()).repeat_interleave(32, -1)
        # half a step; the largest magnitude of a block lies below 8 steps and is stored as 7 at most
        assert (back[pg, p % page] - k[row].double()).abs().le(step).all()
    assert not (cache.k_mant.transpose(1, 2)[~used]).any()


def test_cache_refusals(hb):
    cache = hb.kv4_alloc(4, 2, 16, 64)
    k, t, n = normal(gen(0), 3, 2, 64), i32([[0, 1], [2, -1], [3, -1]]), i32([3, 4, 5])
    for bad in (lambda: hb.kv4_append(cache, k, k.half(), t, n), lambda: hb.kv4_append(cache, k, k[:2], t, n), lambda: hb.kv4_append(cache, k[:2], k[:2], t, n),
                lambda: hb.kv4_append(cache, k[:, :1], k[:, :1], t, n), lambda: hb.kv4_append(cache, k, k, t.long(), n), lambda: hb.kv4_append(cache, k, k, t, n[:2]),
                lambda: hb.kv4_append(cache, k, k, t, n, max_tokens=1), lambda: hb.kv4_append(cache, k, k, t, n, starts=i32([0, 1, 2])),
                lambda: hb.kv4_append(cache, k.double(), k.double(), t, n), lambda: hb.kv4_append(cache, k, k, t.cpu(), n),
                lambda: hb.kv4_append(cache, k.transpose(1, 2).contiguous().transpose(1, 2), k, t, n),
                lambda: hb.kv4_append(hb.Kv4Cache(cache.k_mant, cache.k_exps, cache.v_mant, cache.k_mant), k, k, t, n),
                lambda: hb.kv4_append(hb.Kv4Cache(cache.k_mant, cache.k_exps[:3], cache.v_mant, cache.v_exps), k, k, t, n),
                lambda: hb.kv4_read(cache, -1, t, n), lambda: hb.kv4_attention(normal(gen(0), 3, 3, 64), cache, t, n), lambda: hb.kv4_attention(k, cache, t, n, window=-1),
                lambda: hb.kv4_attention(k[:, :, :32], cache, t, n), lambda: hb.kv4_attention(k, cache, t, n, out=torch.empty(3, 2, 64, device="cuda").half()),
                lambda: hb.kv4_attention(k, cache, t, n, out=torch.empty(2, 2, 64, device="cuda")), lambda: hb.kv4_attention(k[:2], cache, t, n)):
        with pytest.raises(ValueError):
            bad()


# ----------------------------------------------------------------------------- attention


def fill(hb, g, pages, heads, page, D):
    """A cache with values in every row of every page."""
    cache = hb.kv4_alloc(pages, heads, page, D)
    rows = pages * page
    k = normal(g, rows, heads, D) * torch.exp(normal(g, 1, heads, D) * 0.5)
    hb.kv4_append(cache, k, normal(g, rows, heads, D), torch.arange(pages, dtype=torch.int32, device="cuda")[None], i32([rows]))
    return cache


def attend_reference(q, cache, table, lengths, ns, scale, window=0):
    """(out, bound): the definition in 64 bits and the error that the kernel's arithmetic can leave in FP32.

    With S = scale * sum |q k| of a row's largest score and A = sum p |v|: a score is a sum of D exact products in FP32, sixteen and a part of the
    query at a time (each step no worse than 2^-22 of S) and scaled and reduced by the maximum, a rounding of S each; p's error is the score's, in
    numerator and denominator, and 2^-21 of the exponentials; p is rounded to the parts its type has (u(bfloat16) to that power); the sum over the keys
    is again FP32, sixteen at a time."""
    D, page = q.shape[2], cache.k_mant.shape[2]
    heads = cache.k_mant.shape[1]
    G = q.shape[1] // heads
    parts = {torch.bfloat16: 1, torch.float16: 2, torch.float32: 3}[q.dtype]
    out, tol = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    row = 0
    K, V = unpack(cache.k_mant, cache.k_exps), unpack(cache.v_mant, cache.v_exps)
    for b, L in enumerate(lengths):
        n = ns[b]
        pos = torch.arange(L, device="cuda")
        ids = table[b].long()[pos // page]
        i = torch.arange(L - n, L, device="cuda")[:, None]
        seen = (pos[None] <= i) & (i >= 0)
        if window:
            seen &= pos[None] > i - window
        for h in range(heads):
            k, v = K[ids, h, pos % page], V[ids, h, pos % page]
            for hq in range(h * G, h * G + G):
                x = q[row:row + n, hq].double()
                s = (x @ k.t() * scale).masked_fill(~seen, -math.inf)
                top = s.max(-1, keepdim=True).values if L else torch.zeros(n, 1, dtype=torch.float64, device="cuda")
                p = torch.exp(s - torch.where(top.isfinite(), top, 0.0))
                total = p.sum(-1, keepdim=True)
                p = torch.where(total > 0, p / total, 0.0)
                out[row:row + n, hq] = p @ v
                if L:
                    S = (x.abs() @ k.abs().t() * abs(scale)).masked_fill(~seen, 0.0).max(-1, keepdim=True).values
                    A = p @ v.abs()
                    err = 2 * S * ((parts * D / 16 + 8) * 2.0 ** -22) + 2.0 ** -20 + (L / 16 + 8) * 2.0 ** -22 + u(torch.bfloat16) ** parts
                    tol[row:row + n, hq] = A * err
        row += n
    return out, tol + u(q.dtype) * out.abs() + (2.0 ** -25 if q.dtype == torch.float16 else 1e-40)


def check_attention(hb, dtype, heads, group, D, page, lengths, ns, window=0, scale=None, ragged=False, seed=0):
    g = gen(seed + D + page + sum(lengths))
    table, pages = pages_of(lengths, page, g)
    cache = fill(hb, g, pages, heads, page, D)
    q = normal(g, sum(ns), heads * group, D).to(dtype)
    kw = {}
    if ragged:
        kw["starts"] = i32([0] + list(np.cumsum(ns)))
        kw["max_tokens"] = max(ns)
    y = hb.kv4_attention(q, cache, table, i32(lengths), scale=scale, window=window, **kw)
    ref, tol = attend_reference(q, cache, table, lengths, ns, scale if scale is not None else D ** -0.5, window)
    assert y.dtype == dtype and y.shape == q.shape
    assert (y.double() - ref).abs().le(tol).all(), ((y.double() - ref).abs() / tol).max()
    return q, cache, table, y


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,page", [(64, 16), (96, 32), (128, 64), (256, 16)])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 3), (1, 8), (2, 12)])
def test_attention_one_token(hb, dtype, D, page, heads, group):
    check_attention(hb, dtype, heads, group, D, page, [1, 2, 15, 16, 17, 33, 128, 129, 300, 0], [1] * 10)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_attention_long_keys_are_split(hb, dtype, D):
    """Sequences whose keys several CTAs share, next to short and empty ones."""
    check_attention(hb, dtype, 2, 4, D, 64, [5000, 1, 0, 2049, 640, 31], [1] * 6)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,group,n", [(64, 1, 5), (96, 3, 5), (128, 4, 3), (128, 1, 40), (256, 2, 7), (256, 2, 40), (64, 7, 20)])
def test_attention_several_queries(hb, dtype, D, group, n):
    check_attention(hb, dtype, 2, group, D, 32, [n, n + 1, n + 15, 700], [n] * 4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [1, 2, 16, 100, 257])
@pytest.mark.parametrize("n", [1, 6, 33])
def test_attention_window(hb, dtype, window, n):
    check_attention(hb, dtype, 2, 2, 128, 16, [n, 64 + n, 300 + n, 1000], [n] * 4, window=window)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,heads,group,n", [(64, 1, 1, 128), (64, 2, 1, 300), (128, 1, 4, 64), (128, 2, 3, 100), (128, 1, 12, 33), (64, 1, 5, 257)])
@pytest.mark.parametrize("window", [0, 1, 100])
def test_attention_prompts(hb, dtype, D, heads, group, n, window):
    """Rows enough for the kernel of many rows: prompts behind prefixes of no, few and many keys, and ones longer than their length."""
    check_attention(hb, dtype, heads, group, D, 32, [n, n + 1, n + 63, n + 500, n - 7], [n] * 5, window=window)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [0.0, 3.0, -2.0, 1e-3])
def test_attention_prompts_scales(hb, dtype, scale):
    check_attention(hb, dtype, 1, 2, 64, 16, [500, 130], [130, 130], scale=scale)


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_prompts_ragged(hb, dtype):
    """Prompts of 0 to 200 tokens in one call, queries and results slices of larger tensors, an invalid page among one sequence's."""
    lengths, ns, D = [220, 7, 100, 2, 400, 0], [200, 0, 90, 5, 140, 2], 128
    g = gen(19)
    table, pages = pages_of(lengths, 16, g)
    cache = fill(hb, g, pages, 2, 16, D)
    rows = sum(ns)
    q = normal(g, rows + 4, 9, D + 3).to(dtype)[:, 1:7, 2:D + 2]
    big = torch.full((rows + 4, 8, D), 9.0, dtype=dtype, device="cuda")
    out = big[:, 1:7]
    starts = i32([0] + list(np.cumsum(ns)))
    hb.kv4_attention(q, cache, table, i32(lengths), starts=starts, max_tokens=200, out=out)
    ref, tol = attend_reference(q[:rows], cache, table, lengths, ns, D ** -0.5)
    assert (out[:rows].double() - ref).abs().le(tol).all()
    assert (out[rows:] == 9.0).all() and (big[:, 0] == 9.0).all() and (big[:, 7] == 9.0).all()
    good = out.clone()
    assert torch.equal(hb.kv4_attention(q, cache, table, i32(lengths), starts=starts, max_tokens=200)[:rows], good[:rows])
    bad = table.clone()
    bad[4, 3] = pages + 7                                                      # sixteen keys of the fifth sequence
    assert hb.device_status() == 0
    y = hb.kv4_attention(q, cache, bad, i32(lengths), starts=starts, max_tokens=200)
    assert hb.device_status_rc() == (hb.ERR_INDEX, 1001)
    assert torch.equal(y[:295], good[:295]) and torch.isfinite(y[:rows]).all() and not torch.equal(y[295:435], good[295:435])
    free = list(range(48)) + list(range(64, 400))                              # the same as a sequence without those keys, for its last query
    K, V = unpack(cache.k_mant, cache.k_exps), unpack(cache.v_mant, cache.v_exps)
    at = torch.tensor(free, device="cuda")
    ids = table[4].long()[at // 16]
    k, v = K[ids, 0, at % 16], V[ids, 0, at % 16]
    p = torch.softmax(q[434, 0].double() @ k.t() * D ** -0.5, -1)
    assert (y[434, 0].double() - p @ v).abs().le(2 * tol[434, 0] + 1e-5).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_ragged_tokens(hb, dtype):
    """Sequences of 0 to 50 new tokens, rows behind the last sequence's left as they were, first rows without a position."""
    lengths, ns = [30, 7, 100, 2, 400, 0], [3, 0, 50, 5, 1, 2]
    g = gen(9)
    table, pages = pages_of(lengths, 16, g)
    cache = fill(hb, g, pages, 2, 16, 64)
    rows = sum(ns)
    q = normal(g, rows + 4, 6, 64).to(dtype)
    out = torch.full_like(q, 9.0)
    hb.kv4_attention(q, cache, table, i32(lengths), starts=i32([0] + list(np.cumsum(ns))), max_tokens=50, out=out)
    ref, tol = attend_reference(q[:rows], cache, table, lengths, ns, 0.125)
    assert (out[:rows].double() - ref).abs().le(tol).all()
    assert (out[rows:] == 9.0).all()
    assert not out[53:56].any()                                                # three rows of five at negative positions: they see nothing
    assert not out[rows - 2:rows].any()                                        # an empty sequence's
    again = hb.kv4_attention(q, cache, table, i32(lengths), starts=i32([0] + list(np.cumsum(ns))))
    assert torch.equal(again[:rows], out[:rows])


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_strides(hb, dtype):
    """Queries are a slice of a fused projection, the output a slice of a larger tensor."""
    g = gen(3)
    lengths = [200, 17, 64]
    table, pages = pages_of(lengths, 32, g)
    cache = fill(hb, g, pages, 2, 32, 128)
    fused = normal(g, 3, 8 + 4, 128 + 1).to(dtype)
    q = fused[:, 1:9, 1:]
    big = torch.full((3, 10, 200), 5.0, dtype=dtype, device="cuda")
    out = big[:, 1:9, 3:131]
    hb.kv4_attention(q, cache, table, i32(lengths), out=out)
    ref, tol = attend_reference(q, cache, table, lengths, [1] * 3, 128 ** -0.5)
    assert (out.double() - ref).abs().le(tol).all()
    big[:, 1:9, 3:131] = 5.0
    assert (big == 5.0).all()


def test_attention_scores_far_apart_and_one_key_taking_all(hb):
    """Scores over hundreds: all weight on one key, the others underflow; the maximum moves often."""
    for scale in (0.0, 3.0, -2.0, 1e-3):
        check_attention(hb, torch.float32, 1, 2, 64, 16, [900, 5], [1, 1], scale=scale)


@pytest.mark.parametrize("D", [64, 128])
def test_attention_ignores_what_no_row_sees(hb, D):
    """Rows of the last page behind the length, never written: any bytes there, the same result."""
    g = gen(4)
    lengths = [37, 1, 70]
    table, pages = pages_of(lengths, 32, g, spare=0)
    cache = fill(hb, g, pages, 1, 32, D)
    q = normal(g, 3, 4, D)
    y = hb.kv4_attention(q, cache, table, i32(lengths))
    for b, L in enumerate(lengths):
        if L % 32:
            pg = int(table[b, L // 32])
            for t in (cache.k_mant, cache.v_mant):
                t[pg, :, L % 32:] = 0xFF
            for t in (cache.k_exps, cache.v_exps):
                t[pg, :, L % 32:] = 127
    assert torch.equal(hb.kv4_attention(q, cache, table, i32(lengths)), y)


@pytest.mark.parametrize("lengths", [[5000, 3, 700], [90, 17, 64]])
def test_attention_repeats_itself_and_runs_in_a_graph(hb, lengths):
    """The same bits every time, on another stream, and from a graph replayed after lengths, queries and cache have changed in place."""
    g = gen(8)
    table, pages = pages_of([max(lengths)] * 3, 64, g)
    cache = fill(hb, g, pages, 2, 64, 128)
    q, n = normal(g, 3, 8, 128).bfloat16(), i32(lengths)
    y = hb.kv4_attention(q, cache, table, n)
    for _ in range(3):
        assert torch.equal(hb.kv4_attention(q, cache, table, n), y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = hb.kv4_attention(q, cache, table, n)
    side.synchronize()
    assert torch.equal(z, y)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(q)
    k = normal(g, 3, 2, 128).bfloat16()
    with torch.cuda.graph(graph):
        hb.kv4_append(cache, k, k, table, n)
        hb.kv4_attention(q, cache, table, n, out=out)
    for step in (1, 2):
        n.sub_(1).clamp_(min=0)
        q.copy_(normal(g, 3, 8, 128))
        k.copy_(normal(g, 3, 2, 128))
        graph.replay()
        ref, tol = attend_reference(q, cache, table, n.tolist(), [1] * 3, 128 ** -0.5)
        assert (out.double() - ref).abs().le(tol).all()


def test_two_graphs_keep_their_own_workspaces(hb):
    """Two captured calls of different sizes replayed in turn and at the same time: each has the result it had alone."""
    g = gen(12)
    calls = []
    for lengths, heads in (([3000, 100], 2), ([9000], 4)):
        table, pages = pages_of(lengths, 64, g)
        calls.append((normal(g, len(lengths), heads * 4, 128).half(), fill(hb, g, pages, heads, 64, 128), table, i32(lengths)))
    want = [hb.kv4_attention(*c) for c in calls]
    graphs, outs = [], []
    for c in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(hb.kv4_attention(*c))
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for s, gr in zip(streams, graphs):
            with torch.cuda.stream(s):
                gr.replay()
                gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_pages_and_lengths_out_of_range_are_left_out_and_reported(hb):
    """Numbers in device memory cannot be refused by the call: keys of a page that is none are not seen, and the status says so."""
    g = gen(6)
    lengths = [60, 33]
    table, pages = pages_of(lengths, 16, g, spare=0)
    cache = fill(hb, g, pages, 1, 16, 64)
    q = normal(g, 2, 2, 64)
    good = hb.kv4_attention(q, cache, table, i32(lengths))
    assert hb.device_status() == 0
    bad = table.clone()
    bad[0, 1] = pages
    y = hb.kv4_attention(q, cache, bad, i32(lengths))
    assert hb.device_status_rc() == (hb.ERR_INDEX, 1001)
    assert torch.equal(y[1], good[1]) and torch.isfinite(y).all()
    hb.kv4_append(cache, q[:, :1], q[:, :1], i32([[-5], [10 ** 6]]), i32([1, 1]))            # nothing is written
    assert hb.device_status_rc() == (hb.ERR_INDEX, 1001)
    assert torch.equal(hb.kv4_attention(q, cache, table, i32(lengths)), good)
    hb.kv4_attention(q, cache, table, i32([60, 1000]))                                       # longer than the table
    assert hb.device_status_rc() == (hb.ERR_INDEX, 1002)
    y = hb.kv4_attention(q, cache, table, i32(lengths), starts=i32([0, 5, 1]), out=torch.full_like(q, 3.0))
    assert hb.device_status_rc() == (hb.ERR_INDEX, 1002)
    assert (y == 3.0).all()
    assert hb.device_status_rc() == (hb.OK, 0)


def test_offsets_beyond_32_bits(hb):
    """A cache whose arrays pass 2^32 bytes: pages at its end are written, read and attended."""
    pages, heads, page, D = 40000, 8, 256, 128                                 # 5.2 GB of mantissas each
    free, _ = torch.cuda.mem_get_info()
    if free < 16 << 30:
        pytest.skip("not enough device memory")
    cache = hb.kv4_alloc(pages, heads, page, D)
    g = gen(7)
    table, n = i32([[pages - 1, 0], [pages - 2, 39000]]), [300, 290]
    k, v = normal(g, 600, heads, D), normal(g, 600, heads, D)
    hb.kv4_append(cache, k, v, table, i32(n), starts=i32([0, 300, 590]), max_tokens=300)
    rk, rv = hb.kv4_read(cache, 290, table, i32(n))
    for x, r in ((k, rk), (v, rv)):
        want = torch.cat([x[10:300], x[300:590]])
        assert ((r - want).abs() <= want.unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True).div(4).expand(-1, -1, -1, 32).flatten(-2)).all()
    q = normal(g, 2, heads * 2, D)
    small = hb.Kv4Cache(*(t[[pages - 1, 0, pages - 2, 39000]].contiguous() for t in (cache.k_mant, cache.k_exps, cache.v_mant, cache.v_exps)))
    y, z = hb.kv4_attention(q, cache, table, i32(n)), hb.kv4_attention(q, small, i32([[0, 1], [2, 3]]), i32(n))
    assert torch.equal(y, z)


# ----------------------------------------------------------------------------- together


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_served_attention_layer(hb, dtype):
    """Prompt and three decode steps of an attention layer whose projections were trained in block floating point: product, write,
    attention, product, with ragged prompts. Each step against the definition on that step's own inputs."""
    from paper_1804_01526_b200.autograd import HbfpLinear
    from paper_1804_01526_b200.serving import Int8Linear
    torch.manual_seed(0)
    width, heads, group, D, page = 256, 2, 2, 64, 16
    qkv = Int8Linear.from_hbfp(HbfpLinear(width, (heads * group + 2 * heads) * D, tile=32))
    proj = Int8Linear.from_hbfp(HbfpLinear(heads * group * D, width, tile=32, bias=False))
    g = gen(1)
    ns = [20, 1, 33]
    table, pages = pages_of([n + 3 for n in ns], page, g)
    cache = hb.kv4_alloc(pages, heads, page, D)
    lengths, starts = list(ns), [0, 20, 21, 54]
    for step in range(4):
        rows = sum(ns)
        x = normal(g, rows, width).to(dtype)
        y = qkv(x)
        check_product(hb, x, hb.Int8Rows(qkv.weight_q, qkv.weight_scale, width), qkv.bias, y)
        y = y.view(rows, -1, D)
        q, k, v = y[:, :heads * group], y[:, heads * group:heads * group + heads], y[:, heads * group + heads:]
        kw = dict(starts=i32(starts), max_tokens=max(ns)) if step == 0 else {}
        hb.kv4_append(cache, k, v, table, i32(lengths), **kw)
        o = hb.kv4_attention(q, cache, table, i32(lengths), **kw)
        ref, tol = attend_reference(q, cache, table, lengths, ns, D ** -0.5)
        assert (o.double() - ref).abs().le(tol).all()
        z = proj(o.flatten(1))
        assert z.shape == (rows, width)
        check_product(hb, o.flatten(1), hb.Int8Rows(proj.weight_q, proj.weight_scale, heads * group * D), None, z)
        ns = [1, 1, 1]
        lengths = [n + 1 for n in lengths]
    assert proj(o.view(3, 1, -1)).shape == (3, 1, width)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,heads,group,n", [(128, 1, 1, 128), (64, 2, 4, 100), (128, 2, 2, 200)])
@pytest.mark.parametrize("window", [0, 2500])
@pytest.mark.parametrize("longest", [9001, 7001])
def test_attention_prompts_share_long_keys(hb, dtype, D, heads, group, n, window, longest):
    """Few tiles of many rows: CTAs share a tile's keys, also where a sequence has keys for one of them only, or none."""
    lengths = [longest, 130, n, 0, 2048 + n]
    q, cache, table, y = check_attention(hb, dtype, heads, group, D, 64, lengths, [n, 3, n, 1, n], window=window, ragged=True)
    again = hb.kv4_attention(q, cache, table, i32(lengths), window=window, starts=i32(np.cumsum([0, n, 3, n, 1, n]).tolist()), max_tokens=n)
    assert torch.equal(again, y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,heads,group,n", [(64, 2, 1, 33), (128, 1, 3, 11), (128, 2, 5, 13), (64, 1, 16, 7)])
def test_attention_rows_between_few_and_many(hb, dtype, D, heads, group, n):
    check_attention(hb, dtype, heads, group, D, 16, [n, 400, 1, 1500], [n] * 4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
def test_attention_many_rows_of_one_head_behind_long_keys(hb, dtype, D):
    """Tiles of many rows that a cluster each would not fill the GPU with."""
    check_attention(hb, dtype, 1, 2, D, 64, [20000], [70])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lengths,n", [([40, 700], 2), ([9000, 5], 2), ([300, 200], 130), ([9000, 200], 130)])
def test_attention_a_query_that_is_no_number_stays_by_itself(hb, dtype, lengths, n):
    g = gen(3)
    table, pages = pages_of(lengths, 64, g)
    cache = fill(hb, g, pages, 1, 64, 128)
    q = normal(g, 2 * n, 2, 128).to(dtype)
    y = hb.kv4_attention(q, cache, table, i32(lengths))
    q[1, 1, 5], q[n, 0] = math.nan, math.nan
    z = hb.kv4_attention(q, cache, table, i32(lengths))
    assert z[1, 1].isnan().all()
    if lengths[1] >= n:
        assert z[n, 0].isnan().all()
    y[1, 1], y[n, 0], z[1, 1], z[n, 0] = 0, 0, 0, 0
    assert torch.equal(y, z)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,page,heads,group,n", [(96, 16, 1, 1, 130), (96, 64, 2, 3, 45), (256, 16, 1, 2, 70), (256, 64, 2, 1, 200), (256, 32, 1, 17, 1)])
@pytest.mark.parametrize("window", [0, 1, 100])
def test_attention_prompts_of_other_widths(hb, dtype, D, page, heads, group, n, window):
    check_attention(hb, dtype, heads, group, D, page, [n, n + 1, n + 63, n + 500, n - 7 if n > 7 else 0], [n] * 5, window=window)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [96, 256])
@pytest.mark.parametrize("longest", [3000, 9001])
def test_attention_prompts_of_other_widths_share_long_keys(hb, dtype, D, longest):
    n = 300
    check_attention(hb, dtype, 2, 1, D, 64, [longest, 130, n, 0, 2048 + n], [n, 3, n, 1, n], window=0, ragged=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_attention_prompts_strides_and_places(hb, dtype, D):
    """Queries and results that are slices of wider rows, an element past a multiple of sixteen bytes."""
    g = gen(D)
    lengths, n = [190, 400], 90
    table, pages = pages_of(lengths, 16, g)
    cache = fill(hb, g, pages, 2, 16, D)
    q = normal(g, 2 * n, 4, D).to(dtype)
    y = hb.kv4_attention(q, cache, table, i32(lengths))
    wide = torch.full((2 * n * 5 * D + 1,), 7.0, dtype=dtype, device="cuda")
    out = wide[1:].view(2 * n, 5, D)[:, :4]
    src = torch.empty(2 * n * 4 * (D + 3) + 1, dtype=dtype, device="cuda")[1:].view(2 * n, 4, D + 3)[:, :, :D]
    src.copy_(q)
    assert hb.kv4_attention(src, cache, table, i32(lengths), out=out) is out
    assert torch.equal(out, y) and (wide[1:].view(2 * n, 5, D)[:, 4] == 7).all() and wide[0] == 7
    with pytest.raises(ValueError):
        hb.kv4_attention(q, cache, table, i32(lengths), out=torch.empty(1, 4, D, dtype=dtype, device="cuda").expand(2 * n, 4, D))


@pytest.mark.parametrize("dtype", DTYPES)
def test_int8_linear_under_a_trace_forward_mode_and_transforms(hb, dtype):
    """A trace records the layer and replays it on other tokens, and other numbers of them; what has no derivative of a kind says so."""
    import torch.autograd.forward_ad as fwad
    from paper_1804_01526_b200.serving import Int8Linear
    g = gen(21)
    layer = Int8Linear(normal(g, 96, 40), normal(g, 40))
    x = normal(g, 2, 5, 96).to(dtype)
    traced = torch.jit.trace(layer, (x,), check_trace=False)
    for other in (x, normal(g, 2, 5, 96).to(dtype), normal(g, 7, 1, 96).to(dtype).requires_grad_(True), normal(g, 3, 2, 192).to(dtype)[..., ::2]):
        want = layer(other)
        got = traced(other)
        assert torch.equal(got, want) and got.dtype == dtype and not got.requires_grad
    with fwad.dual_level(), pytest.raises(NotImplementedError):
        layer(fwad.make_dual(x, torch.ones_like(x)))
    for transform in (lambda: torch.func.jvp(layer, (x,), (x,)), lambda: torch.func.grad(lambda v: layer(v).float().sum())(x), lambda: torch.func.vmap(layer)(x[None])):
        with pytest.raises(RuntimeError, match="functorch transforms"):
            transform()
    assert torch.equal(layer(x), traced(x))


def test_serving_calls_refuse_a_trace_and_tangents(hb):
    """A trace of the calls by themselves would replay results that nothing fills."""
    import torch.autograd.forward_ad as fwad
    g = gen(22)
    table, n = i32([[0, 1]]), i32([20])
    cache, w = fill(hb, g, 2, 1, 16, 64), hb.int8_quantize(normal(g, 8, 64))
    k = normal(g, 1, 1, 64)
    before = [t.clone() for t in (cache.k_mant, cache.k_exps, cache.v_mant, cache.v_exps)]

    def append(x):
        hb.kv4_append(cache, x, x, table, n)
        return x

    calls = [lambda x: hb.int8_quantize(x[0]).q, lambda x: hb.int8_gemm(x[0], w), append, lambda x: hb.kv4_attention(x, cache, table, n)]
    for call in calls + [lambda x: hb.kv4_read(cache, 1, table, n)]:
        with pytest.raises(RuntimeError, match="trace"):
            torch.jit.trace(call, (k,), check_trace=False)
    for call in calls:
        with fwad.dual_level(), pytest.raises(RuntimeError, match="derivatives"):
            call(fwad.make_dual(k, torch.ones_like(k)))
    assert all(torch.equal(a, b) for a, b in zip(before, (cache.k_mant, cache.k_exps, cache.v_mant, cache.v_exps)))
    assert hb.kv4_attention(k.requires_grad_(True), cache, table, n).isfinite().all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,first", [(2, 300, 0), (3, 4096, 0), (3, 523, 1), (40, 300, 0), (5, 9001, 3), (200, 77, 0), (2100, 1024, 0)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_int8_rows_that_hold_no_finite_number_are_nan(hb, dtype, M, K, first, bad):
    """Whatever the sign, the place and the kernel: q is 0 there, the row's scale is the infinity or NaN, and 0 times it is NaN in every result."""
    g = gen(K + M)
    x = normal(g, M, K + 8).to(dtype)[:, first:first + K]
    rows = sorted({0, 1, M - 1})
    for i, r in enumerate(rows):
        x[r, (K - 1) * i // max(len(rows) - 1, 1)] = bad
    w = hb.int8_quantize(normal(g, 3000 if M > 1000 else 24, K))
    q = hb.int8_quantize(x)
    assert not q.q[rows].any() and not q.scale[rows].isfinite().any()
    for y in (hb.int8_gemm(x, w), hb.int8_gemm(q, w, dtype=dtype)):
        assert y[rows].isnan().all()
        clean = torch.ones(M, dtype=torch.bool, device="cuda")
        clean[rows] = False
        assert y[clean].isfinite().all()


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_int8_channels_that_hold_no_finite_number_are_nan(hb, bad):
    g = gen(31)
    w = normal(g, 300, 70)
    w[17, 3] = bad
    q = hb.int8_quantize(w, 0)
    assert not q.q[3].any() and not q.scale[3].isfinite()
    y = hb.int8_gemm(normal(g, 5, 300), q)
    assert y[:, 3].isnan().all() and y.isnan().sum() == 5


def test_int8_gemm_columns_past_two_gigabytes_of_a_row(hb):
    """A row of results longer than 2^31 bytes: the columns behind are those of the same channels by themselves."""
    N, K, M = (1 << 29) + 100, 16, 5
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 28 << 30:
        pytest.skip("not enough device memory")
    g = gen(41)
    w = hb.Int8Rows(torch.zeros(N, K, dtype=torch.int8, device="cuda"), torch.ones(N, device="cuda"), K)
    parts = [slice(0, 300), slice((1 << 29) - 130, (1 << 29) + 10), slice(N - 77, N)]
    for p in parts:
        w.q[p] = torch.randint(-127, 128, (p.stop - p.start, K), dtype=torch.int8, device="cuda", generator=g)
        w.scale[p] = normal(g, p.stop - p.start).abs()
    x = normal(g, M, K)
    y = hb.int8_gemm(x, w)
    for p in parts:
        some = hb.Int8Rows(w.q[p].contiguous(), w.scale[p].contiguous(), K)
        check_product(hb, x, some, None, y[:, p])
        assert torch.equal(y[:, p], hb.int8_gemm(x, some))
        y[:, p] = 0
    assert all(not y[:, i:i + (1 << 27)].any() for i in range(0, N, 1 << 27))
    del w, x, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-42])
def test_attention_scales_near_zero_and_keys_of_the_largest_size(hb, dtype, rows, scale):
    """Scores of 1e37 times nothing, or times next to nothing (1e-5), weigh all keys alike: the average of the values, to FP32's accuracy for the
    sums and the type's for probabilities and result, whatever the number of rows."""
    g = gen(51)
    cache, n = hb.kv4_alloc(2, 1, 16, 64), 32
    k, v = torch.zeros(n, 1, 64, device="cuda"), normal(g, n, 1, 64)
    k[::3, 0, 5] = 2.0 ** 120
    table, lengths = i32([[0, 1]]), i32([n])
    hb.kv4_append(cache, k, v, table, lengths)
    q = torch.full((rows, 1, 64), 10.0, device="cuda", dtype=dtype)
    y = hb.kv4_attention(q, cache, table, lengths, scale=scale)
    V = unpack(cache.v_mant, cache.v_exps).transpose(1, 2).flatten(0, 1)[:, 0]
    for i in range(max(0, rows - n), rows):
        seen = V[:n - rows + i + 1]
        assert (y[i, 0].double() - seen.mean(0)).abs().le(3e-5 * seen.abs().mean(0) + 2 * u(dtype) * seen.abs().mean(0) + 1e-30).all()


def test_a_cache_without_heads_is_refused(hb):
    """(The query heads are counted in heads of the cache.)"""
    cache = hb.Kv4Cache(*(torch.empty(2, 0, 16, w, dtype=t, device="cuda") for w, t in ((32, torch.uint8), (2, torch.int8)) * 2))
    table, n = i32([[0, 1]]), i32([3])
    for call in (lambda: hb.kv4_attention(normal(gen(0), 1, 2, 64), cache, table, n), lambda: hb.kv4_read(cache, 1, table, n),
                 lambda: hb.kv4_append(cache, torch.empty(1, 0, 64, device="cuda"), torch.empty(1, 0, 64, device="cuda"), table, n)):
        with pytest.raises(ValueError, match="extents"):
            call()


@pytest.mark.parametrize("length,n", [(50, 5), (48 + 70, 70), (49, 49), (200, 3)])
def test_positions_behind_the_page_table_are_left_out(hb, length, n):
    """A sequence longer than its table of 48: new tokens that have a place go there, the rest nowhere, and nothing else is touched. The other
    sequence is written as ever."""
    g = gen(length)
    cache = fill(hb, g, 5, 2, 16, 64)
    arrays = (cache.k_mant, cache.k_exps, cache.v_mant, cache.v_exps)
    old = [t.clone() for t in arrays]
    k, v = normal(g, n + 1, 2, 64), normal(g, n + 1, 2, 64)
    table, starts = i32([[3, 0, 4], [1, -1, -1]]), i32([0, n, n + 1])
    hb.kv4_append(cache, k, v, table, i32([length, 7]), starts=starts)
    assert hb.device_status_rc() == (hb.ERR_INDEX, 1002)
    want = hb.Kv4Cache(*(t.clone() for t in old))
    there = max(0, min(n, 48 - (length - n)))
    if there:
        hb.kv4_append(want, k[:there], v[:there], table[:1], i32([length - n + there]))
    hb.kv4_append(want, k[n:], v[n:], table[1:], i32([7]))
    assert hb.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(arrays, (want.k_mant, want.k_exps, want.v_mant, want.v_exps)))
    rk, rv = hb.kv4_read(cache, n, table[:1], i32([length]))
    assert hb.device_status_rc() == (hb.ERR_INDEX, 1002)
    assert not rk[there:].any() and not rv[there:].any()
    if there:
        ek, ev = hb.kv4_read(cache, there, table[:1], i32([length - n + there]))
        assert torch.equal(rk[:there], ek) and torch.equal(rv[:there], ev)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("pages,length,n", [(3, 50, 5), (3, 48 + 70, 70), (3, 49, 1), (300, 4990, 1), (300, 4990, 200), (5, 81, 40), (3, 4000, 2)])
@pytest.mark.parametrize("window", [0, 30])
def test_attention_behind_the_page_table(hb, dtype, D, pages, length, n, window):
    """Rows of a sequence longer than its table see what the table holds of the keys up to their own positions: the definition in 64 bits, and the
    bound of attend_reference with that many keys."""
    g = gen(length + n + D)
    cap = 16 * pages
    cache = fill(hb, g, pages, 1, 16, D)
    table = torch.randperm(pages, generator=g, device="cuda").int()[None]
    q = normal(g, n, 2, D).to(dtype)
    y = hb.kv4_attention(q, cache, table, i32([length]), window=window)
    assert hb.device_status_rc() == (hb.ERR_INDEX, 1002)
    K, V = (unpack(m, e)[table[0].long()].transpose(0, 1).flatten(1, 2)[0] for m, e in ((cache.k_mant, cache.k_exps), (cache.v_mant, cache.v_exps)))
    i, j = torch.arange(length - n, length, device="cuda")[:, None], torch.arange(cap, device="cuda")[None]
    seen = (j <= i) & (j > i - window if window else j >= 0)
    parts = {torch.bfloat16: 1, torch.float16: 2, torch.float32: 3}[dtype]
    for h in range(2):
        x = q[:, h].double()
        s = (x @ K.t() * D ** -0.5).masked_fill(~seen, -math.inf)
        p = torch.where(seen.any(-1, keepdim=True), torch.softmax(s, -1), 0.0)
        ref = p @ V
        S = (x.abs() @ K.abs().t() * D ** -0.5).masked_fill(~seen, 0.0).max(-1, keepdim=True).values
        err = 2 * S * ((parts * D / 16 + 8) * 2.0 ** -22) + 2.0 ** -20 + (cap / 16 + 8) * 2.0 ** -22 + u(torch.bfloat16) ** parts
        tol = (p @ V.abs()) * err + u(dtype) * ref.abs() + (2.0 ** -25 if dtype == torch.float16 else 1e-40)
        assert (y[:, h].double() - ref).abs().le(tol).all(), ((y[:, h].double() - ref).abs() / tol).max()


def test_sequences_of_more_tokens_than_positions_have_bits_are_empty(hb):
    g = gen(61)
    cache = fill(hb, g, 3, 1, 16, 64)
    arrays = (cache.k_mant, cache.k_exps, cache.v_mant, cache.v_exps)
    old = [t.clone() for t in arrays]
    table, k = i32([[0, 1, 2]] * 2), normal(g, 2, 1, 64)
    good = hb.kv4_attention(k, cache, table, i32([20, 40]))
    for length in (1 << 30, 2 ** 31 - 1):
        hb.kv4_append(cache, k[:1], k[:1], table[:1], i32([length]))
        assert hb.device_status_rc() == (hb.ERR_INDEX, 1002)
        y = hb.kv4_attention(k, cache, table, i32([length, 40]), out=torch.full_like(k, 3.0))
        assert hb.device_status_rc() == (hb.ERR_INDEX, 1002)
        assert not y[0].any() and torch.equal(y[1], good[1])
        many = hb.kv4_attention(normal(g, 200, 1, 64), cache, table[:1], i32([length]), window=2 ** 31 - 1, out=torch.full((200, 1, 64), 3.0, device="cuda"))
        assert hb.device_status_rc() == (hb.ERR_INDEX, 1002) and not many.any()
    many = hb.kv4_attention(normal(g, 200, 1, 64), cache, table[:1], i32([(1 << 30) - 1]))
    assert hb.device_status_rc() == (hb.ERR_INDEX, 1002) and many.isfinite().all() and many.any()
    assert all(torch.equal(a, b) for a, b in zip(arrays, old))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N", [1, 2, 3, 7, 31, 33, 60, 61, 62, 63, 65, 97, 126, 127, 129, 250, 252, 253])
@pytest.mark.parametrize("M,times", [(1, 1), (5, 1), (300, 1), (300, 90)])
def test_int8_gemm_stores_nothing_behind_a_row(hb, dtype, N, M, times):
    """Results of every last column in rows on 16-byte borders that go on: what lies behind the last column, to the next border and beyond, stays."""
    g = gen(N + M)
    N, K = N + 256 * (times - 1), 70
    x, w = normal(g, M, K).to(dtype), hb.int8_quantize(normal(g, N, K))
    full = torch.full((M + 1, -(-(N + 9) // 8) * 8), 42.0, dtype=dtype, device="cuda")
    out = full[:M, :N]
    hb.int8_gemm(x, w, out=out)
    check_product(hb, x, w, None, out)
    out.fill_(42.0)
    assert (full == 42.0).all()


@pytest.mark.parametrize("M,N,K", [(1, 40, 201), (3, 40, 250), (5, 40, 201), (40, 40, 129), (200, 96, 257), (200, 96, 300), (2500, 1500, 333), (40, 100, 17), (300, 300, 1)])
def test_int8_gemm_reads_nothing_behind_the_contraction(hb, M, N, K):
    """Both operands converted before and anything behind their rows, up to 31 bytes: exact sums of the first K."""
    g = gen(K)
    pitch = (K + 15) // 16 * 16 + 16
    a, b = (torch.randint(-127, 128, (r, pitch), dtype=torch.int8, device="cuda", generator=g) for r in (M, N))
    y = hb.int8_gemm(hb.Int8Rows(a, torch.ones(M, device="cuda"), K), hb.Int8Rows(b, torch.ones(N, device="cuda"), K))
    assert torch.equal(y.double(), a[:, :K].double() @ b[:, :K].double().t())      # below 2^24: whole numbers in FP32


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K", [(2500, 4999, 2003), (4096, 4096, 1100), (3801, 1279, 1500), (38301, 380, 1030),        # pairs of SMs, 256, 256, 128, 128 channels
                                   (1111, 777, 3001), (100, 6500, 1500), (100, 13000, 900), (129, 6500, 900), (128, 12800, 1024)])      # a tile per CTA, 64, 64, 128 ...
def test_int8_gemm_of_many_tiles_and_stages(hb, dtype, M, N, K):
    """Contractions of more steps than a kernel has stages, more tiles than it has accumulators; results stored as tiles (rows on 16-byte borders)
    and element by element (rows off them), with nothing around them touched."""
    g = gen(M + N + K)
    x = normal(g, M, K).mul_(torch.exp(normal(g, M, 1))).to(dtype)
    w = hb.int8_quantize(normal(g, N, K) * torch.exp(normal(g, N, 1)))
    bias = normal(g, N)
    y = hb.int8_gemm(x, w, bias=bias)
    if dtype == torch.float16 and y.isinf().any():
        # Beyond 65520, half a step behind binary16's largest number, the rounded result is an infinity. What is rounded is the FP32 result, which a
        # call for that type gives and which the bound holds for; the rest of y is its rounding.
        exact = hb.int8_gemm(x, w, bias=bias, dtype=torch.float32)
        check_product(hb, x, w, bias, exact)
        assert torch.equal(y.isinf(), exact.abs() >= 65520) and torch.equal(y, exact.half())
    else:
        check_product(hb, x, w, bias, y)
    pitch = -(-(N + 8) // 8) * 8
    for width, first in ((pitch, 0), (pitch + 1, 3)):
        full = torch.full((M + 2, width), 42.0, dtype=dtype, device="cuda")
        out = full[1:M + 1, first:first + N]
        hb.int8_gemm(x, w, bias=bias, out=out)
        assert torch.equal(out, y)
        out.fill_(42.0)
        assert (full == 42.0).all()


def split_bytes(hb, dtype, heads, group, D, page, width, sequences, n, window):
    """What a call of so many tokens a sequence asks for as workspace: 0 where its launch is one."""
    import ctypes
    from tests.test_serving_cpu import batch, cache
    got = ctypes.c_size_t()
    b = batch(sequences=sequences, tokens=sequences * n, max_tokens=n, table_pages=width, table_ld=width)
    rc = hb.lib().hbfp_kv4_attention_workspace(ctypes.byref(cache(heads=heads, dim=D, page=page)), ctypes.byref(b), DTYPES.index(dtype), group, window, ctypes.byref(got))
    assert rc == hb.OK
    return got.value


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("heads,group,n,window,lengths", [
    (16, 1, 1, 2000, [9000, 4096, 1999, 100, 0] * 3),            # many tiles: eight rows a CTA in the join, few parts of a tile
    (8, 4, 3, 4096, [9000, 4096, 4099, 100, 2] * 3),             # 12 rows
    (8, 5, 4, 4096, [9000, 4200, 1999, 3, 64] * 3),              # 20 rows (256 wide: two tiles of rows)
    (2, 8, 1, 13000, [20000, 13000, 13063, 0]),                  # few tiles of many parts: a row a CTA in the join
    (1, 3, 4, 13000, [20000, 13001, 300, 4]),
    (1, 7, 4, 16000, [30000]),
    (1, 8, 1, 30000, [60000] + [100] * 59)])                     # one tile of many parts among many tiles
def test_attention_window_over_keys_that_are_split(hb, dtype, D, heads, group, n, window, lengths):
    """A launch that shares out the units of all sequences' windows, and its join: sequences shorter and longer than the window, units that start
    at its rounded edge."""
    page = 64
    many = D == 256 and dtype == torch.bfloat16 and group * n > 16 and window < 8000      # these take the kernel of many rows, in one launch
    assert (split_bytes(hb, dtype, heads, group, D, page, -(-max(lengths) // page), len(lengths), n, window) > 0) != many
    q, cache, table, y = check_attention(hb, dtype, heads, group, D, page, lengths, [n] * len(lengths), window=window)
    assert torch.equal(hb.kv4_attention(q, cache, table, i32(lengths), window=window), y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("heads,group,n,lengths", [(2, 3, 4, [20000, 700, 4]), (1, 16, 1, [40000]), (8, 4, 3, [9000, 5000, 3, 100] * 4), (4, 7, 4, [9000, 2049, 31, 640] * 6),
                                                   (1, 4, 7, [70000] + [90] * 59)])
def test_attention_wider_tiles_over_keys_that_are_split(hb, dtype, D, heads, group, n, lengths):
    """Tiles of 16 and 32 rows in both forms of the join, with few and many parts."""
    assert split_bytes(hb, dtype, heads, group, D, 64, -(-max(lengths) // 64), len(lengths), n, 0) > 0
    check_attention(hb, dtype, heads, group, D, 64, lengths, [n] * len(lengths))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,D,page", [(1, 64, 16), (3, 96, 32), (8, 128, 64), (2, 256, 16)])
@pytest.mark.parametrize("count", [1, 5, 33, 71])
def test_read_gives_what_was_written_and_zeros_where_there_is_no_position(hb, dtype, heads, D, page, count):
    """Keys and values exactly, of more positions than some of the sequences have; the oracle's conversion is what was written."""
    g = gen(D + count)
    lengths = [0, 1, 2, 31, 32, 70, 131]
    table, pages = pages_of(lengths, page, g)
    cache = hb.kv4_alloc(pages, heads, page, D)
    for t in (cache.k_mant, cache.k_exps, cache.v_mant, cache.v_exps):
        t.fill_(0x5A)
    x = (normal(g, sum(lengths), 2, heads, D) * torch.exp(2 * normal(g, 1, 2, heads, 1))).to(dtype)
    starts = np.cumsum([0] + lengths)
    hb.kv4_append(cache, x[:, 0], x[:, 1], table, i32(lengths), starts=i32(starts.tolist()))
    got = hb.kv4_read(cache, count, table, i32(lengths))
    for side in range(2):
        q, s = oracle.quantize(np.ascontiguousarray(x[:, side].float().cpu().numpy().reshape(-1, D)), 1, oracle.Format(mant_bits=4, block=32))
        value = (q.reshape(-1, D // 32, 32) * np.exp2(s.astype(np.float64))[..., None]).reshape(-1, heads, D)
        want = np.zeros((len(lengths), count, heads, D))
        for b, L in enumerate(lengths):
            m = min(L, count)
            if m:
                want[b, count - m:] = value[starts[b + 1] - m:starts[b + 1]]
        assert got[side].shape == (len(lengths) * count, heads, D) and got[side].dtype == torch.float32
        assert np.array_equal(got[side].double().cpu().numpy(), want.reshape(-1, heads, D))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M", [1, 3, 16, 300])
def test_int8_gemm_into_its_activations(hb, dtype, M):
    """Refused where the product reads them itself (up to three tokens), right where they are converted first and in the other half of their rows."""
    g = gen(71)
    w = hb.int8_quantize(normal(g, 64, 64))
    both = normal(g, M, 128).to(dtype)
    x, y = both[:, :64], both[:, 64:]
    want = hb.int8_gemm(x.clone(), w)
    hb.int8_gemm(x, w, out=y)
    assert torch.equal(y, want)
    for out in (x, both[:, 32:96]):
        if M > 3:
            keep = x.clone()
            assert torch.equal(hb.int8_gemm(x, w, out=out), want)
            x.copy_(keep)
            continue
        with pytest.raises(hb.HbfpError) as e:
            hb.int8_gemm(x, w, out=out)
        assert e.value.code == hb.ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lengths,n,heads,group", [([40, 700], 1, 2, 4), ([5000, 3], 1, 4, 4), ([5000, 3, 1999] * 8, 1, 8, 2), ([20000, 40], 3, 2, 5), ([300, 600], 130, 2, 2), ([9000, 300], 130, 1, 2)])
def test_attention_into_its_queries(hb, dtype, lengths, n, heads, group):
    """Every row is read where it is written and before: one launch, clusters, split keys, many rows."""
    g = gen(72)
    table, pages = pages_of(lengths, 64, g)
    cache = fill(hb, g, pages, heads, 64, 128)
    q = normal(g, len(lengths) * n, heads * group, 128).to(dtype)
    want = hb.kv4_attention(q, cache, table, i32(lengths))
    assert hb.kv4_attention(q, cache, table, i32(lengths), out=q) is q
    assert torch.equal(q, want)


def test_a_sequence_too_long_for_positions_reads_as_zeros(hb):
    """Not as whatever the new result's memory held."""
    g = gen(81)
    cache = fill(hb, g, 3, 2, 16, 64)
    table = i32([[0, 1, 2]] * 3)
    want = hb.kv4_read(cache, 7, table[:1], i32([40]))
    for _ in range(3):
        junk = [torch.full((3 * 7, 2, 64), 5.0, device="cuda") for _ in range(8)]
        del junk
        k, v = hb.kv4_read(cache, 7, table, i32([1 << 30, 40, 2 ** 31 - 1]))
        assert hb.device_status_rc() == (hb.ERR_INDEX, 1002)
        assert not k[:7].any() and not v[:7].any() and not k[14:].any() and not v[14:].any()
        assert torch.equal(k[7:14], want[0]) and torch.equal(v[7:14], want[1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("heads,group,n,window", [(1, 3, 96, 0), (8, 4, 224, 0), (3, 1, 300, 5), (2, 7, 188, 0), (8, 8, 43, 30)])
def test_attention_of_padded_batches_of_many_rows(hb, dtype, D, heads, group, n, window):
    """Sequences far shorter than their rows: whole row tiles without a key are zeros, every time, whatever their queries and what the result held."""
    lengths = [0, 1, n, 0, 7, n + 40, 1]
    g = gen(D + n)
    table, pages = pages_of(lengths, 32, g)
    cache = fill(hb, g, pages, heads, 32, D)
    q = normal(g, len(lengths) * n, heads * group, D).to(dtype)
    ref, tol = attend_reference(q, cache, table, lengths, [n] * len(lengths), D ** -0.5, window)
    out = torch.empty_like(q)
    for _ in range(10):
        hb.kv4_attention(q, cache, table, i32(lengths), window=window, out=out.fill_(9.0))
        assert (out.double() - ref).abs().le(tol).all()
        for b, L in enumerate(lengths):
            assert not out[b * n:(b + 1) * n - L].any()
