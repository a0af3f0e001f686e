"""Serving operators without a GPU: what the C ABI and the binding refuse before anything is launched."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def hb():
    from paper_1804_01526_b200 import build
    build.build()
    from paper_1804_01526_b200 import binding
    return binding


class _Cache(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("heads", ctypes.c_int32), ("dim", ctypes.c_int32), ("page", ctypes.c_int32), ("pages", ctypes.c_int64),
                ("k_mant", ctypes.c_void_p), ("k_exps", ctypes.c_void_p), ("v_mant", ctypes.c_void_p), ("v_exps", ctypes.c_void_p)]


class _Batch(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("sequences", ctypes.c_int32), ("table", ctypes.c_void_p), ("table_ld", ctypes.c_int64),
                ("table_pages", ctypes.c_int32), ("max_tokens", ctypes.c_int32), ("lengths", ctypes.c_void_p), ("starts", ctypes.c_void_p), ("tokens", ctypes.c_int64)]


P = 0x10000        # stands for a device address: nothing here is read


def cache(**kw):
    d = dict(struct_size=ctypes.sizeof(_Cache), heads=2, dim=64, page=16, pages=4, k_mant=P, k_exps=P, v_mant=P, v_exps=P)
    d.update(kw)
    return _Cache(**d)


def batch(**kw):
    d = dict(struct_size=ctypes.sizeof(_Batch), sequences=3, table=P, table_ld=2, table_pages=2, max_tokens=1, lengths=P, starts=None, tokens=3)
    d.update(kw)
    return _Batch(**d)


def test_int8_quantize_refusals(hb):
    f = hb.lib().hbfp_int8_quantize
    ok = dict(x=P, dtype=0, d0=4, d1=20, ld=20, axis=1, q=P, pitch=32, scale=P)

    def call(**kw):
        a = {**ok, **kw}
        return f(a["x"], a["dtype"], a["d0"], a["d1"], a["ld"], a["axis"], a["q"], a["pitch"], a["scale"], None)

    for bad in (dict(dtype=3), dict(dtype=-1), dict(d0=-1), dict(d1=-1), dict(ld=19), dict(axis=2), dict(x=None), dict(q=None), dict(scale=None),
                dict(pitch=16), dict(axis=0, pitch=0)):
        assert call(**bad) == hb.ERR_INVALID_ARG, bad
    for bad in (dict(pitch=40), dict(q=P + 8)):
        assert call(**bad) == hb.ERR_ALIGNMENT, bad
    assert call(d0=1 << 30) == hb.ERR_UNSUPPORTED


def test_int8_gemm_refusals(hb):
    f = hb.lib().hbfp_int8_gemm
    ok = dict(M=4, N=8, K=20, a=P, ta=0, lda=20, sa=None, w=P, ldw=32, sw=P, bias=None, y=P, ty=0, ldy=8, ws=P, bytes=1 << 20)

    def call(**kw):
        a = {**ok, **kw}
        return f(a["M"], a["N"], a["K"], a["a"], a["ta"], a["lda"], a["sa"], a["w"], a["ldw"], a["sw"], a["bias"], a["y"], a["ty"], a["ldy"], a["ws"], a["bytes"], None)

    for bad in (dict(M=-1), dict(K=-1), dict(ta=4), dict(ty=3), dict(ldy=7), dict(lda=19), dict(ldw=16), dict(a=None), dict(w=None), dict(sw=None), dict(y=None),
                dict(ta=3, lda=32)):
        assert call(**bad) == hb.ERR_INVALID_ARG, bad
    for bad in (dict(ldw=24), dict(w=P + 4), dict(ta=3, lda=24, sa=P), dict(ta=3, lda=32, sa=P, a=P + 1), dict(M=4000, ws=P + 16)):
        assert call(**bad) == hb.ERR_ALIGNMENT, bad
    assert call(M=4000, ws=None) == hb.ERR_WORKSPACE and call(M=4000, bytes=16) == hb.ERR_WORKSPACE
    for bad in (dict(K=131072, lda=131072, ldw=131072), dict(M=1 << 30), dict(N=1 << 30, ldy=1 << 30)):      # the sum has to fit int32
        assert call(**bad) == hb.ERR_UNSUPPORTED, bad
    assert call(M=0) == hb.OK and call(N=0, ldy=0) == hb.OK
    n = ctypes.c_size_t()
    assert hb.lib().hbfp_int8_gemm_workspace(5, 7, 100, 3, ctypes.byref(n)) == hb.OK and n.value == 0
    assert hb.lib().hbfp_int8_gemm_workspace(5, 7, 100, 1, None) == hb.ERR_INVALID_ARG


@pytest.mark.parametrize("call", ["append", "read", "attention", "workspace"])
def test_kv4_refusals(hb, call):
    L = hb.lib()

    def go(c=None, b=None, dtype=0, group=1, window=0):
        c, b = c or cache(), b or batch()
        c, b = ctypes.byref(c), ctypes.byref(b)
        if call == "append":
            return L.hbfp_kv4_append(c, b, dtype, None, 128, 64, None, 128, 64, None)
        if call == "read":
            return L.hbfp_kv4_read(c, b, 1, None, None, None)
        if call == "workspace":
            return L.hbfp_kv4_attention_workspace(c, b, dtype, group, window, None)
        return L.hbfp_kv4_attention(c, b, dtype, None, 128, 64, group, 1.0, window, None, 128, 64, None, 0, None)

    invalid = [dict(c=cache(struct_size=8)), dict(b=batch(struct_size=8)), dict(c=cache(heads=0)), dict(c=cache(pages=-1)), dict(c=cache(k_mant=None)),
               dict(c=cache(v_exps=None)), dict(b=batch(sequences=-1)), dict(b=batch(table_pages=-1)), dict(b=batch(table_ld=1)), dict(b=batch(lengths=None)), dict(b=batch(table=None))]
    if call != "read":
        invalid += [dict(dtype=3), dict(b=batch(tokens=4)), dict(b=batch(max_tokens=-1)), dict(b=batch(tokens=-3))]
    if call == "attention":
        invalid += [dict(group=0), dict(window=-1)]
    for bad in invalid:
        assert go(**bad) == hb.ERR_INVALID_ARG, bad
    if call == "workspace":
        return
    for bad in (dict(c=cache(page=8)), dict(c=cache(page=24)), dict(c=cache(dim=80)), dict(c=cache(dim=32)), dict(b=batch(table_pages=1 << 27, table_ld=1 << 27)),
                dict(b=batch(sequences=70000, tokens=70000))):
        assert go(**bad) == hb.ERR_UNSUPPORTED, bad
    assert go(c=cache(k_mant=P + 8)) == hb.ERR_ALIGNMENT
    assert go(b=batch(sequences=0, tokens=0)) == hb.OK                       # nothing to do
    if call == "append":
        assert go() == hb.ERR_INVALID_ARG                                    # no k


def test_binding_refuses_what_it_can_see(hb):
    x = torch.zeros(4, 32)
    w = hb.Int8Rows(torch.zeros(8, 32, dtype=torch.int8), torch.ones(8), 32)
    with pytest.raises(ValueError):
        hb.int8_quantize(x)                                                  # not on the GPU
    with pytest.raises(ValueError):
        hb.int8_gemm(x, w)
    with pytest.raises(ValueError):
        hb.int8_gemm(hb.Int8Rows(w.q, w.scale, 30), w)
    with pytest.raises(ValueError):
        hb.int8_gemm(x, w, dtype=torch.float64)
    with pytest.raises(ValueError):
        hb.int8_quantize(x, out=hb.Int8Rows(w.q, w.scale, 31))
    for bad in (dict(page=8), dict(page=48), dict(dim=80), dict(heads=0), dict(pages=-1)):
        with pytest.raises(ValueError):
            hb.kv4_alloc(**{**dict(pages=2, heads=1, page=16, dim=64, device="cpu"), **bad})
    c = hb.kv4_alloc(2, 1, 16, 64, device="cpu")
    t, n = torch.zeros(1, 1, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    k = torch.zeros(1, 1, 64)
    with pytest.raises(ValueError):
        hb.kv4_append(c, k, k, t, n)
    with pytest.raises(ValueError):
        hb.kv4_read(c, 1, t, n)
    with pytest.raises(ValueError):
        hb.kv4_attention(k, c, t, n)
    with pytest.raises(TypeError):
        hb.kv4_attention(None, hb.Kv4Cache(None, None, None, None), t, n)


def test_status_of_index_errors_has_a_text(hb):
    assert "out of range" in hb.status_string(hb.ERR_INDEX)


def test_attention_refuses_a_scale_that_is_no_number(hb):
    """Also one whose product with log2(e) is none. Nothing else is wrong with the calls: without a sequence they have nothing to do."""
    c, b = ctypes.byref(cache()), ctypes.byref(batch(sequences=0, tokens=0))

    def go(scale):
        return hb.lib().hbfp_kv4_attention(c, b, 0, None, 128, 64, 1, scale, 0, None, 128, 64, None, 0, None)

    for scale in (float("nan"), float("inf"), -float("inf"), 3.0e38, -3.0e38):
        assert go(scale) == hb.ERR_INVALID_ARG, scale
    for scale in (0.0, -2.0, 1e-45, 2.3e38):
        assert go(scale) == hb.OK, scale


def test_int8_gemm_refuses_a_result_over_activations_that_it_reads_itself(hb):
    """Where the addresses say so. The other half of the same rows is another matrix; what is converted first has been read when results are stored.
    (Calls that the check lets through are made only where there is no GPU for them to run on.)"""
    f = hb.lib().hbfp_int8_gemm
    A = 1 << 20

    def call(y, M=3, N=20, K=20, ta=0, ty=0, lda=64, ldy=64):
        return f(M, N, K, A, ta, lda, P if ta == 3 else None, P, 32, P, None, y, ty, ldy, None, 0, None)

    for y in (A, A + 4 * 19, A + 4 * 45, A + 256, A - 4 * 19, A - 4 * 64, A + 4 * (128 + 19), A - 4 * (128 + 19)):
        assert call(y) == hb.ERR_INVALID_ARG, y - A
    assert call(A + 2 * 19, ta=1, ty=1) == hb.ERR_INVALID_ARG
    assert call(A, M=1) == call(A + 4 * 19, M=1) == call(A - 4 * 19, M=1) == call(A + 4 * 19, M=1, ldy=32) == hb.ERR_INVALID_ARG
    for M in (2, 7, 300):
        assert call(A + 16, M=M, ta=3, lda=256, ldy=64) == hb.ERR_INVALID_ARG
    assert call(A, M=7) == call(A, M=300) == hb.ERR_WORKSPACE
    if torch.cuda.is_available():
        return
    for y in (A + 4 * 20, A + 4 * 44, A - 4 * 20, A - 4 * 44, A + 4 * (128 + 20), A + 4 * 192, A - 4 * 192, A - 4 * (128 + 20), A + (1 << 40)):
        assert call(y) != hb.ERR_INVALID_ARG, y - A
    assert call(A + 2 * 20, ta=1, ty=1) != hb.ERR_INVALID_ARG and call(A + 4 * 20, M=1, ldy=32) != hb.ERR_INVALID_ARG
