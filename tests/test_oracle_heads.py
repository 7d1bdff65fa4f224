"""Pins of the oracle of the output head's operators, and the refusals of their entry points (checked on the host, so no
GPU is needed: nothing is enqueued)."""
import numpy as np
import pytest

from oracle import heads
from paper_2111_09389_b200 import _lib

OK, INVALID, UNSUPPORTED = 0, 1, 2
P = 1 << 20          # a device address that no call gets as far as using


# ------------------------------------------------------------------ 8-bit floats
def test_codes_and_their_values():
    """Values of the format by hand, every code's own value, halves to the even code, halves beyond the last step."""
    hand = {0x00: 0.0, 0x01: 2.0 ** -9, 0x07: 7 * 2.0 ** -9, 0x08: 2.0 ** -6, 0x38: 1.0, 0x39: 1.125, 0x7e: 448.0, 0xb8: -1.0, 0xfe: -448.0}
    for code, value in hand.items():
        assert heads.E4M3[code] == value
        assert heads.e4m3_encode(np.array([value]))[0] == code
    codes = np.array([c for c in range(256) if c not in (0x7f, 0xff)])
    assert np.array_equal(heads.e4m3_encode(heads.E4M3[codes]), codes)
    mid = (heads.E4M3[0x38] + heads.E4M3[0x39]) / 2, (heads.E4M3[0x39] + heads.E4M3[0x3a]) / 2
    assert list(heads.e4m3_encode(np.array(mid))) == [0x38, 0x3a]
    assert list(heads.e4m3_encode(np.array([2.0 ** -10, 1.5 * 2.0 ** -9, -2.0 ** -11]))) == [0x00, 0x02, 0x80]


def test_scales_at_their_borders():
    x = np.zeros((6, 130))
    x[0, 0], x[1, 0], x[2, 0], x[3, 0], x[4, 0] = 448, np.nextafter(448, 500), 2.0 ** -149, np.inf, 1.0
    x[4, 129] = -7.0
    q, s = heads.quantize_e4m3(x)
    assert [list(r) for r in s] == [[127, 127], [128, 127], [0, 127], [255, 127], [119, 121], [127, 127]]
    assert q[0, 0] == 0x7e and q[1, 0] == 0x76 and (q[3, :128] == 0x7f).all() and q[3, 128] == 0
    assert heads.E4M3[q[4, 0]] * 2.0 ** -8 == 1.0 and heads.E4M3[q[4, 129]] * 2.0 ** -6 == -7.0
    v = heads.dequantize_e4m3(q, s)
    assert v[4, 129] == -7.0 and np.isnan(v[3, :128]).all() and v[3, 129] == 0


def test_product_by_hand():
    q, s = heads.quantize_e4m3(np.array([[[1.0, -2.0, 0.5]], [[4.0, 0.0, 1.0]]]))
    r, t = heads.quantize_e4m3(np.array([[[3.0, 1.0, 2.0], [0.0, 0.0, 0.25]], [[1.0, 5.0, 8.0], [2.0, 2.0, 2.0]]]))
    c, size = heads.matmul_e4m3(q, s, r, t, bias=np.array([[1.0, 0.0], [0.0, -1.0]]))
    assert c.tolist() == [[[3.0, 0.125]], [[12.0, 9.0]]] and size.tolist() == [[[6.0, 0.125]], [[12.0, 10.0]]]


def test_pitches():
    L = _lib.lib()
    assert [L.lpdt_e4m3_pitch(c) for c in (0, 1, 16, 17, 1000)] == [0, 16, 16, 32, 1008]
    assert [L.lpdt_e4m3_scale_pitch(c) for c in (0, 1, 128, 129, 512, 513, 4096)] == [0, 4, 4, 4, 4, 8, 32]
    assert L.lpdt_e4m3_pitch(-1) == -1 and L.lpdt_e4m3_scale_pitch(-1) == -1


def test_quantizer_refusals():
    names = "x dtype nodes rows cols x_node x_row q scale qt scale_t stream".split()
    base = dict(x=P, dtype=0, nodes=2, rows=3, cols=5, x_node=15, x_row=5, q=P, scale=P, qt=P, scale_t=P, stream=0)
    call = lambda **kw: _lib.lib().lpdt_quantize_e4m3(*[{**base, **kw}[n] for n in names])
    for empty in (dict(nodes=0), dict(rows=0), dict(cols=0), dict(nodes=0, x=0, q=0, scale=0)):
        assert call(**empty) == OK
    for bad in (dict(x=0), dict(dtype=3), dict(dtype=-1), dict(nodes=-1), dict(rows=-1), dict(cols=-1), dict(scale=0), dict(q=0),
                dict(qt=0), dict(scale_t=0), dict(q=0, scale=0, qt=0, scale_t=0), dict(x_row=4), dict(x_node=-1), dict(q=P + 8),
                dict(qt=P + 1), dict(x=P + 2), dict(x=P + 1, dtype=1)):
        assert call(**bad) == INVALID, bad
    assert call(rows=1 << 31, qt=0, scale_t=0) == UNSUPPORTED
    assert call(rows=1 << 30, cols=512, x_row=512, qt=0, scale_t=0) == UNSUPPORTED
    assert call(rows=1 << 24) == UNSUPPORTED


def test_product_refusals():
    names = "nodes M N K A sA B sB bias bias_node addend C c_dtype c_node c_row status stream".split()
    base = dict(nodes=2, M=3, N=5, K=7, A=P, sA=P, B=P, sB=P, bias=0, bias_node=0, addend=0, C=P, c_dtype=0, c_node=15, c_row=5,
                status=0, stream=0)
    call = lambda **kw: _lib.lib().lpdt_matmul_e4m3(*[{**base, **kw}[n] for n in names])
    for empty in (dict(nodes=0), dict(M=0), dict(N=0), dict(N=0, A=0, C=0)):
        assert call(**empty) == OK
    for bad in (dict(nodes=-1), dict(M=-1), dict(N=-1), dict(K=0), dict(K=-5), dict(A=0), dict(sA=0), dict(B=0), dict(sB=0), dict(C=0),
                dict(c_dtype=7), dict(A=P + 8), dict(B=P + 4), dict(sA=P + 2), dict(sB=P + 1), dict(C=P + 2), dict(addend=P + 1),
                dict(c_row=4), dict(c_node=14), dict(bias=P, bias_node=-1), dict(bias=P + 2), dict(status=P + 1)):
        assert call(**bad) == INVALID, bad
    assert call(K=(1 << 30) + 1) == UNSUPPORTED and call(M=1 << 31, c_node=1 << 40) == UNSUPPORTED


# ------------------------------------------------------------------ reports and losses
def test_logprobs_by_hand():
    x = np.array([[0.0, np.log(3.0), -np.inf], [2.0, 2.0, 2.0], [-np.inf] * 3])
    o = heads.token_logprobs(x, np.array([1, -1, 0]), 1.0, 2)
    assert np.allclose(o["lse"][:2], [np.log(4), 2 + np.log(3)]) and o["lse"][2] == -np.inf
    assert np.allclose(o["logprob"], [np.log(0.75), 0, -np.inf]) and np.allclose(o["entropy"], [np.log(4) - 0.75 * np.log(3), np.log(3), 0])
    assert o["top_index"].tolist() == [[1, 0], [0, 1], [0, 1]] and np.allclose(o["top_logprob"][0], np.log([0.75, 0.25]))


def difference(f, x, step=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += step
        down[i] -= step
        g[i] = (f(up) - f(down)) / (2 * step)
    return g


@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_logprobs_gradient_by_differences(temperature):
    rng = np.random.default_rng(0)
    x, tokens = rng.standard_normal((3, 7)) * 2, np.array([2, -1, 6])
    g, h, l = rng.standard_normal((3, 3))
    f = lambda x: sum((w * heads.token_logprobs(x, tokens, temperature)[n]).sum() for w, n in ((g, "logprob"), (h, "entropy"), (l, "lse")))
    assert np.allclose(heads.token_logprobs_bwd(x, tokens, g, h, l, temperature), difference(f, x), atol=1e-8)


@pytest.mark.parametrize("tail", [True, False])
def test_distillation_by_hand_and_by_differences(tail):
    """Two listed of three tokens; a token listed twice, a short list, no list, a row of weight 0."""
    x = np.log(np.array([[[0.5, 0.3, 0.2]]]))
    value, index = np.log(np.array([[[0.6, 0.1]]])), np.array([[[0, 2]]])
    t = np.array([0.6, 0.1, 0.3]) if tail else np.array([6 / 7, 1 / 7, 0])
    p = np.array([0.5, 0.2, 0.3])
    want = sum(a * np.log(a / b) for a, b in zip(t, p) if a)
    loss, row, grad = heads.distill_topk(x, value, index, tail)
    assert np.allclose([loss[0], row[0, 0]], want)
    assert np.allclose(grad[0, 0], np.array([0.5 - t[0], 0.3 - t[2], 0.2 - t[1]]))
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 3, 6))
    index = rng.integers(0, 6, (2, 3, 4))
    index[0, 1, 2:], index[0, 2], index[1, 0, 1] = -1, -1, index[1, 0, 0]
    value = np.log(rng.dirichlet(np.ones(4), (2, 3)) * 0.8)
    weight = np.array([[1.0, 2.0, 1.0], [0.5, 0.0, 3.0]])
    f = lambda x: heads.distill_topk(x, value, index, tail, 0.7, weight)[0].sum()
    assert np.allclose(heads.distill_topk(x, value, index, tail, 0.7, weight)[2], difference(f, x), atol=1e-8)


def test_report_refusals():
    names = "rows V x dtype stride temperature tokens logprob entropy lse k top index status stream".split()
    base = dict(rows=3, V=9, x=P, dtype=0, stride=9, temperature=1.0, tokens=P, logprob=P, entropy=P, lse=P, k=2, top=P, index=P, status=0, stream=0)
    call = lambda **kw: _lib.lib().lpdt_token_logprobs(*[{**base, **kw}[n] for n in names])
    assert call(rows=0) == OK and call(rows=0, x=0) == OK
    for bad in (dict(rows=-1), dict(V=0), dict(V=-3), dict(x=0), dict(dtype=9), dict(stride=8), dict(temperature=0.0), dict(temperature=-1.0),
                dict(temperature=float("nan")), dict(temperature=float("inf")), dict(tokens=0), dict(k=10), dict(k=-1), dict(top=0),
                dict(index=0), dict(logprob=0, entropy=0, lse=0, k=0), dict(x=P + 2), dict(x=P + 1, dtype=2), dict(tokens=P + 2), dict(lse=P + 1),
                dict(top=P + 3), dict(status=P + 2)):
        assert call(**bad) == INVALID, bad
    assert call(k=129, V=200, stride=200) == UNSUPPORTED and call(V=(1 << 30) + 1, stride=1 << 31) == UNSUPPORTED and call(rows=1 << 28) == UNSUPPORTED


def test_report_gradient_refusals():
    names = "rows V x dtype stride temperature tokens lse entropy g h l dx dstride stream".split()
    base = dict(rows=3, V=9, x=P, dtype=0, stride=9, temperature=1.0, tokens=P, lse=P, entropy=P, g=P, h=P, l=P, dx=P * 2, dstride=9, stream=0)
    call = lambda **kw: _lib.lib().lpdt_token_logprobs_bwd(*[{**base, **kw}[n] for n in names])
    assert call(rows=0) == OK
    for bad in (dict(rows=-1), dict(V=0), dict(x=0), dict(dx=0), dict(lse=0), dict(tokens=0), dict(entropy=0), dict(g=0, h=0, l=0), dict(dstride=8),
                dict(stride=1), dict(dx=P, dstride=10), dict(dx=P + 1), dict(temperature=0.0), dict(dtype=3), dict(lse=P + 2), dict(h=P + 1)):
        assert call(**bad) == INVALID, bad
    assert call(rows=1 << 28) == UNSUPPORTED


def test_distillation_refusals():
    names = "nodes B V x dtype stride temperature k value index tail weight loss row_loss dx dstride status stream".split()
    base = dict(nodes=2, B=3, V=9, x=P, dtype=0, stride=9, temperature=1.0, k=2, value=P, index=P, tail=1, weight=0, loss=P, row_loss=P, dx=2 * P,
                dstride=9, status=0, stream=0)
    call = lambda **kw: _lib.lib().lpdt_distill_topk(*[{**base, **kw}[n] for n in names])
    assert call(nodes=0) == OK
    for bad in (dict(nodes=-1), dict(B=0), dict(V=0), dict(x=0), dict(value=0), dict(index=0), dict(loss=0), dict(row_loss=0), dict(k=0), dict(k=-2),
                dict(tail=2), dict(stride=8), dict(dstride=3), dict(dx=P, dstride=12), dict(temperature=0.0), dict(temperature=float("nan")),
                dict(dtype=-1), dict(x=P + 1), dict(dx=2 * P + 2), dict(value=P + 2), dict(index=P + 1), dict(weight=P + 3), dict(loss=P + 2)):
        assert call(**bad) == INVALID, bad
    assert call(k=129) == UNSUPPORTED and call(V=(1 << 20) + 1, stride=1 << 21, dstride=1 << 21) == UNSUPPORTED


def test_recorded_sequences_take_the_calls():
    """Empty calls of each run in a recorded sequence; a bad one is refused there as by itself."""
    import ctypes as C
    from paper_2111_09389_b200 import api
    f = C.c_uint32.from_buffer(C.c_float(1.0)).value
    items = {"lpdt_quantize_e4m3": [0, 0, 0, 1, 1, 1, 1, 0, 0, 0, 0], "lpdt_matmul_e4m3": [0, 1, 1, 1] + [0] * 12,
             "lpdt_token_logprobs": [0, 5, 0, 0, 5, f] + [0] * 8, "lpdt_token_logprobs_bwd": [0, 5, 0, 0, 5, f] + [0] * 8,
             "lpdt_distill_topk": [0, 1, 5, 0, 0, 5, f, 1, 0, 0, 1] + [0] * 6}
    words = []
    for name, args in items.items():
        i = api.lpdt_call_id(name)
        assert i >= 0, name
        words += [i, 0] + args
    code = lambda w: (C.c_uint64 * len(w))(*w)
    assert api.lpdt_run_calls(code(words), [0]) == (0, 4)
    words[-8] = 7                                              # tail
    words[-17] = 1                                             # nodes
    assert api.lpdt_run_calls(code(words), [0])[0] == INVALID


def test_the_binding_refuses_other_types():
    """64-bit token numbers, log probabilities of 16 bits and codes that are no bytes would be read as something else."""
    import torch
    from paper_2111_09389_b200 import api
    z, i64, b16, i8 = torch.zeros(4), torch.zeros(4, dtype=torch.int64), torch.zeros(4, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int8)
    on_gpu = type("Logits", (), dict(is_cuda=True, dtype=torch.float32, data_ptr=lambda self: P))()
    for bad, call in ((i64, lambda t: api.lpdt_token_logprobs(1, 4, on_gpu, tokens=t)), (b16, lambda t: api.lpdt_token_logprobs(1, 4, on_gpu, lse=t)),
                      (i64, lambda t: api.lpdt_token_logprobs_bwd(1, 4, on_gpu, t, None, None, on_gpu)),
                      (b16, lambda t: api.lpdt_distill_topk(1, 1, 4, on_gpu, 1, t, None, None, None)),
                      (z, lambda t: api.lpdt_distill_topk(1, 1, 4, on_gpu, 1, None, t, None, None)),
                      (i8, lambda t: api.lpdt_quantize_e4m3(on_gpu, 1, 1, 4, q=t)), (z, lambda t: api.lpdt_matmul_e4m3(1, 1, 1, 1, t, None, None, None, on_gpu)),
                      (b16, lambda t: api.lpdt_matmul_e4m3(1, 1, 1, 1, None, None, None, None, on_gpu, bias=t))):
        with pytest.raises(AssertionError, match="expected, not " + str(bad.dtype)):
            call(bad)
