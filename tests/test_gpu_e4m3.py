"""8-bit floats with a scale for each block of 128: codes and scales equal to the oracle's bit for bit, products against
64-bit sums, refusals."""
import numpy as np
import pytest
import torch

from oracle import heads
from paper_2111_09389_b200 import api

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def quantize(x, both=True, rows_form=True, **kw):
    """(q, s, qt, st) of x [nodes][rows][cols] as numpy, cut to the columns, from buffers filled with a pattern."""
    n, r, c = x.shape
    new = lambda a, b: torch.full((n, a, b), 0xA5, dtype=torch.uint8, device="cuda")
    q, s = (new(r, api.lpdt_e4m3_pitch(c)), new(r, api.lpdt_e4m3_scale_pitch(c))) if rows_form else (None, None)
    qt, st = (new(c, api.lpdt_e4m3_pitch(r)), new(c, api.lpdt_e4m3_scale_pitch(r))) if both else (None, None)
    api.lpdt_quantize_e4m3(x, n, r, c, q, s, qt, st, **kw)
    cut = lambda t, k: None if t is None else t.cpu().numpy()[..., :k]
    return cut(q, c), cut(s, -(-c // 128)), cut(qt, r), cut(st, -(-r // 128))


def check_quantized(x, got):
    ref = x.double().cpu().numpy()
    for (q, s), want in (((got[0], got[1]), ref), ((got[2], got[3]), ref.transpose(0, 2, 1))):
        if q is not None:
            qr, sr = heads.quantize_e4m3(want)
            assert np.array_equal(s, sr)
            assert np.array_equal(q, qr)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 1, 4096), (3, 7, 129), (2, 130, 127), (1, 128, 128), (2, 257, 300), (1, 1, 5),
                                   (5, 33, 16), (1, 700, 1000), (1, 4096, 640)])
def test_quantize(shape, dtype):
    g = torch.Generator().manual_seed(sum(shape))
    x = (torch.randn(shape, generator=g) * torch.exp(2 * torch.randn(shape[0], shape[1], 1, generator=g))).to(dtype).cuda()
    check_quantized(x, quantize(x))
    check_quantized(x, quantize(x, both=False))
    check_quantized(x, quantize(x, rows_form=False))


def edge_values():
    """Blocks at the borders: amax on and beside 448 * 2^e, the largest and smallest floats, ties, zeros of both signs,
    NaN and infinities."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((24, 256)).astype(np.float32)
    for i, e in enumerate((-140, -128, -127, -20, 0, 1, 100, 119)):
        for j, v in enumerate((np.float32(448), np.nextafter(np.float32(448), np.float32(0)), np.nextafter(np.float32(448), np.float32(1e9)))):
            x[3 * i + j, :128] *= 0.25 * np.exp2(np.float64(e))
            x[3 * i + j, 5] = np.float64(v) * np.exp2(np.float64(e))
    x[0, 128:] = 0
    x[1, 128:] = -0.0
    x[2, 200] = np.nan
    x[3, 201] = np.inf
    x[4, 202] = -np.inf
    x[5, 128:] = np.finfo(np.float32).max
    x[6, 128:] = np.float32(1e-45)
    x[7, 128:] = np.arange(128) / 16 + 1 / 32                    # halves between codes
    x[7, 128] = 448
    x[8, 128:] = (np.arange(128) - 64) * 2.0 ** -10              # about the type's smallest steps
    x[8, 255] = 448
    x[9, 128:] = 3.0
    x[9, 130] = np.finfo(np.float32).tiny
    return torch.from_numpy(x)[None]


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_at_its_edges(dtype):
    x = edge_values()
    x = (x if dtype != torch.float16 else x.clamp(-60000, 60000) * 2.0 ** -8).to(dtype).cuda()
    check_quantized(x, quantize(x))
    check_quantized(x, quantize(x, both=False))
    t = x.transpose(1, 2).contiguous()
    check_quantized(t, quantize(t))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset,row_stride,node_stride", [(0, 304, 40000), (1, 301, 39991), (4, 304, 40004), (3, 300, 38400)])
def test_quantize_strided(dtype, offset, row_stride, node_stride):
    n, r, c = 2, 128, 300
    flat = torch.randn(offset + n * node_stride, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    x = torch.as_strided(flat, (n, r, c), (node_stride, row_stride, 1), offset)
    for kw in (dict(), dict(both=False)):
        check_quantized(x, quantize(x, x_row_stride=row_stride, x_node_stride=node_stride, **kw))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("r,c", [(5, 131), (131, 5), (1, 1), (257, 300)])
def test_quantize_behind_the_last_column(r, c, dtype):
    """Codes up to the pitch are zeros, or NaN where the last block is; no scale behind the last block is written, and no byte behind the form."""
    x = torch.randn(1, r, c, generator=torch.Generator().manual_seed(r)).to(dtype)
    x[0, r - 1, c - 1] = float("nan")
    x[0, 0, 0] = float("inf")
    cols, rows = api.lpdt_e4m3_pitch(c), api.lpdt_e4m3_pitch(r)
    for both in (False, True):
        q, s = (torch.full((r + 1, w), 0xA5, dtype=torch.uint8, device="cuda") for w in (cols, api.lpdt_e4m3_scale_pitch(c)))
        qt, st = (torch.full((c + 1, w), 0xA5, dtype=torch.uint8, device="cuda") for w in (rows, api.lpdt_e4m3_scale_pitch(r)))
        api.lpdt_quantize_e4m3(x.cuda(), 1, r, c, q, s, qt if both else None, st if both else None)
        for form, scales, size, length, values in ((q, s, r, c, x[0]), (qt, st, c, r, x[0].t()))[:1 + both]:
            form, scales, blocks = form.cpu(), scales.cpu(), -(-length // 128)
            bad = ~torch.isfinite(values[:, (blocks - 1) * 128:].float()).all(1)
            assert (form[:size, length:] == torch.where(bad, 0x7f, 0).to(torch.uint8)[:, None]).all()
            assert (scales[:size, blocks:] == 0xA5).all() and (scales[:size, blocks - 1] == 255).equal(bad)
            assert (form[size:] == 0xA5).all() and (scales[size:] == 0xA5).all()


def operands(nodes, M, N, K, seed, exact):
    """Codes and scales of A and B.  exact: small whole numbers, whose sums are whole numbers below 2^24."""
    rng = np.random.default_rng(seed)
    out = []
    for rows in (M, N):
        if exact:
            v = rng.integers(-4, 5, (nodes, rows, K)).astype(np.float64)
            q = heads.e4m3_encode(v)
            s = rng.integers(127, 129, (nodes, rows, -(-K // 128))).astype(np.uint8)
        else:
            q, s = heads.quantize_e4m3((rng.standard_normal((nodes, rows, K)) * np.exp(rng.standard_normal((nodes, rows, 1)))).astype(np.float32))
        out += [q, s]
    return out


def padded(a, pitch, fill=0xA5):
    t = np.full(a.shape[:-1] + (pitch,), fill, np.uint8)
    t[..., :a.shape[-1]] = a
    return torch.from_numpy(t).cuda()


def device_operands(ops, K):
    qa, sa, qb, sb = ops
    P, S = api.lpdt_e4m3_pitch(K), api.lpdt_e4m3_scale_pitch(K)
    return padded(qa, P), padded(sa, S), padded(qb, P), padded(sb, S)


# one token; few rows, whose K several CTAs share; ragged; one block; many blocks of K; several nodes; more tiles than SMs; pairs of SMs
SHAPES = [(1, 1, 16, 128), (1, 1, 4096, 4096), (1, 1, 1, 1), (2, 3, 5, 7), (1, 17, 300, 1000), (3, 64, 200, 513), (4, 150, 130, 257),
          (1, 128, 128, 129), (1, 33, 1, 8191), (1, 240, 256, 384), (1, 500, 1023, 640), (1, 1025, 2049, 300), (2, 700, 1500, 1200),
          (1, 2048, 2048, 512), (5, 1, 129, 2000), (1, 4100, 515, 130),
          (1, 90, 4100, 2900), (2, 1615, 4810, 3788), (3, 433, 4791, 2776), (2, 4188, 4744, 259)]


@pytest.mark.parametrize("shape", SHAPES)
def test_matmul_of_whole_numbers_is_exact(shape):
    """|a b| <= 16 * 4, K <= 8191: every partial sum is a whole number below 2^24, so any order gives the same bits."""
    nodes, M, N, K = shape
    ops = operands(*shape, seed=M + N, exact=True)
    want, _ = heads.matmul_e4m3(*ops)
    C = torch.full((nodes, M, N), 7.5, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.lpdt_matmul_e4m3(nodes, M, N, K, *device_operands(ops, K), C, dev_status=status)
    assert api.lpdt_check_status(status) == 0
    assert np.array_equal(C.double().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES[::2])
def test_matmul(shape, dtype):
    """Products are exact in fp32; each of the K/32 steps of accumulation may lose up to 33 terms' bits below 2^-24 of the largest
    magnitude that it adds, at most sum|ab|; then up to two additions and the rounding to the type of C."""
    nodes, M, N, K = shape
    ops = operands(*shape, seed=M * N + K, exact=False)
    rng = np.random.default_rng(5)
    bias = rng.standard_normal((nodes, N)).astype(np.float32)
    addend = torch.from_numpy(rng.standard_normal((nodes, M, N))).to(dtype)
    A = device_operands(ops, K)
    for kw, ref in (({}, {}), (dict(bias=torch.from_numpy(bias).cuda(), bias_node_stride=N), dict(bias=bias)),
                    (dict(bias=torch.from_numpy(bias).cuda(), bias_node_stride=N, addend=addend.cuda()),
                     dict(bias=bias, addend=addend.double().numpy()))):
        want, size = heads.matmul_e4m3(*ops, **ref)
        C = torch.empty(nodes, M, N, dtype=dtype, device="cuda")
        api.lpdt_matmul_e4m3(nodes, M, N, K, *A, C, **kw)
        total = size + sum(np.abs(np.broadcast_to(v[:, None] if v.ndim == 2 else v, size.shape)) for v in ref.values())
        tol = 33 * -(-K // 32) * 2.0 ** -24 * size + 2 * 2.0 ** -23 * total + torch.finfo(dtype).eps / 2 * np.abs(want) + 2.0 ** -25
        got = C.double().cpu().numpy()
        over = np.abs(want) + tol >= torch.finfo(dtype).max         # fp16: infinity from 65520 on
        err = np.abs(got - want)
        assert ((err <= tol) | (over & (np.abs(got) >= torch.finfo(dtype).max) & (np.sign(got) == np.sign(want)))).all(), (err / tol).max()


# wide tiles of pairs: one a pair, several; rows that end in each half of them; several nodes; the last with an addend too
WIDE = [(2, 231, 6725, 2861), (2, 906, 5701, 1478), (3, 337, 4272, 2094), (3, 747, 5016, 1793), (3, 789, 2479, 2097), (1, 519, 7988, 2962)]


@pytest.mark.parametrize("shape", WIDE)
def test_matmul_in_wide_tiles_is_exact(shape):
    test_matmul_of_whole_numbers_is_exact(shape)


@pytest.mark.parametrize("dtype,shape", [(torch.float32, WIDE[5]), (torch.bfloat16, WIDE[4]), (torch.float16, WIDE[1])])
def test_matmul_in_wide_tiles(shape, dtype):
    test_matmul(shape, dtype)


@pytest.mark.parametrize("shape", [(1, 96, 160, 8192), (1, 1, 200, 16000), (1, 300, 300, 1000)])
def test_matmul_loses_no_more_than_its_steps_cut(shape):
    """A step adds 32 products to the sum, 33 values each cut below 2^-24 of the largest magnitude M among them and what is summed so far:
    a bound for each element from its own partial sums, not from sum |a b|.  On the whole, cuts of products have either sign
    and 1/sqrt(3) of their bound, those of the sum one: sqrt(steps * 32 / 3) + steps / 2 cuts, partial sums on average 2/3 of the last."""
    nodes, M, N, K = shape
    ops = operands(*shape, seed=K, exact=False)
    C = torch.empty(nodes, M, N, device="cuda")
    api.lpdt_matmul_e4m3(nodes, M, N, K, *device_operands(ops, K), C)
    a, b = (torch.from_numpy(heads.dequantize_e4m3(ops[i], ops[i + 1])[0]).cuda() for i in (0, 2))
    total, tol, steps = torch.zeros(M, N, dtype=torch.float64, device="cuda"), 0.0, -(-K // 32)
    for k in range(0, K, 32):
        largest = (a[:, k:k + 32].abs()[:, None] * b[:, k:k + 32].abs()[None]).amax(-1)
        before = total.abs()
        total = total + a[:, k:k + 32] @ b[:, k:k + 32].t()
        tol = tol + 33 * 2.0 ** -24 * torch.maximum(torch.maximum(before, total.abs()), largest)
    err = (C[0].double() - total).abs()
    assert (err <= tol).all()
    assert err.norm() <= ((steps * 32 / 3) ** 0.5 + steps / 2) * 2.0 ** -24 * total.norm()


# The forms that a product takes, each with the kernel that has to answer: tiles of one turn and of several, K above and up to 8 blocks (from
# where on the epilogue asks for the addend early), results of 4 and 2 bytes.
F32, BF16, F16 = DTYPES
FORMS = [
    ((3, 131, 6709, 1167), F32, True, "<single>"), ((3, 298, 4144, 16), F32, True, "<single>"), ((2, 1, 5698, 1064), BF16, True, "<single>"),
    ((2, 231, 6725, 2861), F32, True, "<two an SM>"), ((3, 3, 6966, 17), F16, True, "<two an SM>"),
    ((1, 64, 9000, 8192), F32, True, "<K by 2>"), ((1, 1, 6265, 1595), F16, True, "<K by 2>"), ((1, 1, 5149, 477), F32, False, "<K by 2>"),
    ((1, 1, 2442, 1753), F32, True, "<K by 4>"), ((1, 1, 1530, 914), BF16, True, "<K by 8>"), ((1, 3, 253, 1176), F32, True, "<K by 8>"),
    ((3, 219, 3321, 3829), F32, False, "<pairs>"), ((1, 8192, 4096, 1024), F32, True, "<pairs>"), ((2, 1500, 5000, 1024), F32, True, "<pairs>"),
    ((3, 211, 7953, 1734), F32, True, "<pairs>"), ((2, 3585, 7531, 137), BF16, False, "<pairs>"), ((3, 2095, 2193, 773), F16, True, "<pairs>"),
    ((2, 493, 7097, 3142), F32, True, "<pairs, 256 rows>"), ((3, 715, 3962, 1367), BF16, False, "<pairs, 256 rows>"),
    ((2, 2742, 1576, 3853), F32, True, "<pairs, 288 rows>"), ((1, 4779, 1979, 2215), F32, False, "<pairs, 288 rows>"), ((1, 519, 7988, 2962), F32, True, "<pairs, 288 rows>"),
    ((3, 950, 3747, 3111), F32, True, "<pairs, 320 rows>"), ((2, 906, 5701, 1478), F16, False, "<pairs, 320 rows>"),
    ((2, 2717, 2206, 3497), F32, True, "<pairs, 352 rows>"), ((3, 337, 4272, 2094), BF16, False, "<pairs, 352 rows>"),
    ((1, 1816, 6331, 4177), F32, True, "<pairs, 384 rows>"), ((3, 747, 5016, 1793), F16, False, "<pairs, 384 rows>"),
    ((3, 4663, 923, 3930), F32, True, "<pairs, 416 rows>"), ((1, 2375, 5813, 2332), F32, False, "<pairs, 416 rows>"), ((3, 789, 2479, 2097), BF16, False, "<pairs, 416 rows>")]


@pytest.mark.parametrize("shape,dtype,addend,form", FORMS)
def test_matmul_takes_each_form_and_is_exact(shape, dtype, addend, form):
    """Whole numbers: sums below 2^24 in fp32 whatever the order, then the one rounding to the type of C.  With an addend into another matrix
    and onto itself."""
    nodes, M, N, K = shape
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    codes = torch.from_numpy(heads.e4m3_encode(np.arange(-4.0, 5.0))).cuda()
    P, S, nb = api.lpdt_e4m3_pitch(K), api.lpdt_e4m3_scale_pitch(K), -(-K // 128)
    f, values = [], []
    for rows in (M, N):
        v = torch.randint(0, 9, (nodes, rows, K), generator=g, device="cuda")
        e = torch.randint(0, 2, (nodes, rows, nb), generator=g, device="cuda")
        q, s = (torch.full((nodes, rows, w), 0xA5, dtype=torch.uint8, device="cuda") for w in (P, S))
        q[..., :K], s[..., :nb] = codes[v], (e + 127).to(torch.uint8)
        f += [q, s]
        values.append((v - 4).double() * torch.exp2(e.double()).repeat_interleave(128, -1)[..., :K])
    want = torch.matmul(values[0], values[1].transpose(1, 2))
    x = torch.randint(-99, 100, (nodes, M, N), generator=g, device="cuda").to(dtype) if addend else None
    want = (want if x is None else want + x.double()).float().to(dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for onto in ((x.clone(), torch.empty_like(x)) if addend else (torch.empty(nodes, M, N, dtype=dtype, device="cuda"),)):
        api.lpdt_matmul_e4m3(nodes, M, N, K, *f, onto, addend=onto if addend and torch.equal(onto, x) else x, dev_status=status)
        assert api.lpdt_last_kernel() == "lpdt::tc::matmul_e4m3_kernel" + form
        assert torch.equal(onto, want)
    assert api.lpdt_check_status(status) == 0


@pytest.mark.parametrize("shape", [(2, 37, 100, 256), (1, 300, 515, 640), (3, 1, 64, 2048)])
def test_matmul_into_a_flat_vector_and_onto_itself(shape):
    """Rows apart from one another inside a flat vector: nothing between them is written; addend = C accumulates."""
    nodes, M, N, K = shape
    ops = operands(*shape, seed=9, exact=True)
    want, _ = heads.matmul_e4m3(*ops)
    row, node = N + 5, M * (N + 5) + 11
    flat = torch.full((3 + nodes * node,), -3.0, device="cuda")
    C = torch.as_strided(flat, (nodes, M, N), (node, row, 1), 3)
    A = device_operands(ops, K)
    expect = flat.clone()
    torch.as_strided(expect, (nodes, M, N), (node, row, 1), 3).copy_(torch.from_numpy(want - 3.0))
    api.lpdt_matmul_e4m3(nodes, M, N, K, *A, C, c_row_stride=row, c_node_stride=node, addend=C)
    assert torch.equal(flat, expect)


def test_matmul_rows_with_nan_scales_stay_by_themselves():
    ops = operands(1, 40, 200, 300, seed=2, exact=True)
    ops[1][0, 7, 1] = 255
    ops[0][0, 7, 128:256] = 0x7f
    ops[3][0, 100, 2] = 255
    want, _ = heads.matmul_e4m3(*ops)
    C = torch.empty(1, 40, 200, device="cuda")
    api.lpdt_matmul_e4m3(1, 40, 200, 300, *device_operands(ops, 300), C)
    got = C.cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(got[0, 7]).all() and np.isnan(got[0, :, 100]).all()
    assert np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])


@pytest.mark.parametrize("ea,eb", [(0, 127), (254, 20), (200, 50), (127, 1)])
def test_matmul_at_the_ends_of_the_scales(ea, eb):
    """Factors from 2^-127 on; the product of the two is a float of ordinary size or as small as floats get."""
    qa = heads.e4m3_encode(np.full((1, 2, 32), 1.5))
    qb = heads.e4m3_encode(np.full((1, 16, 32), 2.0))
    sa, sb = np.full((1, 2, 1), ea, np.uint8), np.full((1, 16, 1), eb, np.uint8)
    want, _ = heads.matmul_e4m3(qa, sa, qb, sb)
    C = torch.empty(1, 2, 16, device="cuda")
    api.lpdt_matmul_e4m3(1, 2, 16, 32, *device_operands((qa, sa, qb, sb), 32), C)
    assert np.abs(C.double().cpu().numpy() - want).max() <= 2.0 ** -126
    if want.max() > 2.0 ** -100:
        assert np.array_equal(C.double().cpu().numpy(), want)


def test_two_streams_at_once_give_the_same_bits():
    """Products of every form (shared K, one and two tiles an SM, pairs, wide tiles) side by side on two streams, and captured into two graphs."""
    shapes = [(1, 1, 4096, 4096), (1, 1025, 2049, 300), (2, 700, 1500, 1200), (3, 433, 4791, 2776), (2, 906, 5701, 1478), (1, 64, 4096, 2048)]
    rng = torch.Generator(device="cuda").manual_seed(3)
    sets = []
    for n, M, N, K in shapes:
        f = []
        for r in (M, N):
            x = torch.randn(n, r, K, generator=rng, device="cuda", dtype=torch.float32)
            q = torch.empty(n, r, api.lpdt_e4m3_pitch(K), dtype=torch.uint8, device="cuda")
            s = torch.empty(n, r, api.lpdt_e4m3_scale_pitch(K), dtype=torch.uint8, device="cuda")
            api.lpdt_quantize_e4m3(x, n, r, K, q, s)
            f += [q, s]
        C = [torch.empty(n, M, N, dtype=torch.bfloat16, device="cuda") for _ in range(5)]
        api.lpdt_matmul_e4m3(n, M, N, K, *f, C[0])
        sets.append(((n, M, N, K), f, C))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    order = (list(range(6)), [4, 0, 5, 2, 1, 3])
    for rep in range(3):
        for step in range(6):
            for i, stream in enumerate(streams):
                shape, f, C = sets[order[i][step]]
                with torch.cuda.stream(stream):
                    api.lpdt_matmul_e4m3(*shape, *f, C[1 + i], dev_status=status)
    graphs = []
    for i, stream in enumerate(streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            for k in order[i]:
                shape, f, C = sets[k]
                api.lpdt_matmul_e4m3(*shape, *f, C[3 + i], dev_status=status)
        graphs.append(g)
    torch.cuda.synchronize()
    for rep in range(2):
        for g, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                g.replay()
    torch.cuda.synchronize()
    assert api.lpdt_check_status(status) == 0
    for _, _, C in sets:
        assert all(torch.equal(C[0], c) for c in C[1:])


def test_three_products_of_a_layer():
    """Forward, backward-data and backward-weight from the quantizer's two forms, as a layer uses them."""
    g = torch.Generator().manual_seed(0)
    n, r, cin, cout = 2, 200, 300, 150
    X, W, dY = (torch.randn(*s, generator=g).cuda() for s in ((n, r, cin), (n, cout, cin), (n, r, cout)))
    f = {}
    for name, t in (("X", X), ("W", W), ("dY", dY)):
        rows, cols = t.shape[1:]
        new = lambda a, b: (torch.empty(n, a, api.lpdt_e4m3_pitch(b), dtype=torch.uint8, device="cuda"),
                            torch.empty(n, a, api.lpdt_e4m3_scale_pitch(b), dtype=torch.uint8, device="cuda"))
        f[name], f[name + "t"] = new(rows, cols), new(cols, rows)
        api.lpdt_quantize_e4m3(t, n, rows, cols, *f[name], *f[name + "t"])
    Y, dX, dW = (torch.empty(*s, device="cuda") for s in ((n, r, cout), (n, r, cin), (n, cout, cin)))
    api.lpdt_matmul_e4m3(n, r, cout, cin, *f["X"], *f["W"], Y)
    api.lpdt_matmul_e4m3(n, r, cin, cout, *f["dY"], *f["Wt"], dX)
    api.lpdt_matmul_e4m3(n, cout, cin, r, *f["dYt"], *f["Xt"], dW)
    for got, a, b in ((Y, X, W), (dX, dY, W.transpose(1, 2)), (dW, dY.transpose(1, 2), X.transpose(1, 2))):
        a, b = a.double().cpu().numpy(), b.double().cpu().numpy()
        K = a.shape[-1]
        want = np.matmul(a, b.transpose(0, 2, 1))
        # each operand is off by half a step: 2^-4 of its value, or half of the smallest step (2^-10 of its block's scale <= amax / 224)
        ea, eb = (np.abs(v) * 2.0 ** -4 + 2.0 ** -10 * np.abs(v).max() / 224 for v in (a, b))
        tol = np.matmul(ea, np.abs(b).transpose(0, 2, 1)) + np.matmul(np.abs(a) + ea, eb.transpose(0, 2, 1))
        err = np.abs(got.double().cpu().numpy() - want)
        assert (err <= tol + K * 2.0 ** -20).all()
        assert np.sqrt((err ** 2).mean() / (want ** 2).mean()) < 0.06              # rms: two operands of 2^-4 / sqrt(3) at most
