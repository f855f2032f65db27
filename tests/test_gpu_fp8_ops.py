"""The e4m3 operators on plain tensors (quantisers and block-scaled product)
against float64 and against the bits that their definitions fix."""
import math

import pytest
import torch

from paper_2606_22541_gb300 import _native, api

pytestmark = pytest.mark.gpu
DEV = "cuda"
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(shape, seed, std=1.0):
    return torch.randn(shape, generator=gen(seed), device=DEV) * std


def view(t, rows, cols, ld, offset=0):
    """A [rows, cols] view with row stride ld at an element offset of flat t."""
    return t[offset:offset + rows * ld].view(rows, ld)[:, :cols]


def store(rows, cols, ld, offset, dtype, fill):
    flat = torch.full((rows * ld + offset + 64,), fill, device=DEV).to(dtype)
    return flat, view(flat, rows, cols, ld, offset)


# ------------------------------------------------------------------ quantisers

def encode(v):
    """The definition in fp32: scale amax * fl(1 / 448) per 128 columns, quotient by division."""
    n, c = v.shape
    p = torch.nn.functional.pad(v, (0, -c % 128)).view(n, -1, 128)
    s = p.nan_to_num(0.0, math.inf, -math.inf).abs().amax(2) * torch.tensor(1.0 / 448.0, device=DEV)
    s = torch.where(s > 0, s, torch.ones_like(s))
    q = (p / s[:, :, None]).clamp(-448, 448).to(F8).view(n, -1)[:, :c]
    return q, s


SHAPES = [(1, 1), (1, 128), (3, 127), (2, 129), (5, 256), (7, 1000), (64, 7168), (33, 2052), (1, 14336), (300, 8),
          (1000, 640), (2, 65536)]


@pytest.mark.parametrize("n,c", SHAPES)
@pytest.mark.parametrize("pad,offset", [(0, 0), (16, 0), (5, 3), (4, 4)])
def test_quantise_gives_the_definitions_bits(n, c, pad, offset):
    flat, x = store(n, c, c + pad, offset, torch.bfloat16, math.nan)
    x.copy_(randn((n, c), n + c) * torch.exp(randn((1, c), c, 3.0)))
    qflat, q = store(n, c, c + pad, offset, F8, 1.0)
    before = qflat.clone()
    sflat, s = store(n, -(-c // 128), -(-c // 128) + pad, 0, torch.float32, 7.0)
    api.asap_moe_fp8_quantize(x, q, s)
    rq, rs = encode(x.float())
    assert torch.equal(s, rs)
    assert torch.equal(q.contiguous().view(torch.uint8), rq.contiguous().view(torch.uint8))
    # nothing beside the rows is written
    q.view(torch.uint8).copy_(before.view(torch.uint8)[offset:offset + n * (c + pad)].view(n, c + pad)[:, :c])
    assert torch.equal(qflat.view(torch.uint8), before.view(torch.uint8))
    s.fill_(7.0)
    assert (sflat == 7.0).all()


def test_quantise_special_values():
    x = torch.zeros((6, 256), dtype=torch.bfloat16, device=DEV)
    x[1, 3] = 1e-38          # a group whose scale is subnormal
    x[1, 4] = -5e-39
    x[2] = randn((256,), 1).bfloat16()
    x[2, 7] = math.nan
    x[3] = randn((256,), 2).bfloat16()
    x[3, 130] = -math.inf
    x[4] = 3.3895e38         # the largest bf16
    x[5, 0] = 9.2e-41        # the smallest
    q = torch.empty((6, 256), dtype=F8, device=DEV)
    s = torch.empty((6, 2), device=DEV)
    api.asap_moe_fp8_quantize(x, q, s)
    rq, rs = encode(x.float())
    assert torch.equal(s, rs)
    v, rv = q.float(), rq.float()
    assert (s[0] == 1.0).all() and (v[0] == 0).all()
    assert torch.equal(v[1], rv[1]) and torch.equal(v[5], rv[5])
    assert v[2, 7].isnan() and torch.equal(v[2].nan_to_num(9), rv[2].nan_to_num(9))
    assert s[3, 1] == math.inf and v[3, 128:].isnan().all() and torch.equal(v[3, :128], rv[3, :128])
    assert (v[4] == 448).all()


@pytest.mark.parametrize("n,c", SHAPES)
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_swiglu_quantise(n, c, offset):
    """Halves of one row, as a product leaves them.  v is computed in fp32 within a few 2^-23 of its value: scales within
    that, and values equal but for those within it of the boundary between two e4m3 values."""
    flat, y = store(n, 2 * c, 2 * c + offset, offset, torch.bfloat16, math.nan)
    y.copy_(randn((n, 2 * c), 3 * n + c, 2.0))
    gate, up = y[:, :c], y[:, c:]
    q = torch.empty((n, c), dtype=F8, device=DEV)
    s = torch.empty((n, -(-c // 128)), device=DEV)
    api.asap_moe_fp8_swiglu_quantize(gate, up, q, s)
    g = gate.double()
    v = g * g.sigmoid() * up.double()
    rq, rs = encode(v.float())
    assert float(((s - rs).abs() / rs).max()) <= 16 * 2.0 ** -23
    got = q.double() * s.double().repeat_interleave(128, 1)[:, :c]
    spread = s.double().repeat_interleave(128, 1)[:, :c]
    # half a step of e4m3: 2^-4 of the value, 2^-10 of the scale below its smallest normal number
    step = torch.maximum(v.abs() * 2.0 ** -4, spread * 2.0 ** -10)
    assert ((got - v).abs() <= step * (1 + 1e-4)).all()
    assert float((q.float() != rq.float()).float().mean()) <= 1e-4 + 2.0 / (n * c)


def test_swiglu_extremes():
    g = torch.tensor([[0.0, -0.0, 100.0, -100.0, 3e38, -3e38, 88.5, -88.5]], device=DEV).bfloat16().repeat(1, 16)
    u = torch.ones_like(g)
    q = torch.empty(g.shape, dtype=F8, device=DEV)
    s = torch.empty((1, 1), device=DEV)
    api.asap_moe_fp8_swiglu_quantize(g, u, q, s)
    v = q.float()[0, :8] * s[0, 0]
    want = torch.tensor([0.0, 0.0, 0.0, 0.0, 3e38, 0.0, 0.0, 0.0], device=DEV)
    assert torch.allclose(v, want, rtol=0.07, atol=0.0)


# ------------------------------------------------------------------ product

def operands(m, n, k, seed, pad=0):
    ld = -(-k // 16) * 16 + 16 * pad

    def values(rows, s):
        flat, t = store(rows, k, ld, 0, F8, math.nan)  # what lies between the rows is not read as a number
        t.copy_(randn((rows, k), s, 100.0).clamp(-448, 448).to(F8))
        return t

    nb = -(-k // 128)
    a, b = values(m, seed), values(n, seed + 1)
    sa = torch.rand((m, nb), generator=gen(seed + 2), device=DEV) + 0.1
    sb = torch.rand((-(-n // 128), nb), generator=gen(seed + 3), device=DEV) + 0.1
    return a, sa, b, sb


def product64(a, sa, b, sb):
    (m, k), n = a.shape, b.shape[0]
    out = torch.zeros((m, n), dtype=torch.float64, device=DEV)
    rows = torch.arange(n, device=DEV) // 128
    for i in range(sa.shape[1]):
        c = slice(128 * i, min(k, 128 * i + 128))
        out += (a[:, c].double() @ b[:, c].double().t()) * sa[:, i, None].double() * sb[rows, i].double()
    return out


def magnitude64(a, sa, b, sb):
    """Sum of the products' magnitudes: what fp32 summation errors scale with."""
    return product64(a.float().abs().to(F8), sa, b.float().abs().to(F8), sb)


MS = [1, 2, 15, 16, 17, 31, 32, 33, 45, 63, 64, 65, 127, 128, 129, 200, 300]
NK = [(1, 1), (128, 128), (129, 16), (64, 127), (130, 129), (256, 512), (257, 1000), (1000, 2304), (384, 4100)]


@pytest.mark.parametrize("n,k", NK)
def test_product_against_float64(n, k):
    """bf16 rounding: 2^-9 of the value; fp32 sums of k products: at most a few 2^-23 of the sum of their magnitudes
    per block of 128 and per block (the tensor core's own sums keep at least 2^-21 of a block's magnitudes)."""
    for m in MS:
        a, sa, b, sb = operands(m, n, k, 7 * m + n + k, pad=m % 2)
        cflat, out = store(m, n, n + m % 3, m % 2, torch.bfloat16, 7.0)
        api.asap_moe_fp8_matmul(a, sa, b, sb, out)
        ref = product64(a, sa, b, sb)
        bound = ref.abs() * 2.0 ** -8 + magnitude64(a, sa, b, sb) * (2.0 ** -20 + sa.shape[1] * 2.0 ** -22)
        assert ((out.double() - ref).abs() <= bound).all(), m
        rel = float((out.double() - ref).norm() / ref.norm())
        assert rel <= 2.0 ** -8, (m, rel)
        again = torch.empty_like(out)
        api.asap_moe_fp8_matmul(a, sa, b, sb, again)
        assert torch.equal(out.contiguous(), again)
        out.fill_(7.0)
        assert (cflat == 7.0).all()  # nothing beside the rows is written


@pytest.mark.parametrize("m,n,k", [(1, 4096, 7168), (40, 14336, 4096), (500, 4096, 2048), (1500, 2050, 3000),
                                   (4, 640, 65536), (3000, 128, 128), (20000, 8, 256)])
def test_larger_products(m, n, k):
    a, sa, b, sb = operands(m, n, k, m)
    out = torch.full((m, n), 7.0, dtype=torch.bfloat16, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    api.asap_moe_fp8_matmul(a, sa, b, sb, out, status=status)
    ref = product64(a, sa, b, sb)
    rel = float((out.double() - ref).norm() / ref.norm())
    assert rel <= 2.0 ** -8 and int(status) == 0, rel


@pytest.mark.parametrize("m", [1, 40, 150])
def test_rows_and_columns_that_are_no_numbers_stay_alone(m):
    a, sa, b, sb = operands(m + 2, 300, 700, 5)
    out = torch.empty((m + 2, 300), dtype=torch.bfloat16, device=DEV)
    api.asap_moe_fp8_matmul(a, sa, b, sb, out)
    clean = out.clone()
    a.view(torch.uint8)[1, 699] = 0x7F   # NaN
    b.view(torch.uint8)[200, 5] = 0xFF
    sa[0, 3] = math.inf
    api.asap_moe_fp8_matmul(a, sa, b, sb, out)
    assert out[1].isnan().all() and out[:, 200].isnan().all()
    rows = [i for i in range(m + 2) if i > 1]
    cols = [j for j in range(300) if j != 200]
    assert torch.equal(out[rows][:, cols], clean[rows][:, cols])
    assert not out[0, cols].isfinite().any()


def test_exact_small_integers():
    """Products of small whole numbers are exact at every size, so the order of summation cannot hide a misplaced term."""
    for m in (1, 16, 33, 64, 65, 130):
        for n, k in ((200, 300), (513, 1290)):
            g = gen(m + n)
            a = torch.zeros((m, -(-k // 16) * 16), device=DEV)
            b = torch.zeros((n, a.shape[1]), device=DEV)
            a[:, :k] = torch.randint(-1, 2, (m, k), generator=g, device=DEV).float()
            b[:, :k] = torch.randint(-1, 2, (n, k), generator=g, device=DEV).float()
            nb = -(-k // 128)
            sa = 2.0 ** torch.randint(0, 2, (m, nb), generator=g, device=DEV).float()
            sb = 2.0 ** torch.randint(0, 2, (-(-n // 128), nb), generator=g, device=DEV).float()
            out = torch.empty((m, n), dtype=torch.bfloat16, device=DEV)
            api.asap_moe_fp8_matmul(a.to(F8)[:, :k], sa, b.to(F8)[:, :k], sb, out)
            ref = product64(a[:, :k], sa, b[:, :k], sb)
            assert torch.equal(out, ref.bfloat16())


def test_streams_and_graph():
    ops = [operands(m, 700, 1500, m) for m in (1, 20, 64, 300)]
    outs = [torch.empty((o[0].shape[0], 700), dtype=torch.bfloat16, device=DEV) for o in ops]
    want = []
    for o, out in zip(ops, outs):
        api.asap_moe_fp8_matmul(*o, out)
        want.append(out.clone())
    streams = [torch.cuda.Stream() for _ in ops]
    torch.cuda.synchronize()
    for out in outs:
        out.fill_(7.0)
    torch.cuda.synchronize()
    for _ in range(4):
        for o, out, s in zip(ops, outs, streams):
            api.asap_moe_fp8_matmul(*o, out, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    x = randn((45, 1500), 3).bfloat16()
    q = torch.empty((45, 1504), dtype=F8, device=DEV)[:, :1500]
    s = torch.empty((45, 12), device=DEV)
    out = torch.empty((45, 700), dtype=torch.bfloat16, device=DEV)
    _, _, b, sb = ops[0]

    def chain():
        api.asap_moe_fp8_quantize(x, q, s)
        api.asap_moe_fp8_matmul(q, s, b, sb, out)

    chain()
    ref = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        chain()
        chain()
    for t in (q.view(torch.uint8), s, out):
        t.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


def test_empty_extents_do_nothing():
    e = dict(device=DEV)
    api.asap_moe_fp8_quantize(torch.empty((0, 64), dtype=torch.bfloat16, **e), torch.empty((0, 64), dtype=F8, **e),
                              torch.empty((0, 1), **e))
    api.asap_moe_fp8_quantize(torch.empty((4, 0), dtype=torch.bfloat16, **e), torch.empty((4, 0), dtype=F8, **e),
                              torch.empty((4, 0), **e))
    a, sa, b, sb = operands(3, 5, 32, 1)
    api.asap_moe_fp8_matmul(a[:0], sa[:0], b, sb, torch.empty((0, 5), dtype=torch.bfloat16, **e))
    api.asap_moe_fp8_matmul(a, sa, b[:0], sb[:0], torch.empty((3, 0), dtype=torch.bfloat16, **e))


def test_refusals():
    a, sa, b, sb = operands(20, 30, 200, 1)
    out = torch.full((20, 30), 7.0, dtype=torch.bfloat16, device=DEV)
    mm = api.asap_moe_fp8_matmul
    for bad in [(a.float(), sa, b, sb, out), (a, sa.double(), b, sb, out), (a, sa[:, :1], b, sb, out),
                (a, sa, b[:, :100], sb, out), (a, sa, b, sb, out.float()), (a, sa, b, sb, out[:, :20]),
                (a.cpu(), sa, b, sb, out), (a[0], sa, b, sb, out), (a, sa, b, sb, out.t().contiguous().t()),
                (a, sa[:1].expand(20, -1), b, sb, out)]:
        with pytest.raises((ValueError, _native.AsapError)):
            mm(*bad)
    flat = torch.zeros(20 * 208 + 64, dtype=torch.uint8, device=DEV)
    for ld, off in ((200, 0), (208, 8)):  # rows off the 16-byte grid
        with pytest.raises(_native.AsapError) as e:
            mm(view(flat, 20, 200, ld, off).view(F8), sa, b, sb, out)
        assert e.value.code == _native.ASAP_ERR_INVALID and "16-byte" in str(e.value)
    x = torch.zeros((4, 300), dtype=torch.bfloat16, device=DEV)
    q, s = torch.empty((4, 300), dtype=F8, device=DEV), torch.empty((4, 3), device=DEV)
    for bad in [(x.float(), q, s), (x, q[:, :200], s), (x, q, s[:, :2]), (x, q.float(), s), (x.t(), q.t(), s),
                (x[:1].expand(4, -1), q, s)]:
        with pytest.raises((ValueError, _native.AsapError)):
            api.asap_moe_fp8_quantize(*bad)
    wide = torch.zeros((4, 700), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        api.asap_moe_fp8_swiglu_quantize(x, wide[:, :300], q, s)
    L = _native.lib()
    assert L.asap_moe_fp8_matmul(None, 16, None, 1, None, 16, None, 1, None, 1, 1, 1, 1, None, None) == \
        _native.ASAP_ERR_INVALID
    assert L.asap_moe_fp8_quantize(None, 1, 1, 1, None, 1, None, 1, None) == _native.ASAP_ERR_INVALID
    torch.cuda.synchronize()
    assert (out == 7.0).all()
