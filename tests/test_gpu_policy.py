"""The policy's operators on the GPU against float64 references: values, gradients, edges, streams, graphs, the run together."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2108_13976_amd as wd
from paper_2108_13976_amd import policy

import policy_refs as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS24 = 2.0 ** -24


def generator(*key):
    return torch.Generator().manual_seed(sum(k * 7919 ** i for i, k in enumerate(key)) % (1 << 31))


def normal(gen, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype).to(DEV)


# ---- norm ---------------------------------------------------------------------------------------
def check_norm(x, weight, residual, eps, out, out8):
    """Float32 errors: a sum of `width` squares in chains of at most width / 4 adds and 16 levels, halved by the root; four
    more operations on the way to y (product with rstd, with the weight, the root, the quotient)."""
    width = x.shape[1]
    h, y, rstd = ref.norm(x, weight, residual, eps)
    rel = ((width / 4 + 16) / 2 + 6) * EPS24
    assert torch.equal(out.h.cpu(), h), "h"
    assert ((ref.f64(out.rstd) - rstd).abs() <= rel * rstd).all(), "rstd"
    if out.y is not None:
        assert ((ref.f64(out.y) - y).abs() <= rel * y.abs() + ref.rounding(y * (1 + rel), x.dtype) + 1e-38).all(), "y"
    if out8 is None:
        assert out.q is None and out.scale is None
        return
    scale = torch.stack([b.abs().amax(1) for b in ref.blocks_of(y)], 1).clamp(min=ref.TINY) / ref.LARGEST[out8]
    assert ((ref.f64(out.scale) - scale).abs() <= (rel + 3 * EPS24) * scale).all(), "scale"
    z = y / scale.repeat_interleave(128, 1)[:, :width]
    off = (out.q.cpu().float().double() - z).abs()
    assert (off <= ref.rounding(z, out8) * (1 + 1e-6) + 2 * (rel + 4 * EPS24) * z.abs()).all(), "q"


WIDTHS = [1, 5, 8, 21, 32, 33, 64, 65, 127, 128, 129, 200, 256, 257, 511, 512, 777, 1000, 1024, 1025, 2048, 2049, 2999, 4096, 5001, 8192, 8193, 16384, 16385, 32768]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("width", WIDTHS)
def test_norm_against_float64(width, dtype):
    gen = generator(width, 3)
    for rows, with_residual, out8, weight_dtype in ((1, True, E4M3, F32), (3, False, None, dtype), (71, True, E5M2, dtype)):
        x, r = normal(gen, rows, width, dtype=dtype), normal(gen, rows, width, dtype=dtype, scale=2.0) if with_residual else None
        w = (1 + 0.2 * torch.randn(width, generator=gen)).to(weight_dtype).to(DEV)
        out = wd.rms_norm(x, w, residual=r, eps=1e-5, out8=out8, y=True)
        check_norm(x, w, r, 1e-5, out, out8)


@pytest.mark.parametrize("rows,width", [(20011, 21), (9001, 256), (2500, 999), (700, 3000)])
def test_norm_of_more_rows_than_a_launch_holds_at_once(rows, width):
    gen = generator(rows, width)
    x, r = normal(gen, rows, width, dtype=BF16), normal(gen, rows, width, dtype=BF16)
    check_norm(x, None, r, 1e-6, wd.rms_norm(x, None, residual=r, eps=1e-6, out8=E4M3), E4M3)


def test_norm_of_rows_that_are_zero_tiny_large_or_not_finite():
    gen = generator(1, 2)
    for width in (40, 300, 2100):
        x = normal(gen, 8, width)
        x[0] = 0
        x[1] *= 1e-30   # below the least maximum of a block once weighted, with eps 0 brought back to one
        x[2] *= 1e15
        x[3, 7] = float("nan")
        x[4, 7] = float("inf")
        x[5, :30] = 0
        w = torch.ones(width, device=DEV)
        out = wd.rms_norm(x, w, eps=1e-5, out8=E4M3, y=True)
        fine = [0, 1, 2, 5, 6, 7]
        pick = wd.NormOut(out.h[fine], out.y[fine], out.q[fine], out.scale[fine], out.rstd[fine])
        check_norm(x[fine], w, None, 1e-5, pick, E4M3)
        assert out.q[0].float().abs().max() == 0 and out.scale[0].isfinite().all()
        assert out.y[3].isnan().all() and out.q[3].float().isnan().all() and out.rstd[3].isnan()
        bad = torch.zeros(width, dtype=torch.bool)
        bad[7] = True
        assert torch.equal(out.y[4].isnan().cpu(), bad) and torch.equal(out.q[4].float().isnan().cpu(), bad)
        assert (out.y[4][~bad.to(DEV)] == 0).all() and out.rstd[4] == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width,pitch,offset", [(21, 24, 0), (21, 23, 1), (256, 264, 0), (255, 261, 3), (1500, 1503, 1), (5000, 5003, 1)])
def test_norm_of_strided_rows_in_place_and_what_lies_beside_them(width, pitch, offset, dtype):
    gen = generator(width, pitch, offset)
    rows = 37
    store_x, store_r = normal(gen, rows + 2, pitch + offset, dtype=dtype), normal(gen, rows + 2, pitch + offset, dtype=dtype)
    x, r = store_x[1:-1, offset:offset + width], store_r[1:-1, offset:offset + width]
    before, kept, x0, r0 = store_r.clone(), store_x.clone(), x.clone(), r.clone()
    out = wd.rms_norm(x, None, residual=r, h=r, out8=E4M3, y=True)
    check_norm(x0, None, r0, 1e-5, out, E4M3)
    assert out.h.data_ptr() == r.data_ptr() and torch.equal(store_x, kept)
    before[1:-1, offset:offset + width] = r
    assert torch.equal(store_r, before)


def raw_norm(rows, width, dtype_code, **over):
    cfg = policy.wdp_norm_config(ctypes.sizeof(policy.wdp_norm_config), dtype_code, policy.WDP_F32, policy.WDP_E4M3, rows, width, 1e-5,
                                 width, width, width, width, width, -(-width // 128), 1, width, width, width, torch.cuda.current_stream().cuda_stream)
    for n, v in over.items():
        setattr(cfg, n, v)
    return cfg


def test_norm_writes_nothing_beyond_its_outputs():
    rows, width = 13, 77
    gen = generator(5)
    x = normal(gen, rows, width, dtype=BF16)
    guard = 64
    q = torch.full((rows * 96 + guard,), 0x55, dtype=torch.uint8, device=DEV)
    scale, rstd = torch.full((rows * 3 + guard,), 7.0, device=DEV), torch.full((rows + guard,), 7.0, device=DEV)
    y = torch.full((rows * 80 + guard,), 7.0, dtype=BF16, device=DEV)
    cfg = raw_norm(rows, width, policy.WDP_BF16, q_stride=96, scale_row_stride=3, y_stride=80)
    wd.wdp_norm(cfg, policy.wdp_norm_buffers(x.data_ptr(), None, None, None, y.data_ptr(), q.data_ptr(), scale.data_ptr(), rstd.data_ptr()))
    torch.cuda.synchronize()
    assert (q[:rows * 96].view(rows, 96)[:, width:] == 0x55).all() and (q[rows * 96:] == 0x55).all()
    assert (scale[:rows * 3].view(rows, 3)[:, 1:] == 7).all() and (scale[rows * 3:] == 7).all() and (rstd[rows:] == 7).all()
    assert (y[:rows * 80].view(rows, 80)[:, width:] == 7).all() and (y[rows * 80:] == 7).all()
    check_norm(x, None, None, 1e-5, wd.NormOut(x, y[:rows * 80].view(rows, 80)[:, :width], q[:rows * 96].view(rows, 96)[:, :width].view(E4M3),
                                               scale[:rows * 3].view(rows, 3)[:, :1], rstd[:rows]), E4M3)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,width", [(1, 1), (2, 5), (50, 21), (300, 64), (1000, 100), (77, 256), (4500, 256), (33, 333), (2600, 999), (40, 1024), (9, 2048),
                                        (600, 2999), (3, 8192), (700, 5000), (5, 16385), (2, 32768)])
def test_norm_gradients_against_float64(rows, width, dtype):
    """dx: the mean of width products in chains of at most width / 4 adds and 16 levels, a handful of operations more; dw: rows
    products (two operations each), chains of at most rows adds."""
    gen = generator(rows, width)
    h, dy, dh = (normal(gen, rows, width, dtype=dtype, scale=s) for s in (2.0, 1.0, 0.5))
    w = 1 + 0.2 * normal(gen, width)
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-5)
    for extra, weight in ((dh, w), (None, w.to(dtype)), (None, None)):
        dx, dw = wd.rms_norm_backward(dy, h, weight, rstd, dh=extra)
        want_dx, want_dw, size_dx, size_dw = ref.norm_backward(dy, h, weight, rstd, extra)
        assert ((ref.f64(dx) - want_dx).abs() <= (width / 4 + 24) * EPS24 * size_dx + ref.rounding(want_dx, dtype) * 1.01 + 1e-30).all(), "dx"
        assert ((ref.f64(dw) - want_dw).abs() <= (rows + 40) * EPS24 * size_dw + 1e-30).all(), "dw"
        again_dx, again_dw = wd.rms_norm_backward(dy, h, weight, rstd, dh=extra)
        assert torch.equal(dx, again_dx) and torch.equal(dw, again_dw), "the same in every run"
        only, none = wd.rms_norm_backward(dy, h, weight, rstd, dh=extra, want_dw=False)
        assert none is None and torch.equal(only, dx)


def test_norm_gradients_against_differences():
    """The loss sum(c * y + d * h) along random directions: central differences of the forward kernel's own float32 outputs.
    Step 2^-6: the third derivative's part is about 2^-12 / 6 of the slope's size, the outputs' rounding 2^-24 / 2^-6 of the
    terms' sizes at each of them (their root sum of squares is far below their sum): 2e-3 of the slope's size covers both."""
    gen = generator(8)
    rows, width, step = 40, 200, 2.0 ** -6
    x, r, c, d = (normal(gen, rows, width) for _ in range(4))
    w = 1 + 0.2 * normal(gen, width)

    def loss(x, r, w):
        out = wd.rms_norm(x, w, residual=r, eps=1e-5)
        return float((ref.f64(out.y) * ref.f64(c) + ref.f64(out.h) * ref.f64(d)).sum())

    out = wd.rms_norm(x, w, residual=r, eps=1e-5)
    dx, dw = wd.rms_norm_backward(c, out.h, w, out.rstd, dh=d)
    for which in range(3):
        to = normal(gen, width) if which == 2 else normal(gen, rows, width)
        args = [x, r, w]
        up, down = list(args), list(args)
        up[which], down[which] = args[which] + step * to, args[which] - step * to
        slope = (loss(*up) - loss(*down)) / (2 * step)
        grad = dw if which == 2 else dx
        size = float((ref.f64(grad) * ref.f64(to)).square().sum().sqrt())
        assert abs(slope - float((ref.f64(grad) * ref.f64(to)).sum())) <= 2e-3 * max(size, 1.0) * 4, which


def test_norm_gradients_in_place_and_strided():
    gen = generator(9)
    rows, width = 50, 130
    store = normal(gen, rows, 160, dtype=BF16)
    h, dy = store[:, 3:133], normal(gen, rows, width, dtype=BF16)
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-5)
    want, dw = wd.rms_norm_backward(dy, h.contiguous(), None, rstd)
    got, dw2 = wd.rms_norm_backward(dy, h, None, rstd)
    assert torch.equal(want, got) and torch.equal(dw, dw2)
    cfg = raw_norm(rows, width, policy.WDP_BF16, h_stride=160)
    wd.wdp_norm_backward(cfg, policy.wdp_norm_grad_buffers(dy.data_ptr(), None, h.data_ptr(), None, rstd.data_ptr(), dy.data_ptr(), None, None))
    assert torch.equal(dy, want)


# ---- product --------------------------------------------------------------------------------------
def operands(gen, m, n, k, a_type=E4M3, b_type=E4M3, by_row=False):
    a, a_scale = wd.quantise8(normal(gen, m, k) * torch.exp(normal(gen, m, 1)), a_type, rows=1)
    b, b_scale = wd.quantise8(normal(gen, n, k), b_type, rows=1 if by_row else 128)
    return a, a_scale, b, b_scale


def check_product(a, a_scale, b, b_scale, by_row, c):
    """A block's 128 products are exact in float32 (8 significant bits).  float32 c: 127 adds in whatever order, each off by a
    step at most (an adder that truncates), then two operations a block with the scales.  16-bit c: each of a block's products
    loses less than 2^-14 of the largest product's power of two, which is no more than 2^-14 (largest a) (largest b); 128 of
    them, and the sum's own 2^-23 are below the bound 128 * 2^-14 (largest a) (largest b) for each block."""
    want, size, cut = ref.product(a, a_scale, b, b_scale, by_row)
    blocks = a_scale.shape[1]
    adder = 2 * 127 * EPS24 * size if c.dtype == F32 else 2.0 ** -14 * cut
    assert ((ref.f64(c) - want).abs() <= adder + (2 * blocks + 4) * EPS24 * size + ref.rounding(want, c.dtype) * 1.01 + 1e-38).all()


SIZES = [(1, 1, 1), (1, 5, 21), (2, 3, 127), (5, 128, 128), (16, 17, 129), (17, 16, 255), (50, 256, 256), (33, 129, 1000), (64, 64, 64), (100, 333, 384),
         (129, 127, 130), (200, 40, 2048), (257, 300, 515), (1000, 5, 64), (1, 4096, 512), (7, 1000, 4096), (16, 130, 16384), (300, 513, 1024), (512, 512, 640),
         (700, 700, 1100), (130, 2000, 400), (2000, 64, 900), (70, 4000, 260), (40, 4000, 2050), (20, 5000, 390)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("a_type,b_type,by_row,dtype", [(E4M3, E4M3, False, BF16), (E5M2, E4M3, True, F32), (E4M3, E5M2, False, F16), (E5M2, E5M2, True, BF16)])
def test_product_against_float64(m, n, k, a_type, b_type, by_row, dtype):
    gen = generator(m, n, k)
    a, a_scale, b, b_scale = operands(gen, m, n, k, a_type, b_type, by_row)
    if dtype == F16:  # within the type's range
        a_scale = a_scale * 0.01
    check_product(a, a_scale, b, b_scale, by_row and n != -(-n // 128), wd.product8(a, a_scale, b, b_scale, dtype=dtype))


@pytest.mark.parametrize("m,n,k,by_row", [(2048, 1024, 512, False), (2100, 1000, 700, False), (4096, 256, 256, False), (5003, 256, 256, False), (3000, 200, 200, True), (1500, 1537, 1100, True),
                                           (16384, 5, 21, False), (16385, 64, 128, False), (20001, 47, 200, True), (16400, 33, 256, False), (17000, 64, 257, False), (2050, 8192, 300, False),
                                           (4097, 4096, 130, False), (4100, 2050, 150, True), (9000, 300, 300, False)])
def test_product_of_many_rows(m, n, k, by_row):
    gen = generator(m, n, k)
    args = operands(gen, m, n, k, by_row=by_row)
    for dtype in (BF16, F32):
        check_product(*args, by_row, wd.product8(*args, dtype=dtype))


@pytest.mark.parametrize("m,n,k", [(3, 40, 100), (40, 200, 300), (300, 260, 520), (2500, 256, 256)])
@pytest.mark.parametrize("pitch_a,pitch_b,pitch_c", [(0, 0, 0), (16, 32, 8), (3, 5, 1), (1, 16, 7)])
def test_product_of_strided_rows_with_anything_behind_them(m, n, k, pitch_a, pitch_b, pitch_c):
    """NaN codes behind the rows and a guard around c."""
    gen = generator(m, n, k, pitch_a)
    a, a_scale, b, b_scale = operands(gen, m, n, k)

    def wide(t, pitch):
        store = torch.full((t.shape[0] + 1, k + pitch), 0x7F, dtype=torch.uint8, device=DEV)
        store[:-1, :k] = t.contiguous().view(torch.uint8)
        return store.view(t.dtype)[:-1, :k]

    c = torch.full((m + 1, n + pitch_c + 1), 3.0, device=DEV)
    by_blocks = torch.empty((a_scale.shape[1], m), device=DEV).t()
    by_blocks.copy_(a_scale)
    wd.product8(wide(a, pitch_a), by_blocks, wide(b, pitch_b), b_scale, out=c[:m, :n])
    check_product(a, a_scale, b, b_scale, False, c[:m, :n])
    assert (c[m:] == 3).all() and (c[:, n:] == 3).all()


def test_product_of_codes_that_are_not_finite():
    gen = generator(77)
    for m, n, k in ((4, 20, 300), (200, 300, 300), (2200, 256, 256)):
        a, a_scale, b, b_scale = operands(gen, m, n, k)
        fine = wd.product8(a, a_scale, b, b_scale, dtype=F32)
        a.view(torch.uint8)[m // 2, 200] = 0x7F
        b.view(torch.uint8)[n // 3, 250] = 0xFF
        a_scale[1, 0] = float("inf")
        got = wd.product8(a, a_scale, b, b_scale, dtype=F32)
        assert got[m // 2].isnan().all() and got[:, n // 3].isnan().all() and not got[1].isfinite().any()
        rows, cols = torch.ones(m, dtype=torch.bool, device=DEV), torch.ones(n, dtype=torch.bool, device=DEV)
        rows[[1, m // 2]], cols[n // 3] = False, False
        assert torch.equal(got[rows][:, cols], fine[rows][:, cols])


def test_product_of_one_large_and_many_small_terms():
    """float32 c adds what the 8-bit adder of a 16-bit c would cut: 448 * 448 and 127 products of 1/16 each, in every kernel."""
    for m, n, k in ((4, 40, 128), (300, 300, 128), (2000, 256, 256), (17000, 64, 128), (64, 64, 256)):
        a, b = torch.full((m, k), 0.25, device=DEV), torch.full((n, k), 0.25, device=DEV)
        a[:, ::128], b[:, ::128] = 448.0, 448.0
        args = a.to(E4M3), torch.ones((m, k // 128), device=DEV), b.to(E4M3), torch.ones((-(-n // 128), k // 128), device=DEV)
        assert (wd.product8(*args, dtype=F32) == k // 128 * (448.0 * 448 + 127 / 16)).all()
        check_product(*args, False, wd.product8(*args))


def test_product_of_infinite_e5m2_codes():
    a, a_scale = torch.ones((3, 130), device=DEV).to(E5M2), torch.ones((3, 2), device=DEV)
    b, b_scale = torch.ones((5, 130), device=DEV).to(E4M3), torch.ones((1, 2), device=DEV)
    a[1, 129] = float("inf")
    c = wd.product8(a, a_scale, b, b_scale, dtype=F32)
    assert (c[1] == float("inf")).all() and (c[[0, 2]] == 130).all()


def test_product_gives_the_same_in_every_run():
    gen = generator(4)
    for m, n, k in ((8, 512, 8192), (1000, 300, 700), (4096, 512, 512)):
        args = operands(gen, m, n, k)
        first = wd.product8(*args)
        for _ in range(3):
            assert torch.equal(first, wd.product8(*args))


# ---- verification ------------------------------------------------------------------------------------
def drafts_of(gen, batch, n, vocab, bonus, dtype=F32, near=0.7):
    logits = 2 * torch.randn((batch, n + bonus, vocab), generator=gen)
    p = torch.softmax(logits, -1).to(dtype)
    q = torch.softmax(logits[:, :n] + near * torch.randn((batch, n, vocab), generator=gen), -1).to(dtype)
    x = torch.multinomial(q.float().view(-1, vocab) + 1e-30, 1, generator=gen).view(batch, n).int() if n else torch.zeros((batch, 0), dtype=torch.int32)
    u = torch.randint(0, 1 << 24, (batch, n + 1), generator=gen).float() / (1 << 24)
    return [t.to(DEV) for t in (p, q, x, u)]


def check_verify(p, q, x, u, lengths=None, **how):
    accepted, tokens = wd.verify_drafts(p, q, x, u, lengths=lengths, **how)
    want_accepted, want_tokens = ref.verify(p, q, x, u, lengths)
    assert np.array_equal(accepted.cpu().numpy(), want_accepted)
    assert np.array_equal(tokens.cpu().numpy(), want_tokens)
    return accepted, tokens


VERIFY = [(1, 1, 1), (700, 1, 5), (257, 3, 5), (64, 8, 2), (33, 2, 16), (40, 4, 17), (21, 1, 100), (9, 3, 1000), (5, 64, 64), (30, 3, 128), (30, 3, 129), (30, 2, 255), (30, 2, 256), (12, 2, 257), (40, 20, 65), (12, 2, 1023), (12, 2, 1024), (7, 3, 1025),
          (6, 4, 4095), (6, 4, 4096), (5, 3, 4097), (4, 2, 8192), (3, 5, 9999), (2, 1, 50000), (1, 2, 131073)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("batch,n,vocab", VERIFY)
def test_verify_against_the_definition(batch, n, vocab, dtype):
    gen = generator(batch, n, vocab)
    for bonus in (0, 1):
        args = drafts_of(gen, batch, n, vocab, bonus, dtype)
        check_verify(*args)
        lengths = torch.randint(-1, n + 2, (batch,), generator=gen, dtype=torch.int32).to(DEV)
        check_verify(*args, lengths=lengths)


@pytest.mark.parametrize("vocab", [5, 16, 17, 300, 3000, 10000])
def test_verify_edges(vocab):
    """Everything accepted, everything refused, no probability left, tokens out of range, numbers at the ends."""
    gen = generator(vocab)
    batch, n = 12, 3
    p, q, x, u = drafts_of(gen, batch, n, vocab, 1)
    u[:, :] = 0.0
    check_verify(p, q, x, u)                       # accepted as long as p(x) > 0; the draw is the first with r > 0
    u[:, :] = 1.0 - 2.0 ** -24
    check_verify(p, q, x, u)
    check_verify(q[:, [0, 1, 2, 2]].clone(), q, x, u)  # p = q: u < 1 accepts everything
    p2 = p.clone()
    p2[:, 0] = 0.5 * q[:, 0]                       # refused at 0 with nothing left of p - q: a draw from p
    check_verify(p2, q, x, u)
    p2[:, 0] = 0.0                                 # and with p empty: the last token
    _, tokens = check_verify(p2, q, x, u)
    assert (tokens[:, 0] == vocab - 1).all()
    p3 = torch.zeros_like(p)
    p3[:, :, vocab // 2] = 1.0                     # all on one token
    _, tokens = check_verify(p3, q, x, u)
    x2 = x.clone()
    x2[0], x2[1], x2[2, 1], x2[3] = -1, vocab, 1 << 30, -(1 << 31)
    u = torch.rand((batch, n + 1), generator=gen).to(DEV)
    accepted, _ = check_verify(p, q, x2, u)
    assert accepted[0] == 0 and accepted[1] == 0 and accepted[2] <= 1 and accepted[3] == 0
    check_verify(p * 3.7, q * 0.2, x, u)           # not normalised
    p4, q4 = p.clone(), q.clone()
    p4[:, :, 1], q4[:, :, 2], p4[:, 1, 3] = float("nan"), float("nan"), -1.0
    check_verify(p4, q4, x, u)
    u[::2, 1] = float("nan")
    u[1::2, n] = float("nan")
    check_verify(p, q, x, u)


@pytest.mark.parametrize("vocab", [5, 200, 2000, 9000])
def test_verify_with_infinite_probabilities(vocab):
    gen = generator(vocab, 1)
    p, q, x, u = drafts_of(gen, 8, 2, vocab, 1)
    p[::2, :, vocab // 3] = float("inf")
    check_verify(p, q, x, u)


def test_verify_without_drafts_is_a_draw():
    gen = generator(3)
    for vocab in (5, 500, 7000):
        p, q, x, u = drafts_of(gen, 30, 0, vocab, 1)
        accepted, tokens = check_verify(p, q, x, u)
        assert (accepted == 0).all() and (tokens >= 0).all()


def test_verify_in_place_strided_and_many_sequences():
    gen = generator(6)
    p, q, x, u = drafts_of(gen, 70001, 1, 5, 0)
    drafted = x.clone()
    accepted, tokens = wd.verify_drafts(p, q, x, u, tokens=x)
    want_accepted, want_tokens = ref.verify(p, q, drafted, u)
    assert tokens.data_ptr() == x.data_ptr() and np.array_equal(x.cpu().numpy(), want_tokens) and np.array_equal(accepted.cpu().numpy(), want_accepted)
    for vocab in (5, 600, 5000):
        p, q, x, u = drafts_of(gen, 9, 3, vocab, 1)
        wide_p, wide_q = torch.full((9, 5, vocab + 3), float("nan"), device=DEV), torch.full((9, 4, vocab + 1), float("nan"), device=DEV)
        wide_p[:, :4, 1:vocab + 1], wide_q[:, :3, :vocab] = p, q
        check_verify(wide_p[:, :4, 1:vocab + 1], wide_q[:, :3, :vocab], x, u)
        first = p[:1].expand(9, -1, -1)  # one target for all sequences: a batch stride of zero
        check_verify(first, q, x, u)


def test_verified_drafts_are_draws_from_the_target():
    """Chi-square over 200 000 sequences, whatever q is: 4 degrees of freedom, 33.4 is passed with probability 1e-6."""
    gen = generator(12)
    batch = 200000
    p = torch.tensor([0.05, 0.4, 0.25, 0.2, 0.1])
    for q in (torch.tensor([0.3, 0.1, 0.2, 0.2, 0.2]), torch.tensor([0.96, 0.01, 0.01, 0.01, 0.01]), p.clone()):
        x = torch.multinomial(q, batch, replacement=True, generator=gen).int().view(-1, 1)
        u = torch.rand((batch, 2), generator=gen)
        _, tokens = wd.verify_drafts(p.to(DEV).expand(batch, 1, 5), q.to(DEV).expand(batch, 1, 5), x.to(DEV), u.to(DEV))
        counts = torch.bincount(tokens[:, 0].long().cpu(), minlength=5).double()
        assert float(((counts - batch * p.double()) ** 2 / (batch * p.double())).sum()) < 33.4


# ---- AdamW ------------------------------------------------------------------------------------------
HYPER = dict(lr=3e-4, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)
NUMELS = [1, 5, 7, 8, 100, 127, 128, 129, 1000, 2048, 2049, 5000, 0, 64]


def tensors_of(gen, sizes, dtype, grad_dtype=None, scale=0.05):
    params = [normal(gen, n, dtype=dtype, scale=scale) for n in sizes]
    grads = [normal(gen, n, dtype=grad_dtype or dtype, scale=0.01) for n in sizes]
    return params, grads


def near(got, want, steps, scale=None):
    """Within `steps` float32 roundings of the terms' size."""
    return ((ref.f64(got) - want).abs() <= steps * EPS24 * (want.abs() if scale is None else scale) + 1e-36).all()


@pytest.mark.parametrize("dtype,grad_dtype,with_master", [(F32, F32, False), (BF16, BF16, True), (BF16, F32, True), (F16, F16, False), (BF16, BF16, False), (F16, F32, True)])
def test_adamw_against_float64_over_three_steps(dtype, grad_dtype, with_master):
    """From the state that stands before each step: m, v are three operations each (of terms no larger than their sizes added),
    p eight more on the update, whose size is lr times a quotient."""
    gen = generator(21)
    params, grads = tensors_of(gen, NUMELS, dtype, grad_dtype)
    masters = [p.float() for p in params] if with_master else None
    opt = wd.AdamW(params, grads, masters=masters, **HYPER)
    for step in (1, 2, 3):
        for g in grads:
            g.copy_(torch.randn(g.shape, generator=gen) * 0.01)
        before = [(ref.f64(masters[i] if with_master else params[i]), ref.f64(grads[i]), ref.f64(opt.exp_avg[i]), ref.f64(opt.exp_avg_sq[i])) for i in range(len(params))]
        opt.step()
        for i, (p, g, m, v) in enumerate(before):
            want_p, want_m, want_v = ref.adamw(p, g, m, v, step, **{"lr": HYPER["lr"], "betas": HYPER["betas"], "eps": HYPER["eps"], "decay": HYPER["weight_decay"]})
            assert near(opt.exp_avg[i], want_m, 4, 0.9 * m.abs() + 0.1 * g.abs()), ("m", step, i)
            assert near(opt.exp_avg_sq[i], want_v, 6), ("v", step, i)
            # the quotient's relative error: m's absolute one over its size included
            moved = (want_p - p).abs() + HYPER["lr"] * 2 * (0.9 * m.abs() + 0.1 * g.abs()) / (1 - 0.9 ** step) / (torch.sqrt(want_v / (1 - 0.999 ** step)) + 1e-8)
            allowed = 4 * EPS24 * p.abs() + 16 * EPS24 * moved + 1e-36
            if with_master:
                assert ((ref.f64(masters[i]) - want_p).abs() <= allowed).all(), ("master", step, i)
                assert torch.equal(params[i], masters[i].to(dtype))
            else:
                assert ((ref.f64(params[i]) - want_p).abs() <= allowed + (ref.rounding(want_p, dtype) * 1.01 if dtype != F32 else 0)).all(), ("p", step, i)
    assert opt.steps == 3


def test_adamw_of_more_tensors_than_a_launch_takes_and_of_mixed_types():
    gen = generator(22)
    sizes = [(37 * i) % 301 for i in range(130)]
    params = [normal(gen, n, dtype=(F32, BF16, BF16, F16)[i // 20 % 4], scale=0.05) for i, n in enumerate(sizes)]
    grads = [normal(gen, n, dtype=p.dtype if i % 7 else F32, scale=0.01) for i, (n, p) in enumerate(zip(sizes, params))]
    masters = [p.float() for p in params]
    for bits in (32, 8):
        a = wd.AdamW([p.clone() for p in params], grads, masters=[m.clone() for m in masters], state_bits=bits, seed=5, **HYPER)
        a.step()
        for i in range(len(params)):
            want, m, v = ref.adamw(ref.f64(masters[i]), ref.f64(grads[i]), 0.0, 0.0, 1, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
            assert ((ref.f64(a.masters[i]) - want).abs() <= 4 * EPS24 * ref.f64(masters[i]).abs() + 20 * EPS24 * HYPER["lr"]).all(), i


def test_adamw_leaves_what_lies_between_the_tensors():
    gen = generator(23)
    for bits in (32, 8):
        store = {n: torch.full((4000,), 0.25, device=DEV) for n in ("p", "g", "m", "v")}
        spans = [(1, 130), (131, 7), (140, 2050), (2300, 1000)]
        views = {n: [t[a:a + k] for a, k in spans] for n, t in store.items()}
        if bits == 8:
            eight = {n: torch.full((4000,), 0x38, dtype=torch.uint8, device=DEV).view(E4M3) for n in ("m", "v")}
            views.update({n: [t[a:a + k] for a, k in spans] for n, t in eight.items()})
            scales = {n: torch.full((64,), 0.25, device=DEV) for n in ("a", "s")}
            views.update({n: [t[i * 18:i * 18 + -(-k // 128)] for i, (_, k) in enumerate(spans)] for n, t in scales.items()})
        opt = wd.AdamW(views["p"], views["g"], state_bits=bits, exp_avg=views["m"], exp_avg_sq=views["v"],
                       avg_scale=views["a"] if bits == 8 else None, sq_scale=views["s"] if bits == 8 else None, **HYPER)
        opt.step()
        inside = torch.zeros(4000, dtype=torch.bool, device=DEV)
        for a, k in spans:
            inside[a:a + k] = True
        assert (store["p"][~inside] == 0.25).all() and (store["p"][inside] != 0.25).all() and (store["g"] == 0.25).all()
        if bits == 32:
            assert (store["v"][~inside] == 0.25).all() and (store["v"][inside] != 0.25).all()
        else:
            assert all((t.view(torch.uint8)[~inside] == 0x38).all() for t in eight.values())
            for t in scales.values():
                assert sum(int(x) for x in t != 0.25) == sum(-(-k // 128) for _, k in spans)


def test_adamw_8_bit_states_are_the_documented_roundings():
    """Each code is where the definition puts it, from the state before the step: units of the code's step plus the random
    fraction, downwards; one apart where that comes within 1e-4 of a whole number (float32: the quotient is off by a few 2^-24
    of at most 16 units, which is below 1e-5)."""
    gen = generator(24)
    sizes = [1000, 3, 128, 517]
    params, grads = tensors_of(gen, sizes, F32)
    opt = wd.AdamW(params, grads, state_bits=8, seed=(7 << 32) + 99, **HYPER)
    for step in (1, 2, 3, (3 << 32) + 5):
        for g in grads:
            g.copy_(torch.randn(g.shape, generator=gen) * torch.exp(3 * torch.randn(g.shape, generator=gen)) * 0.01)
        before = [[ref.f64(t[i].float()) for t in (opt.params, opt.grads, opt.exp_avg, opt.exp_avg_sq)] +
                  [ref.f64(s[i]).repeat_interleave(128)[:n] for s in (opt.avg_scale, opt.sq_scale)] for i, n in enumerate(sizes)]
        opt.step(step=step)
        blocks = 0
        for i, n in enumerate(sizes):
            p, g, m, s, ms, ss = before[i]
            want_p, m, v = ref.adamw(p, g, m * ms, (s * ss) ** 2, step, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
            assert ((ref.f64(opt.params[i]) - want_p).abs() <= 4 * EPS24 * p.abs() + 30 * EPS24 * (want_p - p).abs() + 1e-12).all()
            at = np.arange(n, dtype=np.uint64) + np.uint64(128 * blocks)
            words = ref.philox_words((7 << 32) + 99, at // np.uint64(4), step)[np.arange(n), (at % np.uint64(4)).astype(int)]
            blocks += -(-n // 128)
            for value, codes, scales, bits in ((m, opt.exp_avg[i], opt.avg_scale[i], words & np.uint64(0xFFFF)), (v.sqrt(), opt.exp_avg_sq[i], opt.sq_scale[i], words >> np.uint64(16))):
                want_scale = torch.stack([b.abs().max() for b in value.split(128)]).clamp(min=ref.TINY) / 448
                assert near(scales, want_scale, 12)
                z = value / ref.f64(scales).repeat_interleave(128)[:n]
                units, unit = ref.code_units(z)
                r = torch.from_numpy(bits.astype(np.float64)) / 65536
                low, high = (torch.floor(units + r + d) * unit for d in (-1e-4, 1e-4))
                got = ref.f64(codes.float())
                size = got.abs()
                if value is not m:  # a root above zero stays above it
                    low, high = (torch.where(value > 0, t.clamp(min=2.0 ** -9), t) for t in (low, high))
                assert ((size == low.clamp(max=448)) | (size == high.clamp(max=448))).all()
                assert ((got == 0) | (torch.sign(got) == torch.sign(value))).all()


def test_adamw_8_bit_states_follow_their_means():
    """Gradients of constant size: after 500 steps v is (1 - 0.999^500) g^2 = 0.39 g^2 and m is g.  A code's step is up to 1/8 of
    its value and the roundings of 500 steps average out over 4096 elements: 5 % holds for both means with room; to nearest, v
    would stop where 0.001 / 2 of its root's growth is half a step, below 0.02 g^2."""
    params, grads = [torch.zeros(4096, device=DEV)], [torch.full((4096,), 0.5, device=DEV)]
    opt = wd.AdamW(params, grads, state_bits=8, seed=3, lr=0.0, weight_decay=0.0)
    for _ in range(500):
        opt.step()
    m = opt.exp_avg[0].float().view(-1, 128) * opt.avg_scale[0][:, None]
    s = opt.exp_avg_sq[0].float().view(-1, 128) * opt.sq_scale[0][:, None]
    assert abs(float(m.mean()) / 0.5 - 1) < 0.05 and abs(float((s * s).mean()) / (0.25 * (1 - 0.999 ** 500)) - 1) < 0.1


def test_adamw_with_a_gradient_that_is_not_finite():
    gen = generator(25)
    params, grads = tensors_of(gen, [300, 50], F32)
    grads[0][5], grads[0][200] = float("nan"), float("inf")
    for bits in (32, 8):
        copies = [p.clone() for p in params]
        opt = wd.AdamW(copies, grads, state_bits=bits, **HYPER)
        opt.step()
        bad = ~copies[0].isfinite()
        assert bad[5] and bad[200] and int(bad.sum()) == 2 and copies[1].isfinite().all()
        if bits == 32:
            assert not opt.exp_avg[0][5].isfinite() and int((~opt.exp_avg[0].isfinite()).sum()) == 2
        else:
            assert opt.exp_avg[0].float()[5].isnan() and opt.exp_avg[1].float().isfinite().all()
            assert opt.avg_scale[0][0].isfinite() and opt.avg_scale[0][2].isfinite()


def test_adamw_grad_scale_and_step_on_the_device():
    gen = generator(26)
    params, grads = tensors_of(gen, [700, 30], BF16)
    masters = [p.float() for p in params]
    for bits in (32, 8):
        a = wd.AdamW([p.clone() for p in params], grads, masters=[m.clone() for m in masters], state_bits=bits, **HYPER)
        b = wd.AdamW([p.clone() for p in params], [g.float() * 0.5 for g in grads], masters=[m.clone() for m in masters], state_bits=bits, **HYPER)
        number = torch.zeros(1, dtype=torch.int64, device=DEV)
        for _ in range(3):
            number += 1
            a.step(step_device=number, grad_scale=torch.tensor([0.5], device=DEV))
            b.step()
        for x, y in zip(a.masters, b.masters):
            # the bias corrections come from another pow: a few roundings of updates no larger than 3 lr
            assert ((ref.f64(x) - ref.f64(y)).abs() <= 3 * (3 * HYPER["lr"] * 16 * EPS24 + 2 * EPS24 * ref.f64(y).abs())).all()
        if bits == 32:
            assert all(torch.equal(x, y) for x, y in zip(a.exp_avg, b.exp_avg))


# ---- streams, graphs, all of them together ---------------------------------------------------------
def one_of_each(gen):
    """Calls of every operator on inputs that stay, and a function that runs them and returns what they gave."""
    x, r, w = normal(gen, 60, 200, dtype=BF16), normal(gen, 60, 200, dtype=BF16), 1 + 0.1 * normal(gen, 200)
    b, b_scale = wd.quantise8(normal(gen, 300, 200))
    p, q, d, u = drafts_of(gen, 20, 3, 6000, 1)
    few = drafts_of(gen, 500, 1, 5, 0)
    dy = normal(gen, 60, 200, dtype=BF16)
    wide, wide_scale = wd.quantise8(normal(gen, 256, 4096))
    one, one_scale = wd.quantise8(normal(gen, 4, 4096), rows=1)

    def calls():
        out = wd.rms_norm(x, w, residual=r, out8=E4M3)
        dx, dw = wd.rms_norm_backward(dy, out.h, w, out.rstd)
        return [out.h, out.q.view(torch.uint8), out.scale, out.rstd, dx, dw, wd.product8(out.q, out.scale, b, b_scale), wd.product8(one, one_scale, wide, wide_scale),
                *wd.verify_drafts(p, q, d, u), *wd.verify_drafts(*few)]
    return calls, (x, r, dy, u, few[3])


def test_operators_on_another_stream():
    calls, _ = one_of_each(generator(31))
    want = [t.clone() for t in calls()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = calls()
    both = calls()  # and on two streams at once
    torch.cuda.synchronize()
    for a, b, c in zip(want, got, both):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_operators_in_a_graph_that_is_replayed():
    gen = generator(32)
    calls, changing = one_of_each(gen)
    params, grads = tensors_of(gen, [500, 33], F32)
    number = torch.zeros(1, dtype=torch.int64, device=DEV)
    opt = wd.AdamW([p.clone() for p in params], grads, **HYPER)
    eager = wd.AdamW([p.clone() for p in params], grads, **HYPER)
    calls()
    opt_state = [t for t in opt.params]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin()
        outs = calls()
        number.add_(1)
        opt.step(step_device=number)
        graph.capture_end()
    torch.cuda.current_stream().wait_stream(side)
    for replay in range(4):
        for t in changing[:3]:
            t.copy_((torch.randn(t.shape, generator=gen)).to(t.dtype))
        for t in changing[3:]:
            t.copy_(torch.rand(t.shape, generator=gen))
        grads[0].mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for a, b in zip(got, calls()):
            assert torch.equal(a, b), replay
        eager.step()
        for a, b in zip(opt_state, eager.params):
            assert ((ref.f64(a) - ref.f64(b)).abs() <= (replay + 1) * (3 * HYPER["lr"] * 16 * EPS24 + 2 * EPS24 * ref.f64(b).abs())).all(), replay
        torch.cuda.synchronize()


def test_zero_rows():
    x = torch.empty((0, 40), dtype=BF16, device=DEV)
    out = wd.rms_norm(x, None, residual=x, out8=E4M3)
    assert out.q.shape == (0, 40) and out.scale.shape == (0, 1) and out.h.shape == (0, 40)
    dx, dw = wd.rms_norm_backward(x, x, None, out.rstd)
    assert dx.shape == (0, 40) and (dw == 0).all()
    b, b_scale = wd.quantise8(torch.ones((30, 40), device=DEV))
    assert wd.product8(out.q, out.scale, b, b_scale).shape == (0, 30)
    a, a_scale = wd.quantise8(torch.ones((3, 40), device=DEV), rows=1)
    assert wd.product8(a, a_scale, b[:0], b_scale[:0]).shape == (3, 0)
    p = torch.empty((0, 2, 9), device=DEV)
    accepted, tokens = wd.verify_drafts(p, p[:, :1], torch.empty((0, 1), dtype=torch.int32, device=DEV), torch.empty((0, 2), device=DEV))
    assert accepted.shape == (0,) and tokens.shape == (0, 2)
    wd.AdamW([torch.empty(0, device=DEV)], [torch.empty(0, device=DEV)]).step()


# ---- with the environments -----------------------------------------------------------------------
def tag(gen_seed, E=40, N=24, **over):
    return wd.TagEnvs(**{**dict(num_envs=E, num_agents=N, num_taggers=4, grid_size=12, episode_length=9, seed=gen_seed), **over})


@pytest.mark.parametrize("kind", ["discrete", "continuous"])
@pytest.mark.parametrize("on_a_stream", [False, True])
def test_drafted_actions_are_verified_between_sample_and_step(kind, on_a_stream):
    gen = generator(41)
    stream = torch.cuda.Stream() if on_a_stream else None
    if kind == "discrete":
        envs, twin = tag(3, stream=stream), tag(3)
        shape = (40, 24)
    else:
        envs, twin = (wd.CTagEnvs(num_envs=30, num_agents=12, num_taggers=2, episode_length=9, seed=4, stream=s) for s in (stream, None))
        shape = (30, 12, 2)
    envs.reset(), twin.reset()
    for _ in range(12):
        p, q = (torch.softmax(normal(gen, *shape, 5) * 1.5, -1).contiguous() for _ in range(2))
        u = torch.rand((*shape, 2), generator=gen).to(DEV)
        torch.cuda.synchronize()
        envs.sample(q)
        twin.sample(q)
        kept = envs.verify(p, q, u)
        envs.torch_stream.synchronize()
        draws = twin.action.numel()
        accepted, tokens = ref.verify(p.view(draws, 1, 5), q.view(draws, 1, 5), twin.action.view(draws, 1), u.view(draws, 2))
        assert np.array_equal(kept.cpu().numpy().reshape(-1), accepted.astype(bool))
        assert np.array_equal(envs.action.cpu().numpy().reshape(-1), tokens[:, 0]) and 0 < accepted.mean() < 1
        twin.action.copy_(envs.action)
        torch.cuda.synchronize()
        for e in (envs, twin):
            e.step()
            e.reset(wd.WD_RESET_DONE)
        a, b = envs.to_host(), twin.to_host()
        assert all(np.array_equal(a[n], b[n]) for n in a)
    for bad in (lambda: envs.verify(p[:-1], q, u), lambda: envs.verify(p, q.double(), u), lambda: envs.verify(p, q, u[..., :1]), lambda: envs.verify(p.cpu(), q, u)):
        with pytest.raises(ValueError):
            bad()


def test_a_policy_in_the_loop_and_its_update():
    """Observations through norm, 8-bit products and a residual to probabilities, drafts verified against them, a step; then the
    way back and one step of the optimiser.  Each operator against float64 on what it was given, the weights' gradient through
    the norm against differences of the float64 policy."""
    gen = generator(42)
    envs = tag(5)
    envs.reset()
    rows, width, D = 40 * 24, 96, envs.D
    weights = [normal(gen, width, D, scale=D ** -0.5), normal(gen, width, width, scale=width ** -0.5), normal(gen, 5, width, scale=0.3)]
    norms = [1 + 0.1 * normal(gen, D), 1 + 0.1 * normal(gen, width), 1 + 0.1 * normal(gen, width)]
    eight = [wd.quantise8(w) for w in weights]
    for iteration in range(3):
        x = envs.obs.view(rows, D)
        n0 = wd.rms_norm(x, norms[0], out8=E4M3)
        check_norm(x, norms[0], None, 1e-5, n0, E4M3)
        h0 = wd.product8(n0.q, n0.scale, *eight[0])
        check_product(n0.q, n0.scale, *eight[0], False, h0)
        n1 = wd.rms_norm(h0, norms[1], out8=E4M3)
        check_norm(h0, norms[1], None, 1e-5, n1, E4M3)
        h1 = wd.product8(n1.q, n1.scale, *eight[1])
        n2 = wd.rms_norm(h1, norms[2], residual=h0, out8=E4M3, y=True)
        check_norm(h1, norms[2], h0, 1e-5, n2, E4M3)
        logits = wd.product8(n2.q, n2.scale, *eight[2], dtype=F32)
        check_product(n2.q, n2.scale, *eight[2], False, logits)
        probs = torch.softmax(logits, -1).view(40, 24, 5).contiguous()
        drafts = torch.softmax(logits + 0.5 * normal(gen, rows, 5), -1).view(40, 24, 5).contiguous()
        envs.sample(drafts)
        before = envs.action.clone()
        kept = envs.verify(probs, drafts, torch.rand((40, 24, 2), generator=gen).to(DEV))
        assert torch.equal(envs.action[kept], before[kept]) and int(kept.sum()) > rows // 2
        envs.step()
        envs.reset(wd.WD_RESET_DONE)
    # the loss sum(c * (y of the last norm)), back through the last norm to its weight and both of its inputs
    c = normal(gen, rows, width, dtype=BF16)
    dx, dw = wd.rms_norm_backward(c, n2.h, norms[2], n2.rstd)
    want_dx, want_dw, size_dx, size_dw = ref.norm_backward(c, n2.h, norms[2], n2.rstd, None)
    assert ((ref.f64(dx) - want_dx).abs() <= (width / 4 + 24) * EPS24 * size_dx + ref.rounding(want_dx, BF16) * 1.01).all()
    assert ((ref.f64(dw) - want_dw).abs() <= (rows + 40) * EPS24 * size_dw).all()
    h, to = ref.f64(n2.h), torch.randn(rows, width, generator=gen, dtype=torch.float64)

    def loss(h):
        return float((ref.f64(c) * h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-5) * ref.f64(norms[2])).sum())

    slope, got = (loss(h + 1e-6 * to) - loss(h - 1e-6 * to)) / 2e-6, float((ref.f64(dx) * to).sum())
    assert abs(slope - got) <= 2.0 ** -8 * float((ref.f64(dx) * to).abs().sum()) / rows ** 0.5 + 1e-4 * abs(slope)  # dx is rounded to bfloat16
    params, grads = [norms[2].clone(), weights[2].clone()], [dw, (normal(gen, 5, width) * 0.1)]
    opt = wd.AdamW(params, grads, **HYPER)
    opt.step()
    for p, old, g in zip(params, (norms[2], weights[2]), grads):
        want, _, _ = ref.adamw(ref.f64(old), ref.f64(g), 0.0, 0.0, 1, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
        assert ((ref.f64(p) - want).abs() <= 4 * EPS24 * ref.f64(old).abs() + 20 * EPS24 * HYPER["lr"]).all()


def test_gradients_of_the_8_bit_product_by_the_product_itself():
    """c = a b^T: da = dc b and db = dc^T a are products of the same entry point over the transposed operands, with a scale for
    each row (dc in E5M2); against float64 on the values that were quantised."""
    gen = generator(43)
    m, n, k = 300, 200, 260
    a, b, dc = normal(gen, m, k), normal(gen, n, k), normal(gen, m, n)
    dc8, dc_scale = wd.quantise8(dc, E5M2, rows=1)
    bt8, bt_scale = wd.quantise8(b.t().contiguous(), rows=128)
    da = wd.product8(dc8, dc_scale, bt8, bt_scale, dtype=F32)
    check_product(dc8, dc_scale, bt8, bt_scale, False, da)
    dct8, dct_scale = wd.quantise8(dc.t().contiguous(), E5M2, rows=1)
    at8, at_scale = wd.quantise8(a.t().contiguous(), rows=1)
    db = wd.product8(dct8, dct_scale, at8, at_scale, dtype=F32)
    check_product(dct8, dct_scale, at8, at_scale, True, db)
    # of the exact gradients they are as far as the codes' rounding takes them: half steps of 2^-3 and 2^-4 per term
    for got, want, terms in ((da, ref.f64(dc) @ ref.f64(b), ref.f64(dc).abs() @ ref.f64(b).abs()),
                             (db, ref.f64(dc).t() @ ref.f64(a), ref.f64(dc).abs().t() @ ref.f64(a).abs())):
        assert ((ref.f64(got) - want).abs() <= ((1 + 2.0 ** -3) * (1 + 2.0 ** -4) - 1 + 1e-3) * terms).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [9, 21, 300, 999, 1100, 3001, 4797, 9001, 12001, 16001, 20001])
def test_norm_and_its_gradients_in_place_where_the_row_ends_inside_a_chunk(width, dtype):
    """The row's last chunk overlaps its neighbour's in memory: h over residual, dx over dh and over dy, many rows, twice the same
    as out of place; a value that is not finite among the overlapped ones stays where it is."""
    gen = generator(width, 51)
    rows = 600 if width < 5000 else 300
    x, r, dy, dh = (normal(gen, rows, width, dtype=dtype) for _ in range(4))
    w = 1 + 0.1 * normal(gen, width)
    x[1, width - 3], x[2, max(0, width - 9)] = float("inf"), float("inf")
    want = wd.rms_norm(x, w, residual=r, out8=E4M3, y=True)
    bad = torch.zeros(width, dtype=torch.bool, device=DEV)
    for row, col in ((1, width - 3), (2, max(0, width - 9))):
        bad.zero_()
        bad[col] = True
        assert torch.equal(want.y[row].isnan(), bad) and (want.y[row][~bad] == 0).all()
    h = r.clone()
    got = wd.rms_norm(x, w, residual=h, h=h, out8=E4M3, y=True)
    for a, b in zip(want, got):
        assert torch.equal(a.view(torch.uint8) if a.dtype == E4M3 else torch.nan_to_num(a, nan=7.0), b.view(torch.uint8) if b.dtype == E4M3 else torch.nan_to_num(b, nan=7.0))
    h, rstd = torch.nan_to_num(want.h, posinf=0.5), torch.rsqrt(want.h.float().square().mean(1) + 1e-5)
    dx, dw = wd.rms_norm_backward(dy, h, w, rstd, dh=dh)
    cfg = raw_norm(rows, width, policy.WDP_BF16 if dtype == BF16 else policy.WDP_F32)
    space = torch.empty(wd.wdp_norm_backward_workspace(cfg), dtype=torch.uint8, device=DEV)
    for over_dy in (False, True):
        first, second, dw2 = dy.clone(), dh.clone(), torch.empty_like(dw)
        to = first if over_dy else second
        wd.wdp_norm_backward(cfg, policy.wdp_norm_grad_buffers(first.data_ptr(), second.data_ptr(), h.data_ptr(), w.data_ptr(), rstd.data_ptr(), to.data_ptr(),
                                                               dw2.data_ptr(), space.data_ptr()))
        assert torch.equal(to, dx) and torch.equal(dw2, dw), over_dy


def test_an_earlier_error_of_the_program_is_not_the_operators():
    """A runtime call that failed leaves its status behind (here: a device that does not exist); the operators answer for their own launches."""
    hip = ctypes.CDLL("libamdhip64.so")
    calls, _ = one_of_each(generator(33))
    params, grads = tensors_of(generator(34), [100], F32)
    optimiser = wd.AdamW(params, grads)
    want = [t.clone() for t in calls()]
    torch.cuda.synchronize()
    assert hip.hipSetDevice(4096) != 0
    c = policy.wdp_adamw_config(ctypes.sizeof(policy.wdp_adamw_config), 32, 1e-3, 0.9, 0.999, 1e-8, 0.01, 1, None, None, 0, None)
    wd.wdp_adamw(c, optimiser._table, 1)
    got = calls()
    assert hip.hipGetLastError() != 0  # (still there; torch's own launches would answer with it)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_adamw_refuses_tensors_that_overlap():
    params, grads = tensors_of(generator(35), [300, 300], F32)
    flat = torch.zeros(500, device=DEV)
    for call in (lambda: wd.AdamW([params[0], params[0]], grads), lambda: wd.AdamW([flat[:300], flat[200:]], grads), lambda: wd.AdamW(params, [grads[0], params[0]]),
                 lambda: wd.AdamW(params, grads, exp_avg=[flat[:300], flat[200:]], exp_avg_sq=[torch.zeros(300, device=DEV) for _ in range(2)]),
                 lambda: wd.AdamW(params[:1], grads[:1], masters=params[:1])):
        with pytest.raises(ValueError):
            call()
    wd.AdamW(params, [grads[0], grads[0]]).step()  # (a gradient is read only)
    wd.AdamW([flat[:300], flat[300:]], [grads[0], grads[1][:200]]).step()


def test_adamw_of_one_tensor_beyond_a_launch():
    """2^34 elements and a few: more than one launch's workgroups."""
    many = (1 << 34) + 5000
    if torch.cuda.mem_get_info()[0] < 7 * many:
        pytest.skip("needs 120 GB of free memory")
    param, grad = torch.ones(many, dtype=BF16, device=DEV), torch.full((many,), 0.5, dtype=BF16, device=DEV)
    opt = wd.AdamW([param], [grad], lr=0.25, weight_decay=0.0, state_bits=8)
    opt.step()
    # m = 0.05, s = sqrt(0.001) / 2, the update lr * 1, p = 0.75; scale max / 448, and codes 448, or 416 below it where a quotient
    # that its roundings left just under 448 meets sixteen random zeros
    for at in (0, (1 << 33) - 4096, (1 << 34) - 4096, (1 << 34) - 100, many - 4096):
        part = slice(at, at + 4096)
        assert (param[part] == 0.75).all(), at
        for codes in (opt.exp_avg[0][part].float(), opt.exp_avg_sq[0][part].float()):
            assert ((codes == 448) | (codes == 416)).all() and int((codes == 416).sum()) < 8, at
    for scales, value in ((opt.avg_scale[0], 0.05), (opt.sq_scale[0], 0.5 * 0.001 ** 0.5)):
        low, high = torch.aminmax(scales)
        assert low == high and abs(float(low) * 448 / value - 1) < 1e-5
    del param, grad, opt, part, codes, scales, low, high
    torch.cuda.empty_cache()


@pytest.mark.parametrize("m,n,k,by_row,a_type,b_type,dtype", [
    (3000, 2999, 777, False, E4M3, E4M3, BF16), (2817, 3000, 768, False, E5M2, E4M3, F16), (2900, 2881, 1028, False, E4M3, E5M2, BF16), (3000, 3001, 900, False, E5M2, E5M2, BF16),
    (3000, 2999, 777, True, E4M3, E4M3, BF16), (1500, 1537, 768, True, E5M2, E4M3, F16), (1601, 1500, 1028, True, E4M3, E5M2, BF16), (1500, 1600, 641, True, E5M2, E5M2, BF16)])
def test_product_of_many_blocks_of_k(m, n, k, by_row, a_type, b_type, dtype):
    """Odd and even counts of blocks, ends inside a chunk and at one, NaN codes behind the rows, a guard around c."""
    gen = generator(m, n, k)
    a, a_scale, b, b_scale = operands(gen, m, n, k, a_type, b_type, by_row)
    if dtype == F16:
        a_scale = a_scale * 0.01

    def wide(t):
        store = torch.full((t.shape[0] + 1, -(-k // 16) * 16 + 32), 0x7F, dtype=torch.uint8, device=DEV)
        store[:-1, :k] = t.contiguous().view(torch.uint8)
        return store.view(t.dtype)[:-1, :k]

    c = torch.full((m + 1, n + 9), 3.0, device=DEV, dtype=dtype)
    wd.product8(wide(a), a_scale, wide(b), b_scale, out=c[:m, :n])
    check_product(a, a_scale, b, b_scale, by_row, c[:m, :n])
    assert (c[m:] == 3).all() and (c[:, n:] == 3).all()
    if by_row and n < 1900:  # scales so far apart (50 GB) that their places need more than 32 bits
        far = torch.empty_strided(b_scale.shape, ((1 << 23) + 1, 1), device=DEV)
        far.copy_(b_scale)
        check_product(a, a_scale, b, far, by_row, wd.product8(wide(a), a_scale, wide(b), far, dtype=dtype))
        del far
        torch.cuda.empty_cache()


@pytest.mark.parametrize("m,n,k", [(130, 4090, 2500), (200, 3300, 2049), (33, 2500, 1000), (20, 2450, 777), (17, 200, 5001), (1, 77, 2047), (300, 300, 2999), (64, 4001, 385), (5, 33, 130), (3, 9000, 700), (50, 9001, 400), (2, 17000, 1030)])
@pytest.mark.parametrize("by_row,dtype", [(False, BF16), (True, F16), (True, F32)])
def test_product_of_few_rows(m, n, k, by_row, dtype):
    """NaN codes behind the rows at 16-byte boundaries and at others, a guard around c."""
    gen = generator(m, n, k)
    a, a_scale, b, b_scale = operands(gen, m, n, k, by_row=by_row)
    if dtype == F16:
        a_scale = a_scale * 0.01

    def wide(t, pitch):
        store = torch.full((t.shape[0] + 1, k + pitch), 0x7F, dtype=torch.uint8, device=DEV)
        store[:-1, :k] = t.contiguous().view(torch.uint8)
        return store.view(t.dtype)[:-1, :k]

    for pitch in (-k % 16 + 16, 1 + k % 2):
        c = torch.full((m + 1, n + 9), 3.0, device=DEV, dtype=dtype)
        wd.product8(wide(a, pitch), a_scale, wide(b, pitch), b_scale, out=c[:m, :n])
        check_product(a, a_scale, b, b_scale, by_row, c[:m, :n])
        assert (c[m:] == 3).all() and (c[:, n:] == 3).all()


@pytest.mark.parametrize("m,n,k", [(5, 40, 300), (20, 17, 1000), (70, 40, 130)])
def test_product_of_rows_far_apart(m, n, k):
    gen = generator(m, n, k)
    a, a_scale, b, b_scale = operands(gen, m, n, k)

    def far(t):
        out = torch.empty_strided(t.shape, ((1 << 23) + 16, 1), dtype=torch.uint8, device=DEV)
        out.copy_(t.contiguous().view(torch.uint8))
        return out.view(t.dtype)

    for dtype in (BF16, F32):
        check_product(a, a_scale, b, b_scale, False, wd.product8(far(a), a_scale, far(b), b_scale, dtype=dtype))


@pytest.mark.parametrize("m,n,k", [(5, 33, 7), (3, 17, 15), (20000, 9, 13), (200, 300, 5), (20000, 40, 200), (600, 700, 1001), (1000, 1000, 129)])
@pytest.mark.parametrize("pitch", [0, 1, 2])
def test_product_of_rows_at_odd_addresses(m, n, k, pitch):
    """Rows one behind the other, NaN codes in front of the first and behind the last."""
    gen = generator(m, n, k, 3)
    a, a_scale, b, b_scale = operands(gen, m, n, k)

    def at_odd(t):
        rows = t.shape[0]
        store = torch.full((1 + rows * (k + pitch) + 16,), 0x7F, dtype=torch.uint8, device=DEV)
        out = store[1:1 + rows * (k + pitch)].view(rows, k + pitch)[:, :k]
        out.copy_(t.contiguous().view(torch.uint8))
        return out.view(t.dtype)

    for dtype in (BF16, F32):
        check_product(a, a_scale, b, b_scale, False, wd.product8(at_odd(a), a_scale, at_odd(b), b_scale, dtype=dtype))


@pytest.mark.parametrize("rows,width", [(1, 1), (70000, 3), (70001, 8), (50000, 9), (40003, 16), (600001, 7), (600000, 13)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_of_very_short_rows(rows, width, dtype):
    """One or two lanes a row: outputs, gradients; dw's terms are added in chains of at most rows / 8 and 20 levels."""
    gen = generator(rows, width)
    x, w, r, dy = normal(gen, rows, width, dtype=dtype), 1 + 0.1 * normal(gen, width), normal(gen, rows, width, dtype=dtype), normal(gen, rows, width, dtype=dtype)
    out = wd.rms_norm(x, w, residual=r, out8=E4M3, y=True)
    check_norm(x, w, r, 1e-5, out, E4M3)
    dx, dw = wd.rms_norm_backward(dy, out.h, w, out.rstd)
    xhat = ref.f64(out.h) * ref.f64(out.rstd)[:, None]
    terms = ref.f64(dy) * xhat
    assert ((ref.f64(dw) - terms.sum(0)).abs() <= (rows / 8 + 24) * EPS24 * terms.abs().sum(0)).all()
    g = ref.f64(dy) * ref.f64(w)
    mean = (g * xhat).mean(1, keepdim=True)
    want = ref.f64(out.rstd)[:, None] * (g - xhat * mean)
    size = ref.f64(out.rstd)[:, None] * (g.abs() + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))
    assert ((ref.f64(dx) - want).abs() <= (width + 24) * EPS24 * size + ref.rounding(want, dtype) * 1.01 + 1e-36).all()
