"""8-bit floating-point operators (include/monde_fp8.h) against their definitions in 64 bits, on the same input bytes.

Where the tolerances come from (u = 2^-24, the rounding of one fp32 operation):
  quantisation  every step (amax, / 448, 1 / scale, product, rounding) is one correctly rounded operation: bit-equal
  e4m3 values   half a step: 2^-4 of the magnitude, or 2^-10 of the scale among the subnormals
  norm          fp32 sums in at most 45 dependent additions (32 per thread, 10 across the row) and a handful of
                products: 64 u = 2^-18 relative; bf16 outputs add half a step, 2^-9, and at a tie the fp32 error may
                decide, so one whole step, 2^-8
  product       products of two e4m3 values are exact; an accumulation of 32 of them that keeps at least 22 bits loses
                at most 2^-22 of sum|terms|, four per block, and the blocks are added with u each:
                (2^-20 + blocks * u) * sum|terms|; activations are 1.13-Lipschitz at most, gelu adds a few u
"""
import math

import pytest
import torch

from paper_2405_18832_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
E4M3 = torch.float8_e4m3fn
DT = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": E4M3}


def up(n, m=128):
    return -(-n // m)


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def expand(scale, rows, cols, block_rows=1):
    return scale.repeat_interleave(block_rows, -2)[..., :rows, :].repeat_interleave(128, -1)[..., :cols]


def quantize_ref(v, block_rows=1):
    """The header's formulas, one torch operation in fp32 each, on the CPU."""
    v = v.float()
    rows, cols = v.shape[-2:]
    full = torch.zeros(*v.shape[:-2], up(rows, block_rows) * block_rows, up(cols) * 128)
    full[..., :rows, :cols] = v.abs()
    amax = full.unflatten(-1, (-1, 128)).unflatten(-3, (-1, block_rows)).amax(dim=(-3, -1))
    scale = torch.where(amax < 2.0 ** -100, torch.ones_like(amax), amax / 448.0)
    q = (v * expand(1.0 / scale, rows, cols, block_rows)).to(E4M3)
    return q, scale


def same_e4m3(a, b):
    a, b = a.cpu(), b.cpu()
    nan = a.float().isnan()
    return torch.equal(nan, b.float().isnan()) and torch.equal(a.view(torch.uint8)[~nan], b.view(torch.uint8)[~nan])


def same_f32(a, b):
    return torch.equal(torch.nan_to_num(a.cpu(), nan=-1.0), torch.nan_to_num(b.cpu(), nan=-1.0))


def padded(rows, cols, dtype, pad, device="cuda"):
    """A [rows, cols] view with rows `pad` elements further apart, and the whole buffer, filled with a pattern."""
    raw = torch.full((max(rows, 1), (cols + pad) * torch.empty((), dtype=dtype).element_size()), 0x3c, dtype=torch.uint8,
                     device=device)
    return raw.view(dtype)[:rows, :cols], raw


def untouched(view, raw):
    """Bytes of `raw` outside `view` still hold the pattern."""
    keep = torch.ones(raw.shape, dtype=torch.bool, device=raw.device)
    keep[: view.shape[0], : view.shape[1] * view.element_size()] = False
    return bool((raw[keep] == 0x3c).all())


# ---- norm -------------------------------------------------------------------------------------

@pytest.mark.parametrize("T,d", [(1, 1), (1, 128), (3, 130), (7, 1000), (2, 2047), (33, 2048), (5, 2056), (130, 512),
                                 (4, 8200), (2, 32768), (2, 20001), (1, 1024), (9, 129)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 5])
def test_norm_matches_the_definition(T, d, dtype, pad):
    g = gen(T * 7 + d)
    dt = DT[dtype]
    x0 = torch.randn(T, d, generator=g).to(dt)
    r0 = (torch.randn(T, d, generator=g) * 3).to(dt)
    ga = (1 + 0.2 * torch.randn(d, generator=g)).to(dt)
    x, _ = padded(T, d, dt, pad)
    r, _ = padded(T, d, dt, pad)
    x.copy_(x0)
    r.copy_(r0)
    ro, ro_raw = padded(T, d, dt, pad)
    y, y_raw = padded(T, d, dt, pad)
    q, q_raw = padded(T, d, E4M3, pad)
    s, s_raw = padded(T, up(d), torch.float32, pad)
    for residual, gamma in ((r, ga.cuda()), (None, ga.cuda()), (r, None)):
        B.monde_rmsnorm_quant(x, residual, gamma, 1e-6, ro if residual is not None else None, y, q, s)
        v = x0.double() + (0 if residual is None else r0.double())
        u = v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6)
        if gamma is not None:
            u = u * ga.double()
        step = 2.0 ** -8 if dtype == "bf16" else 0.0
        if residual is not None:
            assert ((ro.cpu().double() - v).abs() <= v.abs() * (step + U) + 1e-30).all()
        assert ((y.cpu().double() - u).abs() <= u.abs() * (step + 64 * U) + 1e-30).all()
        sc = s.cpu().double()
        full = torch.zeros(T, up(d) * 128, dtype=torch.float64)
        full[:, :d] = u.abs()
        ref_scale = full.view(T, -1, 128).amax(-1) / 448
        assert ((sc - ref_scale).abs() <= ref_scale * 66 * U).all()
        back = q.cpu().double() * expand(sc, T, d)
        assert ((back - u).abs() <= u.abs() * (2.0 ** -4 + 2.0 ** -16) + expand(sc, T, d) * 2.0 ** -10 * 1.01).all()
    for view, raw in ((ro, ro_raw), (y, y_raw), (q, q_raw), (s, s_raw)):
        assert untouched(view, raw)


def test_norm_in_place_and_single_outputs():
    T, d = 17, 768
    x0 = torch.randn(T, d, generator=gen(1)).bfloat16().cuda()
    r0 = torch.randn(T, d, generator=gen(2)).bfloat16().cuda()
    ga = torch.randn(d, generator=gen(3)).bfloat16().cuda()
    ro, y = torch.empty_like(x0), torch.empty_like(x0)
    q, s = torch.empty(T, d, dtype=E4M3, device="cuda"), torch.empty(T, 6, device="cuda")
    B.monde_rmsnorm_quant(x0, r0, ga, 1e-5, ro, y, q, s)
    x, r = x0.clone(), r0.clone()
    q2, s2 = torch.empty_like(q), torch.empty_like(s)
    B.monde_rmsnorm_quant(x, r, ga, 1e-5, r, x, q2, s2)            # residual and x take the outputs
    assert torch.equal(r, ro) and torch.equal(x, y) and same_e4m3(q, q2) and torch.equal(s, s2)
    y3, ro3, q3, s3 = torch.empty_like(y), torch.empty_like(y), torch.empty_like(q), torch.empty_like(s)
    B.monde_rmsnorm_quant(x0, r0, ga, 1e-5, None, y3, None, None)
    B.monde_rmsnorm_quant(x0, r0, ga, 1e-5, ro3, None, None, None)
    B.monde_rmsnorm_quant(x0, r0, ga, 1e-5, None, None, q3, s3)
    assert torch.equal(y3, y) and torch.equal(ro3, ro) and same_e4m3(q3, q) and torch.equal(s3, s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_of_zero_huge_and_non_finite_rows(dtype):
    d = 300
    x = torch.randn(5, d, generator=gen(4)).to(DT[dtype])
    x[0] = 0
    x[2, 7] = float("nan")
    x[3, 5] = float("inf")
    x[4] *= 2.0 ** -70                                  # far below eps: the norm is linear there
    xc = x.cuda()
    y = torch.empty_like(xc)
    q, s = torch.empty(5, d, dtype=E4M3, device="cuda"), torch.empty(5, 3, device="cuda")
    B.monde_rmsnorm_quant(xc, None, None, 1e-6, None, y, q, s)
    y, q, s = y.float().cpu(), q.float().cpu(), s.cpu()
    assert (y[0] == 0).all() and (q[0] == 0).all() and (s[0] == 1).all()
    assert torch.isfinite(y[1]).all() and torch.isfinite(q[1]).all()
    assert y[2].isnan().all() and q[2].isnan().all() and s[2].isnan().all()     # the row's mean is NaN
    assert (y[3, torch.arange(d) != 5] == 0).all() and y[3, 5].isnan()           # x / inf, inf / inf
    assert s[3, 0].isnan() and (s[3, 1:] == 1).all()
    ref = x[4].double() / math.sqrt(1e-6)
    assert ((y[4].double() - ref).abs() <= ref.abs() * 2.0 ** -7).all()


# ---- quantisation -----------------------------------------------------------------------------

@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (5, 16), (3, 127), (7, 129), (64, 1000), (300, 384), (17, 2040),
                                       (130, 260), (128, 256), (1000, 136)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("pad", [0, 3])
def test_quantisation_is_bit_equal_to_the_formulas(rows, cols, dtype, block_rows, pad):
    v = (torch.randn(rows, cols, generator=gen(rows + cols)) * torch.exp(2 * torch.randn(rows, 1, generator=gen(9)))).to(DT[dtype])
    x, _ = padded(rows, cols, DT[dtype], pad)
    x.copy_(v)
    q, q_raw = padded(rows, cols, E4M3, pad)
    s, s_raw = padded(up(rows, block_rows), up(cols), torch.float32, pad)
    B.monde_quantize_fp8(x, q, s, block_rows)
    rq, rs = quantize_ref(v, block_rows)
    assert same_e4m3(q, rq) and torch.equal(s.cpu(), rs)
    assert untouched(q, q_raw) and untouched(s, s_raw)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantisation_of_batches_and_special_values(block_rows):
    v = torch.randn(3, 200, 300, generator=gen(5))
    v[0, 0, :128] = 0
    v[0, 1, 3] = float("nan")
    v[1, 2, 200] = float("inf")
    v[1, 130, 5] = -float("inf")
    v[2, 150:, 128:256] = 2.0 ** -110
    v[2, 3, 4] = 3e38
    v[2, 7, 9] = 2.0 ** -120
    x = v.cuda()
    if block_rows == 1:
        x, v = x.view(600, 300), v.view(600, 300)
    q = torch.empty(x.shape, dtype=E4M3, device="cuda")
    s = torch.empty((*x.shape[:-2], up(x.shape[-2], block_rows), 3), device="cuda")
    B.monde_quantize_fp8(x, q, s, block_rows)
    rq, rs = quantize_ref(v, block_rows)
    assert same_f32(s, rs) and same_e4m3(q, rq)
    back = q.cpu().float() * expand(s.cpu(), x.shape[-2], 300, block_rows)
    bad = ~torch.isfinite(back)
    hit = ~torch.isfinite(v)
    assert bad[hit].all()                                                    # what was not finite does not read back finite
    per_block = bad.any(-1).any(-1).sum() if block_rows == 128 else None
    if per_block is None:
        assert not bad[~hit.any(-1)].any()                                   # and rows without any are clean


# ---- products ---------------------------------------------------------------------------------

def operands(seed, src_rows, N, K, E=None):
    g = gen(seed)
    lead = () if E is None else (E,)
    x = (torch.randn(src_rows, K, generator=g) * 140).clamp(-448, 448).to(E4M3)
    xs = torch.exp(torch.randn(src_rows, up(K), generator=g)) / 140
    w = (torch.randn(*lead, N, K, generator=g) * 110).clamp(-448, 448).to(E4M3)
    ws = torch.exp(torch.randn(*lead, up(N), up(K), generator=g)) * (0.05 / 110)
    b = torch.randn(*lead, N, generator=g) * 0.5
    return x, xs, w, ws, b


def activate(z, act):
    if act == "relu":
        return z.clamp(min=0)
    # erfc, as 1 + erf cancels to zero below -8.3 and a block whose values all lie there has a scale of its own
    return 0.5 * z * torch.special.erfc(z * -math.sqrt(0.5)) if act == "gelu" else z


def product_ref(x, xs, w, ws, b, act):
    """(out, bound of the error of its fp32 value), in 64 bits."""
    xd = x.double() * expand(xs.double(), *x.shape)
    wd = w.double() * expand(ws.double(), *w.shape, block_rows=128)
    z = xd @ wd.T
    size = xd.abs() @ wd.abs().T
    if b is not None:
        z = z + b.double()
        size = size + b.double().abs()
    tol = size * (2.0 ** -20 + (up(x.shape[1]) + 2) * U)
    out = activate(z, act)
    return out, 1.13 * tol + out.abs() * 4 * U + (z.abs() * 4 * U if act == "gelu" else 0)


def check_out(out, out_scale, ref, tol):
    rows, N = ref.shape
    got = out.cpu()
    if out.dtype == torch.float32:
        assert ((got.double() - ref).abs() <= tol).all()
    elif out.dtype == torch.bfloat16:
        assert ((got.double() - ref).abs() <= tol + ref.abs() * 2.0 ** -8).all()
    else:
        s = out_scale.cpu().double()
        full = torch.zeros(rows, up(N) * 128, dtype=torch.float64)
        full[:, :N] = ref.abs()
        amax = full.view(rows, -1, 128).amax(-1)
        full[:, :N] = tol
        atol = full.view(rows, -1, 128).amax(-1)
        ref_s = torch.where(amax < 2.0 ** -100, torch.ones_like(amax), amax / 448)
        assert ((s - ref_s).abs() <= atol / 448 + ref_s * 4 * U).all()
        se = expand(s, rows, N)
        assert ((got.double() * se - ref).abs() <= tol * 1.1 + ref.abs() * (2.0 ** -4 + 2.0 ** -16) + se * 2.0 ** -10 * 1.01).all()


def workspace(rows, N, K, E=1):
    return torch.zeros(B.monde_matmul_workspace_bytes(rows, N, K, E), dtype=torch.uint8, device="cuda")


def header_is_clean(ws):
    return not bool(ws[: 256 * 1024].any())


SIZES = [(1, 1, 16), (1, 128, 128), (1, 4096, 1024), (2, 129, 144), (15, 8, 32), (16, 256, 256), (17, 255, 112),
         (31, 1000, 2032), (33, 257, 272), (64, 640, 4096), (65, 127, 128), (100, 384, 512), (127, 128, 1024),
         (128, 256, 128), (129, 264, 384), (200, 136, 160), (257, 520, 256), (300, 1024, 768), (1000, 72, 2048),
         (7, 2048, 8192), (513, 769, 1040), (1300, 4096, 400), (3, 8192, 4096), (20, 1032, 528)]


@pytest.mark.parametrize("rows,N,K", SIZES)
@pytest.mark.parametrize("out", ["bf16", "f32", "e4m3"])
def test_product_matches_the_definition(rows, N, K, out):
    act = ("none", "relu", "gelu")[(rows + N + K // 16) % 3]
    x, xs, w, ws, b = operands(rows + N + K, rows, N, K)
    bias = b if (rows + K // 16) % 2 else None
    ref, tol = product_ref(x, xs, w, ws, bias, act)
    wk = workspace(rows, N, K)
    for pad in (0, 3):          # rows of the output and the scales off their 16-byte boundaries; x padded by 16 bytes
        xg, _ = padded(rows, K, E4M3, 16 if pad else 0)
        xsg, _ = padded(rows, up(K), torch.float32, pad)
        xg.copy_(x)
        xsg.copy_(xs)
        o, o_raw = padded(rows, N, DT[out], pad)
        os_, os_raw = padded(rows, up(N), torch.float32, pad)
        B.monde_matmul_fp8(xg, xsg, w.cuda(), ws.cuda(), None if bias is None else bias.cuda(), o,
                           os_ if out == "e4m3" else None, wk, act=act)
        B.monde_poll_device_status(wk)
        check_out(o, os_, ref, tol)
        assert untouched(o, o_raw) and untouched(os_, os_raw) and header_is_clean(wk)
        if out != "e4m3":
            assert bool((os_raw == 0x3c).all())


def split_rows(counts):
    off = torch.zeros(len(counts) + 1, dtype=torch.int32)
    off[1:] = torch.cumsum(torch.tensor(counts), 0)
    return off


GROUPS = [([0, 3, 0, 0, 129, 1, 64, 0], 256, 256, 2), ([1] * 5, 4096, 1024, 1), ([0, 0, 0, 700], 264, 400, 1),
          ([128, 128, 256], 512, 128, 1), ([17, 0, 33, 300, 2, 90], 1000, 1040, 2), ([0] * 60 + [1] + [0] * 194 + [5], 128, 64, 1),
          ([2, 1, 3], 300, 8192, 4), ([0, 0], 128, 128, 1), ([500, 1, 1, 1, 260], 384, 640, 1),
          ([0, 1290, 30], 4096, 272, 2), ([3, 0, 2, 9, 0, 1, 7, 10], 520, 1040, 2), ([2000], 2048, 256, 1)]


@pytest.mark.parametrize("counts,N,K,k", GROUPS)
@pytest.mark.parametrize("out", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("gather", [False, True])
def test_grouped_product_matches_the_definition(counts, N, K, k, out, gather):
    E, A = len(counts), sum(counts)
    off = split_rows(counts)
    spare = 6                                                    # output rows past the last expert
    rows = A + spare
    src_rows = (max(A, 1) + k - 1) // k + 1 if gather else rows
    act = ("none", "relu", "gelu")[(E + A + K // 16) % 3]
    x, xs, w, ws, b = operands(E + A + N + K, src_rows, N, K, E)
    bias = b if A % 2 else None
    ids = torch.randint(0, src_rows * k, (rows,), generator=gen(3), dtype=torch.int32)
    src = ids.long() // k if gather else torch.arange(rows)
    wk = workspace(rows, N, K, E)
    o, o_raw = padded(rows, N, DT[out], 8)
    os_, os_raw = padded(rows, up(N), torch.float32, 0)
    B.monde_grouped_matmul_fp8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), None if bias is None else bias.cuda(), off.cuda(),
                               ids.cuda() if gather else None, o, os_ if out == "e4m3" else None, wk, act=act, row_div=k)
    B.monde_poll_device_status(wk)
    for e in range(E):
        r = slice(int(off[e]), int(off[e + 1]))
        if r.start == r.stop:
            continue
        ref, tol = product_ref(x[src[r]], xs[src[r]], w[e], ws[e], None if bias is None else bias[e], act)
        check_out(o[r], os_[r], ref, tol)
    assert untouched(o, o_raw) and bool((o_raw[A:] == 0x3c).all()) and bool((os_raw[A:] == 0x3c).all())
    assert header_is_clean(wk)


def test_row_ids_outside_the_operand_read_as_zeros():
    rows, N, K, k = 40, 256, 256, 2
    x, xs, w, ws, b = operands(1, 10, N, K, 2)
    ids = torch.randint(0, 20, (rows,), generator=gen(8), dtype=torch.int32)
    for i, v in ((0, -1), (3, 20), (17, -(2 ** 31)), (25, 2 ** 31 - 1), (39, 21)):
        ids[i] = v
    o = torch.empty(rows, N, device="cuda")
    B.monde_grouped_matmul_fp8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), b.cuda(), torch.tensor([0, 18, 40], dtype=torch.int32).cuda(),
                               ids.cuda(), o, None, workspace(rows, N, K, 2), row_div=k)
    for r in range(rows):
        e, i = int(r >= 18), int(ids[r])
        if 0 <= i < 20:
            ref, tol = product_ref(x[[i // k]], xs[[i // k]], w[e], ws[e], b[e], "none")
            assert ((o[[r]].cpu().double() - ref).abs() <= tol).all()
        else:
            assert torch.equal(o[r].cpu(), b[e])


def test_offsets_that_are_not_ascending_stay_inside_the_output():
    # a caller's mistake: the rows are undefined, but nothing outside `rows` is read or written
    rows, N, K = 50, 128, 128
    x, xs, w, ws, _ = operands(2, rows, N, K, 3)
    o, raw = padded(rows, N, torch.bfloat16, 8)
    wk = workspace(rows, N, K, 3)
    B.monde_grouped_matmul_fp8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), None, torch.tensor([-7, 30, 10, 4000], dtype=torch.int32).cuda(),
                               None, o, None, wk)
    B.monde_poll_device_status(wk)
    assert untouched(o, raw) and header_is_clean(wk)


@pytest.mark.parametrize("out", ["bf16", "e4m3"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
def test_non_finite_rows_blocks_and_experts_do_not_leak(out, act):
    counts, N, K = [3, 130, 0, 20], 384, 512
    off, A = split_rows(counts), sum(counts)
    x, xs, w, ws, b = operands(4, A, N, K, 4)
    o1, s1 = torch.zeros(A, N, dtype=DT[out], device="cuda"), torch.zeros(A, 3, device="cuda")
    args = lambda x, xs, w, ws: (x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), b.cuda(), off.cuda(), None)
    wk = workspace(A, N, K, 4)
    B.monde_grouped_matmul_fp8(*args(x, xs, w, ws), o1, s1 if out == "e4m3" else None, wk, act=act)
    x2, xs2, w2, ws2 = (t.clone() for t in (x, xs, w, ws))
    x2.view(torch.uint8)[2, 100] = 0x7f              # NaN in the last row of expert 0
    xs2[140, 1] = float("inf")                       # an infinite scale in expert 3's rows
    xs2[60, 3] = float("nan")
    w2.view(torch.uint8)[2] = 0x7f                   # an expert without rows: all NaN
    ws2[2] = float("nan")
    w2.view(torch.uint8)[1, 130, 5] = 0xff           # one output column of expert 1
    o2, s2 = torch.zeros_like(o1), torch.zeros_like(s1)
    B.monde_grouped_matmul_fp8(*args(x2, xs2, w2, ws2), o2, s2 if out == "e4m3" else None, wk, act=act)
    a, c = o1.float().cpu(), o2.float().cpu()
    if out == "e4m3":
        a, c = a * expand(s1.cpu(), A, N), c * expand(s2.cpu(), A, N)
    touched = torch.zeros(A, N, dtype=torch.bool)
    touched[[2, 140, 60]] = True
    if out == "e4m3":
        touched[3:133, 128:256] = True               # the block that shares the column's scale
        assert not torch.isfinite(c[3:133, 128:256]).any()
    else:
        touched[3:133, 130] = True
        assert c[3:133, 130].isnan().all()
    assert torch.equal(a[~touched], c[~touched])
    assert c[2].isnan().all() and c[60].isnan().all() and not torch.isfinite(c[140]).all()


# Few rows per expert on average (at most 32): tiles of at most 32 rows take another path through the big kernel than the
# rest.  Row counts on both sides of its tile size, ragged N and K, few tiles with a long K (their K range is split).
TURNED = [([31, 32, 33, 0, 1, 64, 8, 9], 264, 528), ([32] * 8, 256, 128), ([0, 129, 1, 2, 0, 0, 16, 17], 130, 1040),
          ([5, 0, 28, 1], 1032, 4112), ([160, 0, 0, 0, 0, 32], 392, 272), ([33, 0], 8, 16)]


@pytest.mark.parametrize("counts,N,K", TURNED)
@pytest.mark.parametrize("out", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("gather", [False, True])
def test_grouped_product_with_few_rows_per_expert(counts, N, K, out, act, gather):
    E, A, k = len(counts), sum(counts), 2
    assert 32 < A <= 32 * E
    off = split_rows(counts)
    src_rows = A // k + 1 if gather else A
    x, xs, w, ws, b = operands(A + N + K, src_rows, N, K, E)
    ids = torch.randint(0, src_rows * k, (A,), generator=gen(5), dtype=torch.int32)
    src = ids.long() // k if gather else torch.arange(A)
    wk = workspace(A, N, K, E)
    for pad in (0, 3):
        o, o_raw = padded(A, N, DT[out], pad)
        os_, os_raw = padded(A, up(N), torch.float32, pad)
        B.monde_grouped_matmul_fp8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), b.cuda(), off.cuda(),
                                   ids.cuda() if gather else None, o, os_ if out == "e4m3" else None, wk, act=act, row_div=k)
        B.monde_poll_device_status(wk)
        for e in range(E):
            r = slice(int(off[e]), int(off[e + 1]))
            if r.start < r.stop:
                ref, tol = product_ref(x[src[r]], xs[src[r]], w[e], ws[e], b[e], act)
                check_out(o[r], os_[r], ref, tol)
        assert untouched(o, o_raw) and untouched(os_, os_raw) and header_is_clean(wk)


@pytest.mark.parametrize("rows,N,K", [(9, 8200, 4112), (32, 4100, 4096), (32, 20000, 528)])
@pytest.mark.parametrize("out", ["bf16", "f32", "e4m3"])
def test_product_of_few_rows_with_many_weights(rows, N, K, out):
    x, xs, w, ws, b = operands(rows + N, rows, N, K)
    ref, tol = product_ref(x, xs, w, ws, b, "relu")
    wk = workspace(rows, N, K)
    o, s = torch.empty(rows, N, dtype=DT[out], device="cuda"), torch.empty(rows, up(N), device="cuda")
    B.monde_matmul_fp8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), b.cuda(), o, s if out == "e4m3" else None, wk, act="relu")
    B.monde_poll_device_status(wk)
    check_out(o, s, ref, tol)
    assert header_is_clean(wk)


@pytest.mark.parametrize("out", ["bf16", "e4m3"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
def test_non_finite_values_in_tiles_of_few_rows_do_not_leak(out, act):
    counts, N, K = [3, 30, 0, 20], 384, 512
    off, A = split_rows(counts), sum(counts)
    x, xs, w, ws, b = operands(4, A, N, K, 4)
    results = []
    for poison in (False, True):
        if poison:
            x.view(torch.uint8)[2, 100] = 0x7f           # NaN in the last row of expert 0
            xs[40, 1] = float("inf")                     # an infinite scale in expert 3's rows
            xs[20, 3] = float("nan")
            w.view(torch.uint8)[2] = 0x7f                # an expert without rows: all NaN
            ws[2] = float("nan")
            w.view(torch.uint8)[1, 130, 5] = 0xff        # one output column of expert 1
        wk = workspace(A, N, K, 4)
        o, s = torch.zeros(A, N, dtype=DT[out], device="cuda"), torch.zeros(A, 3, device="cuda")
        B.monde_grouped_matmul_fp8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), b.cuda(), off.cuda(), None, o,
                                   s if out == "e4m3" else None, wk, act=act)
        B.monde_poll_device_status(wk)
        v = o.float().cpu()
        results.append(v * expand(s.cpu(), A, N) if out == "e4m3" else v)
    a, c = results
    touched = torch.zeros(A, N, dtype=torch.bool)
    touched[[2, 40, 20]] = True
    columns = slice(128, 256) if out == "e4m3" else slice(130, 131)      # the block that shares the column's scale
    touched[3:33, columns] = True
    assert not torch.isfinite(c[3:33, columns]).any()
    assert torch.equal(a[~touched], c[~touched])
    assert c[2].isnan().all() and c[20].isnan().all() and not torch.isfinite(c[40]).all()


def test_same_bits_every_time_and_on_another_stream():
    counts, N, K = [1, 2, 0, 40, 5, 129], 512, 2048
    off, A = split_rows(counts).cuda(), sum(counts)
    x, xs, w, ws, b = (t.cuda() for t in operands(6, A, N, K, 6))
    wk = workspace(A, N, K, 6)
    first = None
    side = torch.cuda.Stream()
    for i in range(6):
        o, s = torch.zeros(A, N, dtype=E4M3, device="cuda"), torch.zeros(A, 4, device="cuda")
        torch.cuda.synchronize()
        if i % 2:
            B.monde_grouped_matmul_fp8(x, xs, w, ws, b, off, None, o, s, wk, act="gelu", stream=side)
        else:
            B.monde_grouped_matmul_fp8(x, xs, w, ws, b, off, None, o, s, wk, act="gelu")
        torch.cuda.synchronize()
        if first is None:
            first = (o, s)
        assert torch.equal(first[0].view(torch.uint8), o.view(torch.uint8)) and torch.equal(first[1], s)


def test_products_of_different_sizes_share_a_workspace_with_layer_calls():
    wk = torch.zeros(B.MATMUL_WS_MAX, dtype=torch.uint8, device="cuda")
    for rows, N, K in SIZES[:12] + SIZES[:12]:
        x, xs, w, ws, b = operands(rows + K, rows, N, K)
        o = torch.empty(rows, N, device="cuda")
        B.monde_matmul_fp8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), None, o, None, wk)
        ref, tol = product_ref(x, xs, w, ws, None, "none")
        check_out(o, None, ref, tol)
    B.monde_poll_device_status(wk)


def test_zero_rows_and_empty_experts_launch_nothing_harmful():
    x = torch.empty(0, 128, dtype=E4M3, device="cuda")
    xs = torch.empty(0, 1, device="cuda")
    _, _, w, ws, b = operands(3, 1, 256, 128, 2)
    o = torch.empty(0, 256, device="cuda")
    wk = workspace(1, 256, 128, 2)
    B.monde_matmul_fp8(x, xs, w[0].cuda(), ws[0].cuda(), None, o, None, wk)
    B.monde_grouped_matmul_fp8(x, xs, w.cuda(), ws.cuda(), b.cuda(), torch.zeros(3, dtype=torch.int32, device="cuda"), None, o,
                               None, wk)
    B.monde_rmsnorm_quant(o.bfloat16(), None, None, 1e-6, None, o.bfloat16(), None, None)
    B.monde_quantize_fp8(o, torch.empty(0, 256, dtype=E4M3, device="cuda"), torch.empty(0, 2, device="cuda"), 1)
    x, xs, w, ws, b = operands(3, 4, 256, 128, 2)
    o = torch.full((4, 256), 7.0, device="cuda")
    B.monde_grouped_matmul_fp8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), b.cuda(), torch.zeros(3, dtype=torch.int32, device="cuda"),
                               None, o, None, wk)
    assert bool((o == 7).all()) and header_is_clean(wk)


def test_binding_refuses_wrong_tensors():
    x, xs, w, ws, b = (t.cuda() for t in operands(7, 4, 256, 128))
    o, wk = torch.empty(4, 256, device="cuda"), workspace(4, 256, 128)
    ok = (x, xs, w, ws, b, o, None, wk)
    B.monde_matmul_fp8(*ok)
    for i, bad in ((0, x.float()), (0, x.cpu()), (1, xs[:3]), (2, w[:, :112]), (2, w.float()), (3, ws.half()), (4, b[:-1]),
                   (5, o[:, ::2]), (5, o[:3])):
        with pytest.raises(ValueError):
            B.monde_matmul_fp8(*ok[:i], bad, *ok[i + 1:])
    with pytest.raises(B.MondeError):
        B.monde_matmul_fp8(*ok[:-1], wk[:1024])
    with pytest.raises(B.MondeError):
        B.monde_matmul_fp8(*ok[:5], torch.empty(4, 256, dtype=E4M3, device="cuda"), None, wk)
    with pytest.raises(KeyError):
        B.monde_matmul_fp8(*ok, act="swish")
    with pytest.raises(ValueError):
        B.monde_rmsnorm_quant(o, o.bfloat16(), None, 1e-6, None, o, None, None)
    with pytest.raises(B.MondeError):
        B.monde_rmsnorm_quant(o.half(), None, None, 1e-6, None, o.half(), None, None)
