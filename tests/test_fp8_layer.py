"""The layer with e4m3 experts (paper_2405_18832_b200.fp8) against its steps in 64 bits, and against the bf16 layer."""
import math

import pytest
import torch

import parity as P
from paper_2405_18832_b200 import binding as B
from paper_2405_18832_b200 import fp8 as F
from paper_2405_18832_b200 import synthetic as S

pytestmark = pytest.mark.gpu

WORKLOADS = [S.Workload("l8_top1", S.Problem(300, 256, 512, 16, 1, 24, 0, "bf16", "relu"), 1.2, 5, "random"),
             S.Workload("l8_top2", S.Problem(520, 192, 448, 12, 2, 40, 1, "bf16", "gelu"), 1.0, 6, "random"),
             S.Workload("l8_decode", S.Problem(3, 512, 1024, 64, 2, 8, 1, "bf16", "gelu"), 0.0, 7, "none"),
             S.Workload("l8_tall", S.Problem(2200, 256, 4096, 2, 1, 32, 0, "bf16", "relu"), 0.0, 8, "random"),
             S.config("C2")]


def dequant(q, scale, block_rows):
    s = scale.double().repeat_interleave(block_rows, -2)[..., : q.shape[-2], :].repeat_interleave(128, -1)[..., : q.shape[-1]]
    return q.double() * s


def requant(v):
    """e4m3 values of rows in 64 bits, times their scales."""
    n = v.shape[1]
    full = torch.zeros(v.shape[0], -(-n // 128) * 128, dtype=torch.float64, device=v.device)
    full[:, :n] = v
    b = full.view(v.shape[0], -1, 128)
    s = b.abs().amax(-1, keepdim=True) / 448
    s = torch.where(s < 2.0 ** -100 / 448, torch.ones_like(s), s)
    return ((b / s).to(torch.float8_e4m3fn).double() * s).view(full.shape)[:, :n]


@pytest.mark.parametrize("w", WORKLOADS, ids=[w.name for w in WORKLOADS])
def test_layer_matches_its_steps_and_the_bf16_layer(w):
    p = w.problem
    dev = P.to_device(S.generate(w))
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    residual = torch.randn(p.T, p.d_model, generator=g, device="cuda").bfloat16()
    gamma = (1 + 0.1 * torch.randn(p.d_model, generator=g, device="cuda")).bfloat16()
    ex = F.ExpertWeights(dev["W1"], dev["b1"], dev["W2"], dev["b2"])
    buf = F.LayerBuffers(p)
    out, res = F.moe_ffn_layer_forward(p, dev["x"], residual, gamma, 1e-5, dev["Wg"], dev["bg"], ex, buf)
    B.monde_poll_device_status(buf.ws)

    # the ids are those of the call that also copies rows
    full = B.LayerBuffers(p)
    B.monde_route(p, buf.h, dev["Wg"], dev["bg"], full.topk_idx, full.topk_w, full.counts, full.offsets, full.cls,
                  full.hot_ids, full.cold_ids, full.n_hot_cold, None, full.ws)
    B.monde_permute(p, buf.h, full.topk_idx, full.offsets, full.perm, full.inv_perm, full.x_perm, full.ws)
    assert torch.equal(full.perm, buf.perm) and torch.equal(full.inv_perm, buf.inv_perm)
    assert torch.equal(res, (dev["x"].float() + residual.float()).bfloat16())

    # the products and the combine, from the layer's own rows, ids and gate weights
    q, off = dequant(buf.q, buf.q_scale, 1), buf.offsets.tolist()
    y = torch.zeros(p.T * p.top_k, p.d_model, dtype=torch.float64, device="cuda")
    for e in range(p.E):
        r = slice(off[e], off[e + 1])
        if r.start == r.stop:
            continue
        z = q[buf.perm[r].long() // p.top_k] @ dequant(ex.w1[e], ex.w1_scale[e], 128).T
        if ex.b1 is not None:
            z = z + ex.b1[e].double()
        z = z.clamp(min=0) if p.act == "relu" else 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
        y[r] = requant(z) @ dequant(ex.w2[e], ex.w2_scale[e], 128).T
        if ex.b2 is not None:
            y[r] += ex.b2[e].double()
    ref = (y[buf.inv_perm.long()].view(p.T, p.top_k, -1) * buf.topk_w.double()[:, :, None]).sum(1)
    # y and out are rounded to bf16 (2^-9 each, rms 2^-9 / sqrt 3); an e4m3 value that falls the other way is rare
    assert float((out.double() - ref).norm() / ref.norm()) <= 2.0 ** -8

    # against the bf16 layer: four roundings to e4m3 (rows and weights of both products) of at most 2^-4 / sqrt 3 rms each
    B.moe_ffn_layer_forward(p, buf.h, dev["Wg"], dev["bg"], dev["W1"], dev["b1"], dev["W2"], dev["b2"], full)
    b16 = full.out.double()
    assert float((out.double() - b16).norm() / b16.norm()) <= 2 * 2.0 ** -4 / math.sqrt(3)


def test_dense_ffn_and_graph_replay():
    T, d, f = 70, 512, 1280
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    W1, W2, b1, b2 = rnd(f, d) * 0.05, rnd(d, f) * 0.05, rnd(f), rnd(d)
    x, r, gamma = rnd(T, d).bfloat16(), rnd(T, d).bfloat16(), torch.ones(d, device="cuda").bfloat16()
    ffn = F.DenseFfn(W1, b1, W2, b2, 128, act="gelu")
    ro, out = torch.empty_like(x), torch.empty_like(x)
    ffn.forward(x, r, gamma, 1e-5, ro, out)
    v = x.double() + r.double()
    h = v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-5)
    z = h @ W1.double().T + b1.double()
    ref = (0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))) @ W2.double().T + b2.double()
    assert float((out.double() - ref).norm() / ref.norm()) <= 2 * 2.0 ** -4 / math.sqrt(3)
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ffn.forward(x, r, gamma, 1e-5, ro, out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)


def test_offsets_past_32_bits():
    # weights of 4.8 GB and an output of 2.5 G elements: the last rows, columns and experts are checked
    E, N, K = 256, 8192, 2304
    def e4m3(*shape):
        v = torch.empty(shape, dtype=torch.uint8, device="cuda")
        flat, have = v.view(-1), min(v.numel(), 1 << 20)
        flat[:have] = torch.randint(0, 256, (have,), device="cuda").to(torch.uint8) & 0xBF       # below 2, no NaN
        while have < flat.numel():
            n = min(have, flat.numel() - have)
            flat[have:have + n] = flat[:n]
            have += n
        return v.view(torch.float8_e4m3fn)
    w, ws = e4m3(E, N, K), torch.rand(E, N // 128, K // 128, device="cuda")
    x, xs = e4m3(20, K), torch.rand(20, K // 128, device="cuda")
    for rows in (20, 300):              # both kernels
        off = torch.full((E + 1,), 0, dtype=torch.int32, device="cuda")
        off[E:] = rows                  # everything on the last expert
        ids = torch.arange(rows, dtype=torch.int32, device="cuda") % 20
        out, wk = torch.empty(rows, N, device="cuda"), torch.zeros(B.MATMUL_WS_MAX, dtype=torch.uint8, device="cuda")
        B.monde_grouped_matmul_fp8(x, xs, w, ws, None, off, ids, out, None, wk)
        B.monde_poll_device_status(wk)
        ref = dequant(x, xs, 1)[ids.long()] @ dequant(w[-1], ws[-1], 128).T
        assert float((out.double() - ref).norm() / ref.norm()) <= 1e-5
    del w, ws, out
    rows, K = 310_000, 128
    w, ws = e4m3(N, K), torch.rand(N // 128, 1, device="cuda")
    x, xs = e4m3(rows, K), torch.rand(rows, 1, device="cuda")
    out = torch.empty(rows, N, dtype=torch.bfloat16, device="cuda")
    B.monde_matmul_fp8(x, xs, w, ws, None, out, None, wk)
    B.monde_poll_device_status(wk)
    for r in (slice(0, 64), slice(rows - 200, rows)):
        ref = dequant(x[r], xs[r], 1) @ dequant(w, ws, 128).T
        assert float((out[r].double() - ref).norm() / ref.norm()) <= 2.0 ** -8
    y, q, s = torch.empty_like(out), torch.empty(rows, N, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(rows, N // 128, device="cuda")
    B.monde_rmsnorm_quant(out, None, None, 1e-6, None, y, q, s)
    v = out[-3:].double()
    ref = v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-6)
    assert float((y[-3:].double() - ref).norm() / ref.norm()) <= 2.0 ** -8
    assert float((dequant(q[-3:], s[-3:], 1) - ref).norm() / ref.norm()) <= 2.0 ** -4
