"""Products in 8-bit integers (i8_rows.hip, i8_gemm.hip, i8_linear.hip) against the definition in 64 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2604_08971_amd import binding as sf

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF = {t: torch.finfo(t).eps / 2 for t in DT.values()}          # a rounding is off by at most half a step
F32 = 2.0 ** -24


def _say(*a):
    print(*a, flush=True)


def _half(dtype):
    return sf.use_half("f16" if dtype == "f16" else "bf16")


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _stream(g, rows, n, dt):
    x = torch.randn(rows, n, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))
    return x.to(dt)


def _codes64(x):
    """x [rows, n] -> codes, scales (float64).  127 x / a has an exact product and one correctly rounded quotient: a quotient that is no tie
    is at least 2^-25 from one (x and a have 24 bits), so it is not rounded to one."""
    x = x.double()
    a = x.abs().amax(1)
    safe = torch.where(a == 0, torch.ones_like(a), a)
    return torch.round(127 * x / safe[:, None]), a / 127


def _act64(z, act):
    return z if act == sf.SF_ACT_NONE else z.clamp(min=0) if act == sf.SF_RELU else z * torch.special.ndtr(z)


# ------------------------------------------------------------------------------------------------ quantiser
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 7), (5, 8), (4, 512), (9, 520), (2, 1024), (7, 2040), (3, 4096), (2, 4104), (1, 20000)])
def test_quantize_rows_exact(dtype, rows, n):
    _say(f"quantize {dtype} {rows}x{n}")
    g = _gen(rows * 7919 + n)
    x = _stream(g, rows, n, DT[dtype])
    if n >= 7:
        x[0, 1::3] = x[0].abs().max() * torch.tensor([0.5])       # 63.5 steps: a tie, up to 64
        x[0, 2] = -x[0].abs().max() * 0.5
    with _half(dtype):
        q, s = sf.quantize_i8_rows(x.cuda())
    rq, rs = _codes64(x)
    assert torch.equal(q.cpu().double(), rq)
    assert torch.all((s.cpu().double() - rs).abs() <= F32 * rs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_rows_extremes(dtype):
    """Zero rows, the smallest and the largest magnitudes, an infinity or a NaN in one row only."""
    _say("quantize extremes", dtype)
    dt, n = DT[dtype], 24
    fi = torch.finfo(dt)
    x = torch.randn(8, n, generator=_gen(5)).to(dt)
    x[0] = 0
    x[1] = torch.linspace(-1, 1, n).to(dt) * fi.max
    x[2] = torch.linspace(-8, 8, n).round().to(dt) * (2.0 ** -133 if dtype == "bf16" else 2.0 ** -149)        # subnormal
    x[3, 5] = float("inf")
    x[4, 0] = float("nan")
    x[5] = fi.tiny
    q, s = sf.quantize_i8_rows(x.cuda())
    q, s = q.cpu(), s.cpu()
    fine = [0, 1, 2, 5, 6, 7]
    rq, rs = _codes64(x[fine])
    assert torch.equal(q[fine].double(), rq)
    assert torch.all((s[fine].double() - rs).abs() <= F32 * rs + 2.0 ** -150)
    for r in (3, 4):
        assert torch.all(q[r] == 0) and torch.isnan(s[r])


def test_quantize_rows_strided_and_neighbours_untouched():
    _say("quantize strided")
    x = torch.randn(11, 40, generator=_gen(3), dtype=torch.float32)
    for off, n in ((0, 33), (1, 32), (3, 17)):
        v = x.cuda()[:, off:off + n]
        codes = torch.full((12, 48), 77, dtype=torch.int8, device="cuda")
        scale = torch.full((12,), -1.0, device="cuda")
        sf.quantize_i8_rows(v, codes=codes[:11, 3:3 + n], scale=scale[:11])
        rq, rs = _codes64(x[:, off:off + n])
        c = codes.cpu()
        assert torch.equal(c[:11, 3:3 + n].double(), rq)
        assert torch.all(c[11] == 77) and torch.all(c[:, :3] == 77) and torch.all(c[:, 3 + n:] == 77)
        assert scale[11].item() == -1.0


# ------------------------------------------------------------------------------------------------ projection
def _weights(g, N, K):
    w = torch.randn(N, K, generator=g) * K ** -0.5
    q, s = _codes64(w)
    return q.to(torch.int8), s.float()


def _linear_ref(x, W, s, b, act, r):
    """value and a bound of the fp32 chain: sum to float, two scales, bias, activation, residual: each step within 2^-24 of what it
    holds; a slope of the activations is at most 1.13"""
    q, sx = _codes64(x)
    p = (q @ W.double().t()) * sx.float().double()[:, None] * s.double()
    z = p if b is None else p + b.double()
    y = _act64(z, act)
    mag = p.abs() + (0 if b is None else b.double().abs())
    if r is not None:
        y, mag = y + r.double(), mag + r.double().abs()
    return y, 8 * F32 * mag


LINEAR = [(1, 512, 512), (1, 16, 1), (8, 1040, 33), (3, 4096, 70), (9, 48, 31), (2, 8192, 19), (130, 256, 128), (257, 144, 129), (64, 2048, 5),
          (1000, 112, 260), (33, 1168, 513)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,K,N", LINEAR)
def test_linear_against_64_bits(dtype, rows, K, N):
    _say(f"linear {dtype} {rows}x{K}x{N}")
    dt = DT[dtype]
    for k, act in enumerate((sf.SF_ACT_NONE, sf.SF_RELU, sf.SF_GELU_ERF)):
        g = _gen(rows + 31 * K + 7 * N + k)
        x, (W, s) = _stream(g, rows, K, dt), _weights(g, N, K)
        b = torch.randn(N, generator=g).to(dt) if k != 1 else None
        r = torch.randn(rows, N, generator=g).to(dt) if k != 2 else None
        with _half(dtype):
            lin = sf.LinearI8(W.cuda(), s.cuda(), None if b is None else b.cuda())
            y = sf.linear_i8_forward(lin, x.cuda(), act, None if r is None else r.cuda()).cpu().double()
        ref, tol = _linear_ref(x, W, s, b, act, r)
        # the GELU of 16-bit outputs is within 4e-5 of itself
        tol = tol + (HALF[dt] + (4e-5 if act == sf.SF_GELU_ERF and dtype != "f32" else 0)) * (ref.abs() + tol) + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
        assert torch.all((y - ref).abs() <= tol), ((y - ref).abs() / tol).max()


@pytest.mark.parametrize("rows", [2, 100])
def test_linear_strides_alias_and_neighbours(rows):
    """Rows of X, W, R and Y inside wider buffers, at odd places; R is Y."""
    _say("linear strides", rows)
    K, N = 96, 45
    g = _gen(rows)
    x = _stream(g, rows, K + 9, torch.bfloat16)
    W, s = _weights(g, N, K)
    wide = torch.zeros(N, K + 32, dtype=torch.int8)
    wide[:, :K] = W
    wide[:, K:] = 99
    y0 = torch.randn(rows + 1, N + 8, generator=g).to(torch.bfloat16)
    for off in (0, 3):
        lin = sf.LinearI8(wide.cuda()[:, :K], s.cuda())
        buf = y0.cuda()
        out = buf[:rows, off:off + N]
        sf.linear_i8_forward(lin, x.cuda()[:, off:off + K], residual=out, out=out)
        ref, tol = _linear_ref(x[:, off:off + K], W, s, None, sf.SF_ACT_NONE, y0[:rows, off:off + N])
        got = buf.cpu()
        assert torch.all((got[:rows, off:off + N].double() - ref).abs() <= tol + HALF[torch.bfloat16] * (ref.abs() + tol))
        got[:rows, off:off + N] = y0[:rows, off:off + N]
        assert torch.equal(got, y0)


@pytest.mark.parametrize("rows", [4, 70])
def test_linear_rows_that_are_not_finite_stay_alone(rows):
    _say("linear not finite", rows)
    g = _gen(9)
    x, (W, s) = _stream(g, rows, 64, torch.bfloat16), _weights(g, 40, 64)
    bad = x.clone()
    bad[1, 3], bad[2, 0] = float("inf"), float("nan")
    lin = sf.LinearI8(W.cuda(), s.cuda())
    for act in (sf.SF_ACT_NONE, sf.SF_RELU):
        y, yb = sf.linear_i8_forward(lin, x.cuda(), act), sf.linear_i8_forward(lin, bad.cuda(), act)
        keep = [r for r in range(rows) if r not in (1, 2)]
        assert torch.equal(y[keep], yb[keep]) and torch.isnan(yb[1:3]).all()


def test_linear_largest_sums():
    """K at its limit with every code at its largest magnitude: the sum is 127^2 K, below 2^31."""
    _say("linear largest sums")
    K = 65536
    x = torch.ones(17, K, dtype=torch.bfloat16)
    W = torch.full((3, K), 127, dtype=torch.int8)
    W[1] = -127
    s = torch.full((3,), 2.0 ** -20)
    y = sf.linear_i8_forward(sf.LinearI8(W.cuda(), s.cuda()), x.cuda().float()).cpu().double()
    ref = 127.0 * K * 2.0 ** -20
    assert torch.all((y - torch.tensor([ref, -ref, ref])).abs() <= 4 * F32 * ref)


# ------------------------------------------------------------------------------------------------ pruned FFN
def _dense(g, F, d, dt, bias=True):
    w = {"W1": torch.randn(F, d, generator=g) * d ** -0.5, "W2": torch.randn(F, d, generator=g) * F ** -0.5,
         "ln2_g": 1 + 0.1 * torch.randn(d, generator=g), "ln2_b": 0.1 * torch.randn(d, generator=g)}
    if bias:
        w["b1"], w["b2"] = 0.1 * torch.randn(F, generator=g), 0.1 * torch.randn(d, generator=g)
    return {k: v.to(dt) for k, v in w.items()}


def _code_range(v, dv):
    """Lowest and highest code that a row of values v, each known to dv, may get, and what its scale may be off by."""
    a = v.abs().amax(1, keepdim=True)
    da = dv.amax(1, keepdim=True)
    safe, low = torch.where(a == 0, torch.ones_like(a), a), torch.clamp(a - da, min=1e-300)
    spread = 127 * (dv / safe + v.abs() * da / (safe * low)) + 2e-5       # 2e-5: the codes of fp32 values are not decided exactly
    t = 127 * v / safe
    return torch.round(t), torch.round((t - spread).clamp(-127, 127)), torch.round((t + spread).clamp(-127, 127)), a / 127, da / 127


def _ffn_ref(x, W1, s1, b1, W2, s2, b2, act, ln, residual):
    """[rows, d] in 64 bits, and how far fp32 statistics and sums may move it: they decide codes that lie at a border."""
    v = x.double()
    dv = torch.zeros_like(v)
    if ln is not None:
        # fp32 mean, deviations and variance of d values: each within (d / 64 + 12) roundings of the sum of magnitudes
        n = v.shape[1] / 64 + 12
        mean = v.mean(1, keepdim=True)
        dm = n * F32 * v.abs().mean(1, keepdim=True)
        var = ((v - mean) ** 2).mean(1, keepdim=True) + 1e-5
        inv = var.rsqrt()
        dinv = inv * (n * F32 + dm * (v - mean).abs().mean(1, keepdim=True) * 2 / var + 3 * F32)
        t = (v - mean) * inv
        dt_ = dm * inv + (v - mean).abs() * dinv + 2 * F32 * (t.abs() + v.abs() * inv)
        dv = dt_ * ln[0].double().abs() + 2 * F32 * (t * ln[0].double()).abs() + F32 * ln[1].double().abs()
        v = t * ln[0].double() + ln[1].double()
    q, lo, hi, sx, dsx = _code_range(v, dv) if ln is not None else (*(_codes64(x)[0],) * 3, _codes64(x)[1][:, None], 0 * sxz(x))
    z = (q @ W1.double().t()) * sx * s1.double() + b1.double()
    dz = ((hi - lo) @ W1.double().abs().t()) * sx * s1.double() + (q @ W1.double().t()).abs() * (dsx + 3 * F32 * sx) * s1.double() \
        + 2 * F32 * (z.abs() + b1.double().abs())
    h = _act64(z, act)
    # slopes up to 1.13; gelu_erf() is within 7e-7 of itself down to -2 and within 4e-5 of 0.05 below
    dh = 1.13 * dz + 3e-6 * h.abs() + (3e-6 if act == sf.SF_GELU_ERF else 0)
    q, lo, hi, sh, dsh = _code_range(h, dh)
    y = (q @ W2.double()) * sh * s2.double() + b2.double()
    dy = ((hi - lo) @ W2.double().abs()) * sh * s2.double() + (q @ W2.double()).abs() * (dsh + 4 * F32 * sh) * s2.double() + 4 * F32 * (y.abs() + b2.double().abs())
    if residual:
        y = y + x.double()
        dy = dy + 2 * F32 * (y.abs() + x.double().abs())
    return y, dy


def sxz(x):
    return x.double().abs().amax(1, keepdim=True)


FFN = [("bf16", sf.SF_RELU, 1, 1, 64, 256, 100, 1), ("f16", sf.SF_GELU_ERF, 2, 3, 512, 512, 400, 1), ("bf16", sf.SF_GELU_ERF, 3, 2, 208, 320, 257, 2),
       ("bf16", sf.SF_RELU, 2, 129, 256, 1024, 614, 1), ("f16", sf.SF_RELU, 5, 61, 144, 300, 300, 3), ("bf16", sf.SF_GELU_ERF, 1, 300, 768, 640, 577, 1),
       ("bf16", sf.SF_RELU, 9, 40, 128, 128, 1, 4)]


@pytest.mark.parametrize("dtype,act,B,L,d,F,keep,P", FFN)
@pytest.mark.parametrize("pre_ln,residual", [(True, True), (False, False)])
def test_pruned_ffn_against_64_bits(dtype, act, B, L, d, F, keep, P, pre_ln, residual):
    _say(f"ffn {dtype} act={act} {B}x{L} d={d} F={F} keep={keep} P={P} ln={pre_ln}")
    dt, g = DT[dtype], _gen(d + keep + P)
    dense = _dense(g, F, d, dt, bias=keep != 300)
    x = _stream(g, B * L, d, dt)
    idx = torch.stack([torch.randperm(F, generator=g)[:keep].sort().values for _ in range(P)])
    ffn_idx = torch.full((1, P, F), -1, dtype=torch.int32)
    ffn_idx[0, :, :keep] = idx.to(torch.int32)
    pid = torch.randint(0, P, (B,), generator=g).to(torch.int32)
    with _half(dtype):
        desc = sf.make_desc(B, L, d, 8, 2, 8, F, P=P, dtype=sf.SF_F16 if dtype == "f16" else sf.SF_BF16, act=act)
        dev = {k: v.cuda() for k, v in dense.items()}
        d8 = sf.quantize_ffn_i8(dev)
        # the dense weights' codes by the definition, a scale per channel of W1 and per column of W2
        q1, r1 = _codes64(dense["W1"])
        q2, r2 = _codes64(dense["W2"].t().contiguous())
        assert torch.equal(d8["W1"].cpu().double(), q1) and torch.equal(d8["W2"].cpu().double().t(), q2)
        cf = sf.compact_ffn_i8(desc, 0, d8, {"ffn_idx": ffn_idx.cuda()}, keep)
        for p in range(P):
            assert torch.equal(cf.W1q[p, :keep].cpu().double(), q1[idx[p]]) and not cf.W1q[p, keep:].any()
            assert torch.equal(cf.W2Tq[p, :, :keep].cpu().double(), q2[:, idx[p]]) and not cf.W2Tq[p, :, keep:].any()
            assert torch.equal(cf.s1[p, :keep].cpu(), d8["s1"].cpu()[idx[p]]) and not cf.s1[p, keep:].any()
        y = sf.pruned_ffn_i8_forward(desc, cf, x.cuda().view(B, L, d), pid.cuda() if P > 1 else None, pre_ln, residual)
    y = y.cpu().double().view(B, L, d)
    for b in range(B):
        i = idx[pid[b] if P > 1 else 0]
        b1 = dense["b1"][i] if "b1" in dense else torch.zeros(keep)
        b2 = dense["b2"] if "b2" in dense else torch.zeros(d)
        ref, tol = _ffn_ref(x.view(B, L, d)[b], q1[i].to(torch.int8), d8["s1"].cpu()[i], b1, q2.t()[i].to(torch.int8), d8["s2"].cpu(), b2, act,
                            (dense["ln2_g"], dense["ln2_b"]) if pre_ln else None, residual)
        tol = tol + HALF[dt] * (ref.abs() + tol) + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
        assert torch.all((y[b] - ref).abs() <= tol), ((y[b] - ref).abs() / tol).max()


def test_pruned_ffn_zero_and_not_finite_rows():
    _say("ffn zero and not finite rows")
    B, L, d, F = 1, 40, 64, 128
    g = _gen(1)
    dense = _dense(g, F, d, torch.bfloat16, bias=False)
    desc = sf.make_desc(B, L, d, 8, 2, 8, F, dtype=sf.SF_BF16)
    idx = torch.arange(F, dtype=torch.int32).view(1, 1, F).cuda()
    cf = sf.compact_ffn_i8(desc, 0, sf.quantize_ffn_i8({k: v.cuda() for k, v in dense.items()}), {"ffn_idx": idx}, F)
    x = _stream(g, L, d, torch.bfloat16)
    x[3] = 0
    bad = x.clone()
    bad[5, 7], bad[6, 0] = float("nan"), float("-inf")
    y, yb = (sf.pruned_ffn_i8_forward(desc, cf, t.cuda().view(B, L, d), None, False, True)[0] for t in (x, bad))
    assert torch.equal(y[3].cpu(), x[3])
    keep = [r for r in range(L) if r not in (5, 6)]
    assert torch.equal(y[keep], yb[keep]) and torch.isnan(yb[5:7]).all()


def test_calls_repeat_to_the_bit_and_replay_from_a_graph():
    _say("i8 graph")
    g = _gen(2)
    x, (W, s) = _stream(g, 300, 256, torch.bfloat16).cuda(), _weights(g, 200, 256)
    lin = sf.LinearI8(W.cuda(), s.cuda())
    ws = sf.workspace(sf.linear_i8_workspace_bytes(300, 256))
    out = torch.empty(300, 200, dtype=torch.bfloat16, device="cuda")
    ref = sf.linear_i8_forward(lin, x)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        sf.linear_i8_forward(lin, x, out=out, ws=ws)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(out, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sf.linear_i8_forward(lin, x, out=out, ws=ws)
    for k in range(3):
        x.copy_(_stream(_gen(50 + k), 300, 256, torch.bfloat16))
        out.zero_()
        ref = sf.linear_i8_forward(lin, x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)


# Rows and features enough for tiles of 256 x 256: whole ones and ragged ones, K of one stage, of odd stages and of many; rows that start on 16 bytes and
# others; two rounds of workgroups
@pytest.mark.parametrize("dtype,rows,K,N,act,off", [("bf16", 16384, 64, 1024, sf.SF_ACT_NONE, 0), ("f16", 16300, 208, 1000, sf.SF_GELU_ERF, 0),
                                                    ("bf16", 32768, 1296, 513, sf.SF_RELU, 8), ("bf16", 65537, 96, 256, sf.SF_ACT_NONE, 3)])
def test_linear_of_wide_tiles(dtype, rows, K, N, act, off):
    _say(f"linear wide {dtype} {rows}x{K}x{N}")
    dt = DT[dtype]
    g = _gen(rows + K)
    x, (W, s) = _stream(g, rows, K, dt), _weights(g, N, K)
    b, r = torch.randn(N, generator=g).to(dt), torch.randn(rows, N + off, generator=g).to(dt)
    with _half(dtype):
        buf = torch.full((rows, N + off), 5.0, dtype=dt, device="cuda")
        sf.linear_i8_forward(sf.LinearI8(W.cuda(), s.cuda(), b.cuda()), x.cuda(), act, r.cuda()[:, off:], out=buf[:, :N])
    assert (buf[:, N:] == 5).all()
    rows_of = torch.cat([torch.arange(300), torch.randint(300, rows - 300, (400,), generator=g), torch.arange(rows - 300, rows)])
    ref, tol = _linear_ref(x[rows_of], W, s, b, act, r[rows_of, off:])
    y = buf[:, :N][rows_of.cuda()].cpu().double()
    tol = tol + (HALF[dt] + (4e-5 if act == sf.SF_GELU_ERF else 0)) * (ref.abs() + tol) + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
    assert torch.all((y - ref).abs() <= tol), ((y - ref).abs() / tol).max()


# Rows enough for the kernels that hold their weights: K of each, one past and short of a step of 32 rows, several patterns, a last group of features that is
# not whole; against few rows of the same call (other kernels): the same codes, so the same bits
@pytest.mark.parametrize("dtype,act,B,L,d,F,keep,P", [("bf16", sf.SF_RELU, 37, 127, 256, 1200, 1100, 1), ("f16", sf.SF_GELU_ERF, 64, 161, 512, 640, 640, 3),
                                                      ("bf16", sf.SF_GELU_ERF, 9, 1025, 768, 960, 900, 1), ("bf16", sf.SF_RELU, 20, 450, 1008, 520, 520, 5),
                                                      ("bf16", sf.SF_GELU_ERF, 300, 33, 48, 1030, 1030, 7)])
def test_pruned_ffn_of_many_rows(dtype, act, B, L, d, F, keep, P):
    _say(f"ffn many rows {dtype} {B}x{L} d={d} F={F} P={P}")
    dt, g = DT[dtype], _gen(d + L)
    dense = {k: v.cuda() for k, v in _dense(g, F, d, dt).items()}
    x = _stream(g, B * L, d, dt).cuda().view(B, L, d)
    ffn_idx = torch.full((1, P, F), -1, dtype=torch.int32)
    for p in range(P):
        ffn_idx[0, p, :keep] = torch.randperm(F, generator=g)[:keep].sort().values.to(torch.int32)
    pid = torch.randint(0, P, (B,), generator=g).to(torch.int32).cuda()
    with _half(dtype):
        dtype_sf = sf.SF_F16 if dtype == "f16" else sf.SF_BF16
        desc = sf.make_desc(B, L, d, 8, 2, 8, F, P=P, dtype=dtype_sf, act=act)
        cf = sf.compact_ffn_i8(desc, 0, sf.quantize_ffn_i8(dense), {"ffn_idx": ffn_idx.cuda()}, keep)
        x[B // 2, L // 2, 3] = float("inf")                      # one row that is not finite
        y = sf.pruned_ffn_i8_forward(desc, cf, x, pid if P > 1 else None)
        for b in (0, B // 2, B - 1):
            one = sf.make_desc(1, L, d, 8, 2, 8, F, P=P, dtype=dtype_sf, act=act)
            yb = sf.pruned_ffn_i8_forward(one, cf, x[b:b + 1].contiguous(), pid[b:b + 1].contiguous() if P > 1 else None)
            # a hidden value may get the next code where its sum is finished in another order of fp32 roundings: a step of 1 / 127 of the row's
            # largest value in that channel, seen through W2; at most one in a thousand does
            nan = torch.isnan(yb[0])
            assert torch.equal(nan, torch.isnan(y[b])) and nan.any(1).sum() == (1 if b == B // 2 else 0)
            same = (y[b] == yb[0]) | nan
            assert same.float().mean() > 0.98, same.float().mean()
            diff = (y[b].double() - yb[0].double()).abs().nan_to_num(0.0)
            assert diff.max() <= 0.02 * yb[0].double().nan_to_num(0.0).abs().max()
