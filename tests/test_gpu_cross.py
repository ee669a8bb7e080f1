"""Cross attention (cross.hip) against softmax attention in 64 bits."""
from __future__ import annotations

import pytest
import torch

from paper_2604_08971_amd import binding as sf

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SF = {"bf16": sf.SF_BF16, "f16": sf.SF_F16, "f32": sf.SF_F32}
F32 = 2.0 ** -24


def _say(*a):
    print(*a, flush=True)


def _half(dtype):
    return sf.use_half("f16" if dtype == "f16" else "bf16")


def _reference(Q, K, V, group, valid):
    """[B, Lq, nH*dh] in 64 bits and a bound: scores are fp32 sums of dh exact products, weights come through exp2 (a few units) and are
    rounded to 16 bits (half a step; in binary16 the smallest are off by 2^-29 of the largest at most), sums are fp32."""
    B, nH, Lq, dh = Q.shape
    Lk, half = K.shape[2], 0.0 if Q.dtype == torch.float32 else torch.finfo(Q.dtype).eps / 2
    O, T = (torch.zeros(B, Lq, nH, dh, dtype=torch.float64) for _ in range(2))
    for b in range(B):
        keys = slice(None) if valid is None else valid[b].nonzero().flatten()
        for h in range(nH):
            g = int(group[b][h])
            if not 0 <= g < K.shape[1]:
                continue
            q, k, v = Q[b, h].double(), K[b, g].double()[keys], V[b, g].double()[keys]
            if not len(k):
                continue
            s = q @ k.t() / dh ** 0.5
            ds = ((dh + 4) * F32 * (q.abs() @ k.abs().t()) / dh ** 0.5 + 4 * F32 * s.abs()).amax(1, keepdim=True) * 2 + 8 * F32
            w = torch.softmax(s, 1)
            o, mag = w @ v, w @ v.abs()
            O[b, :, h] = o
            T[b, :, h] = (half + 2 * ds + (Lk / 64 + 40) * F32) * (mag + o.abs()) + half * (o.abs() + 1e-30)
            if Q.dtype == torch.float16:
                T[b, :, h] += len(k) * 2.0 ** -29 * v.abs().amax() + 2.0 ** -25
            T[b, :, h] *= 1 + 2 * half
    return O.view(B, Lq, nH * dh), T.view(B, Lq, nH * dh)


def _case(dtype, B, Lq, Lk, nH, nG, dh, mask=None, seed=0, layout="token", group=None, pid=None, spread=1.5):
    g = torch.Generator().manual_seed(seed + Lq * 131 + Lk)
    dt = DT[dtype]
    rnd = lambda *s: torch.randn(*s, generator=g)
    if layout == "token":
        Q = (spread * rnd(B, Lq, nH, dh)).to(dt).transpose(1, 2)
        kv = rnd(B, Lk, 2, nG, dh).to(dt)
        K, V = kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    else:
        Q, K, V = (spread * rnd(B, nH, Lq, dh)).to(dt), rnd(B, nG, Lk, dh).to(dt), rnd(B, nG, Lk, dh).to(dt)
    if group is None:
        group = torch.arange(nH).div(nH // nG, rounding_mode="floor").view(1, nH)
    group = group.to(torch.int32)
    valid = None
    if mask == "scattered":
        valid = torch.rand(B, Lk, generator=g) < 0.6
    elif mask == "segments":
        valid = torch.zeros(B, Lk, dtype=torch.bool)
        for b in range(B):
            a = int(torch.randint(0, Lk, (1,), generator=g))
            valid[b, a:a + max(1, Lk // 3)] = True
    elif mask == "one":
        valid = torch.zeros(B, Lk, dtype=torch.bool)
        valid[torch.arange(B), torch.randint(0, Lk, (B,), generator=g)] = True
    elif mask == "all":
        valid = torch.ones(B, Lk, dtype=torch.bool)
    if valid is not None and mask != "all" and B > 1:
        valid[B - 1] = False                                     # a sample without any
    return Q, K, V, group, valid, pid


def _on(layout, t):
    """The same strides on the device."""
    return t.transpose(1, 2).contiguous().cuda().transpose(1, 2) if layout == "token" else t.cuda()


def _run(dtype, Q, K, V, group, valid, pid=None, layout="token", **kw):
    B, nH, Lq, dh = Q.shape
    with _half(dtype):
        desc = sf.make_desc(B, Lq, nH * dh, nH, nH, dh, 64, dtype=SF[dtype])
        return sf.cross_gqa_forward(desc, _on(layout, Q), _on(layout, K), _on(layout, V), group.cuda(), None if pid is None else pid.cuda(),
                                    None if valid is None else valid.to(torch.uint8).cuda(), **kw)


def _check(dtype, case, layout="token"):
    Q, K, V, group, valid, pid = case
    y = _run(dtype, Q, K, V, group, valid, pid, layout).cpu().double()
    per = group[pid.long()] if pid is not None else group.expand(Q.shape[0], -1)
    ref, tol = _reference(Q, K, V, per, valid)
    bad = (y - ref).abs() > tol
    assert not bad.any(), (((y - ref).abs() / tol).max(), bad.nonzero()[:4])


# one key and one row; tiles with one key and one short of them; rows of one and of several runs; key ranges in workgroups of their own
SIZES = [(1, 1, 1, 1, 1), (2, 1, 63, 3, 1), (1, 1, 4097, 12, 4), (3, 5, 64, 8, 2), (2, 11, 65, 6, 3), (2, 32, 200, 4, 4), (1, 33, 130, 2, 1),
         (2, 128, 257, 4, 2), (1, 129, 1000, 3, 3), (9, 300, 96, 16, 4), (1, 7, 20000, 4, 2), (5, 2, 8, 64, 1)]


@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("f16", 64), ("f16", 128), ("f32", 8), ("f32", 24), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("B,Lq,Lk,nH,nG", SIZES)
def test_cross_against_64_bits(dtype, dh, B, Lq, Lk, nH, nG):
    _say(f"cross {dtype} dh={dh} B={B} Lq={Lq} Lk={Lk} heads={nH}/{nG}")
    _check(dtype, _case(dtype, B, Lq, Lk, nH, nG, dh))
    for k, mask in enumerate(("scattered", "segments")):
        _check(dtype, _case(dtype, B, Lq, Lk, nH, nG, dh, mask, seed=k + 1))


def test_many_rows_of_the_largest_runs():
    """Enough rows for the runs of 256."""
    _say("cross runs of 256")
    for dh, mask in ((64, None), (64, "scattered"), (32, "segments")):
        _check("bf16", _case("bf16", 16, 1025, 70, 32, 4, dh, mask))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("Lq", [1, 40])
def test_what_masked_keys_hold_is_not_used(dtype, Lq):
    _say("cross masked values", dtype, Lq)
    Q, K, V, group, valid, _ = _case(dtype, 3, Lq, 300, 4, 2, 64, "scattered")
    y = _run(dtype, Q, K, V, group, valid)
    for bad in (float("nan"), float("inf"), float("-inf"), torch.finfo(DT[dtype]).min):
        K2, V2 = K.clone(), V.clone()
        out = ~valid[:, None, :, None].expand_as(K)
        K2[out], V2[out] = bad, bad
        assert torch.equal(_run(dtype, Q, K2, V2, group, valid), y)
    assert not y[2].any()                                        # no allowed key: zeros
    full = _case(dtype, 3, Lq, 300, 4, 2, 64, "all")
    assert torch.equal(_run(dtype, *full[:5]), _run(dtype, *full[:4], None))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_and_one_key(dtype):
    """Scores of hundreds that rise tile by tile; a single allowed key gives its value."""
    _say("cross large scores", dtype)
    for Lq in (3, 60):
        Q, K, V, group, valid, _ = _case(dtype, 2, Lq, 500, 4, 2, 64, "one", spread=30.0)
        y = _run(dtype, Q, K, V, group, valid).cpu()
        j = int(valid[0].nonzero())
        want = V[0, :, j].repeat_interleave(2, 0).reshape(-1).expand(Lq, -1)
        assert torch.equal(y[0], want)
        Q, K, V, group, _, _ = _case(dtype, 1, Lq, 500, 4, 2, 64)
        up = torch.linspace(0, 20, 500).view(1, 1, 500, 1)
        K = (K.float() * 0 + up * 0.25).to(DT[dtype])
        Q = Q.abs() + DT_ONE[dtype]
        _check(dtype, (Q, K, V, group, None, None))


DT_ONE = {"bf16": torch.tensor(1.0, dtype=torch.bfloat16), "f32": torch.tensor(1.0)}


def test_maps_patterns_layouts_and_rows_left_alone():
    """Heads of a group that are not neighbours, a map per pattern, a pruned head (its columns stay), another layout, rows of O inside
    wider ones."""
    _say("cross maps")
    group = torch.tensor([[0, 2, 1, 0, 2, 2], [1, 1, 1, 1, 1, -1]])
    pid = torch.tensor([1, 0, 1], dtype=torch.int32)
    for Lq in (2, 70):
        for layout in ("token", "head"):
            case = _case("bf16", 3, Lq, 150, 6, 3, 64, "scattered", layout=layout, group=group, pid=pid)
            Q, K, V, grp, valid, _ = case
            wide = torch.full((3, Lq, 6 * 64 + 24), 7.0, dtype=torch.bfloat16, device="cuda")
            out = wide[:, :, 8:8 + 6 * 64]
            _run("bf16", Q, K, V, grp, valid, pid, layout, out=out)
            ref, tol = _reference(Q, K, V, grp[pid.long()], valid)
            y = wide.cpu()
            assert (y[:, :, :8] == 7).all() and (y[:, :, 8 + 6 * 64:] == 7).all()
            y = y[:, :, 8:8 + 6 * 64]
            for b in (0, 2):
                assert (y[b, :, 5 * 64:] == 7).all()
                y[b, :, 5 * 64:] = 0
            assert ((y.double() - ref).abs() <= tol).all()


def test_strides_of_zero_share_a_tensor():
    """One set of states for all samples, one value for all keys: strides of zero."""
    _say("cross strides of zero")
    g = torch.Generator().manual_seed(4)
    Q = torch.randn(3, 4, 9, 64, generator=g).to(torch.bfloat16)
    K = torch.randn(1, 2, 100, 64, generator=g).to(torch.bfloat16)
    V = torch.randn(1, 2, 1, 64, generator=g).to(torch.bfloat16)
    group = torch.tensor([[0, 0, 1, 1]], dtype=torch.int32).cuda()
    desc = sf.make_desc(3, 9, 256, 4, 4, 64, 64, dtype=sf.SF_BF16)
    Kd, Vd = K.cuda().expand(3, -1, -1, -1), V.cuda().expand(3, -1, 100, -1)
    y = sf.cross_gqa_forward(desc, Q.cuda(), Kd, Vd, group).cpu()
    want = V[0, :, 0].repeat_interleave(2, 0).reshape(-1).expand(3, 9, -1)
    assert ((y.double() - want.double()).abs() <= 2.0 ** -7 * want.double().abs()).all()


def test_states_beyond_32_bits_of_offset():
    """Keys that lie more than 2^32 bytes behind the tensor's start."""
    _say("cross far keys")
    Lk, step = 70000, 1 << 15                                    # 70 000 rows, 64 KB apart: 4.6 GB
    buf = torch.empty(Lk * step, dtype=torch.bfloat16, device="cuda")
    view = buf.view(1, 1, Lk, step)[..., :64]
    small = torch.randn(1, 1, Lk, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(torch.bfloat16)
    view.copy_(small)
    Q = torch.randn(1, 2, 3, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(2)).to(torch.bfloat16)
    group = torch.zeros(1, 2, dtype=torch.int32, device="cuda")
    desc = sf.make_desc(1, 3, 128, 2, 2, 64, 64, dtype=sf.SF_BF16)
    assert torch.equal(sf.cross_gqa_forward(desc, Q, view, view, group), sf.cross_gqa_forward(desc, Q, small, small, group))


def test_cross_repeats_to_the_bit_and_replays_from_a_graph():
    _say("cross graph")
    for Lq, Lk in ((1, 3000), (200, 300)):
        Q, K, V, group, valid, _ = (t.cuda() if t is not None else None for t in _case("bf16", 2, Lq, Lk, 4, 2, 64, "scattered", layout="head"))
        valid = valid.to(torch.uint8)
        desc = sf.make_desc(2, Lq, 256, 4, 4, 64, 64, dtype=sf.SF_BF16)
        out = torch.empty(2, Lq, 256, dtype=torch.bfloat16, device="cuda")
        ws = sf.workspace(sf.cross_gqa_workspace_bytes(desc, Lk, 4, 2))
        call = lambda: sf.cross_gqa_forward(desc, Q, K, V, group, None, valid, out=out, ws=ws)
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for k in range(3):
            Q.copy_(torch.randn(Q.shape, generator=torch.Generator().manual_seed(k)))
            ref = sf.cross_gqa_forward(desc, Q, K, V, group, None, valid)
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref)
