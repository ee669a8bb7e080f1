"""CPU-side checks of the 8-bit integer products, the cross attention and the MoE block of a few tokens: struct layouts,
workspace sizes, and refusals that come before the first launch, of the C entries and of the Python functions."""
from __future__ import annotations

import ctypes as C

import pytest
import torch

from paper_2604_08971_amd import binding as sf

ARG, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4
at = C.c_void_p                                                  # addresses that no check reads through
BF, F32, F16 = sf.SF_BF16, sf.SF_F32, sf.SF_F16
BIG = 1 << 40


def test_struct_layouts():
    assert C.sizeof(sf.SfLinearI8) == 8 + 4 * 8 and sf.SfLinearI8.ldw.offset == 16 and sf.SfLinearI8.bias.offset == 32
    assert C.sizeof(sf.SfDenseFfnI8) == 4 * 8
    assert C.sizeof(sf.SfFfnI8) == 8 + 8 * 8 and sf.SfFfnI8.W1q.offset == 8


def _with(base, **kw):
    args = dict(base)
    args.update(kw)
    return args


# ------------------------------------------------------------------------------------------------ quantize_i8_rows
ROWS = dict(x=at(256), dtype=BF, rows=4, n=24, ldx=24, codes=at(512), ldc=24, scale=at(1024), stream=None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), ARG), (dict(n=0), ARG), (dict(ldx=23), ARG), (dict(ldc=23), ARG), (dict(x=None), ARG), (dict(codes=None), ARG),
    (dict(scale=None), ARG), (dict(x=at(257)), ARG), (dict(x=at(258), dtype=F32), ARG), (dict(scale=at(1026)), ARG),
    (dict(dtype=F16), UNSUPPORTED), (dict(dtype=9), UNSUPPORTED), (dict(rows=(1 << 30) + 1), SHAPE), (dict(rows=0, x=None), 0),
])
def test_quantize_refusals(kw, code):
    assert sf.lib().sf_quantize_i8_rows(*_with(ROWS, **kw).values()) == code


# ------------------------------------------------------------------------------------------------ linear_i8
LINEAR = dict(dtype=BF, rows=3, X=at(4096), ldx=64, act=sf.SF_ACT_NONE, R=None, ldr=0, Y=at(8192), ldy=40, ws=at(1 << 16), bytes=BIG, stream=None)
WEIGHTS = dict(N=40, K=64, W=256, ldw=64, s=512, bias=1024)


@pytest.mark.parametrize("weights,kw,code", [
    (dict(N=0), {}, ARG), (dict(K=0), {}, ARG), (dict(K=72, ldw=80), dict(ldx=72), SHAPE), (dict(K=65552, ldw=65552), dict(ldx=65552), SHAPE),
    (dict(ldw=48), {}, ARG), (dict(ldw=72), {}, ARG), (dict(ldw=(1 << 22) + 16), {}, ARG), (dict(W=264), {}, ARG), (dict(W=0), {}, ARG),
    (dict(s=0), {}, ARG), (dict(s=514), {}, ARG), (dict(bias=1025), {}, ARG),
    ({}, dict(rows=-1), ARG), ({}, dict(rows=(1 << 30) + 1), SHAPE), ({}, dict(ldx=63), ARG), ({}, dict(ldy=39), ARG),
    ({}, dict(R=at(12288), ldr=39), ARG), ({}, dict(X=None), ARG), ({}, dict(Y=None), ARG), ({}, dict(Y=at(4096)), ARG), ({}, dict(Y=at(8193)), ARG),
    ({}, dict(R=at(8192), ldr=48), ARG),                         # Y itself, but with other rows
    ({}, dict(dtype=F16), UNSUPPORTED), ({}, dict(dtype=7), UNSUPPORTED), ({}, dict(act=5), UNSUPPORTED), ({}, dict(dtype=F32, X=at(4098)), ARG),
    ({}, dict(ws=None), WORKSPACE), ({}, dict(bytes=255), WORKSPACE), ({}, dict(ws=at((1 << 16) + 128)), WORKSPACE), ({}, dict(rows=0, X=None, Y=None, ws=None), 0),
])
def test_linear_refusals(weights, kw, code):
    lin = sf.SfLinearI8(**_with(WEIGHTS, **weights))
    assert sf.lib().sf_linear_i8_forward(C.byref(lin), *_with(LINEAR, **kw).values()) == code
    if code:
        assert len(sf.lib().sf_last_error()) > 0


def test_linear_workspace():
    L = sf.lib()
    assert L.sf_linear_i8_forward(None, *LINEAR.values()) == ARG
    for rows, K in ((0, 64), (-1, 64), (1, 0), (1, 65537), ((1 << 30) + 1, 16)):
        assert L.sf_linear_i8_workspace_bytes(rows, K) == 0
    assert L.sf_linear_i8_workspace_bytes(100, 64) >= 100 * 64 + 100 * 4
    lin = sf.SfLinearI8(**WEIGHTS)
    need = L.sf_linear_i8_workspace_bytes(3, 64)
    assert L.sf_linear_i8_forward(C.byref(lin), *_with(LINEAR, bytes=need - 1).values()) == WORKSPACE


# ------------------------------------------------------------------------------------------------ pruned FFN
FFN = dict(k_ffn=100, reserved=0, W1q=256, s1=512, b1=1024, W2Tq=2048, s2=4096, b2=8192, ln2_g=16384, ln2_b=32768)
CALL = dict(X=at(1 << 16), pid=None, pre_ln=1, res=1, Y=at(1 << 17), ws=at(1 << 18), bytes=BIG, stream=None)
DESC = dict(B=2, L=16, d_model=64, Hq=4, Hk=2, dh=16, d_ff=128, dtype=BF)


@pytest.mark.parametrize("desc,ffn,kw,code", [
    (dict(dtype=F32), {}, {}, UNSUPPORTED), (dict(dtype=F16), {}, {}, UNSUPPORTED), (dict(d_model=72), {}, {}, SHAPE),
    (dict(d_model=4112), {}, {}, SHAPE), (dict(d_ff=65536), {}, {}, SHAPE), ({}, dict(k_ffn=0), {}, ARG), ({}, dict(k_ffn=129), {}, ARG),
    ({}, dict(W1q=0), {}, ARG), ({}, dict(s1=0), {}, ARG), ({}, dict(W2Tq=0), {}, ARG), ({}, dict(s2=0), {}, ARG), ({}, dict(ln2_g=0), {}, ARG),
    ({}, dict(ln2_b=0), {}, ARG), ({}, dict(W1q=264), {}, ARG), ({}, dict(W2Tq=2056), {}, ARG), ({}, dict(ln2_g=16386), {}, ARG),
    ({}, dict(s1=514), {}, ARG), ({}, dict(s2=4098), {}, ARG), ({}, dict(b1=1025), {}, ARG), ({}, dict(b2=8193), {}, ARG),
    ({}, {}, dict(X=None), ARG), ({}, {}, dict(Y=None), ARG), ({}, {}, dict(Y=at(1 << 16)), ARG), ({}, {}, dict(X=at((1 << 16) + 8)), ARG),
    (dict(P=3), {}, {}, ARG), ({}, {}, dict(ws=None), WORKSPACE), ({}, {}, dict(bytes=1000), WORKSPACE), ({}, {}, dict(ws=at((1 << 18) + 16)), WORKSPACE),
])
def test_pruned_ffn_refusals(desc, ffn, kw, code):
    d, f = sf.make_desc(**_with(DESC, **desc)), sf.SfFfnI8(**_with(FFN, **ffn))
    assert sf.lib().sf_pruned_ffn_i8_forward(C.byref(d), C.byref(f), *_with(CALL, **kw).values()) == code


def test_pruned_ffn_workspace_and_compaction_refusals():
    L = sf.lib()
    d = sf.make_desc(**DESC)
    assert L.sf_pruned_ffn_i8_forward(C.byref(d), None, *CALL.values()) == ARG
    assert L.sf_pruned_ffn_i8_forward(None, None, *CALL.values()) == ARG
    assert L.sf_pruned_ffn_i8_workspace_bytes(C.byref(d), 100) >= 32 * (64 + 4 + 128 + 4)
    for k in (0, 129, -1):
        assert L.sf_pruned_ffn_i8_workspace_bytes(C.byref(d), k) == 0
    assert L.sf_pruned_ffn_i8_workspace_bytes(C.byref(sf.make_desc(**_with(DESC, dtype=F32))), 100) == 0
    call = lambda desc=d, layer=0, dense=None, idx=at(256), **f: L.sf_compact_ffn_i8(
        C.byref(desc), layer, C.byref(sf.SfDenseFfnI8(**_with(dict(W1=256, W2=512, s1=1024, b1=2048), **(dense or {})))), idx,
        C.byref(sf.SfFfnI8(**_with(FFN, **f))), None)
    assert call(layer=1) == ARG and call(layer=-1) == ARG and call(idx=None) == ARG
    assert call(desc=sf.make_desc(**_with(DESC, dtype=F32))) == UNSUPPORTED
    assert call(desc=sf.make_desc(**_with(DESC, d_model=72))) == SHAPE
    for name in ("W1", "W2", "s1"):
        assert call(dense={name: 0}) == ARG
    for name in ("W1q", "s1", "W2Tq", "b1"):
        assert call(**{name: 0}) == ARG
    assert call(k_ffn=0) == ARG and call(k_ffn=129) == ARG and call(dense=dict(W1=264)) == ARG and call(W1q=264) == ARG


# ------------------------------------------------------------------------------------------------ cross attention
S = sf.SfStrides
CROSS = dict(nH=4, nG=2, Lk=100, Q=at(256), sq=S(64, 16, 64), K=at(512), sk=S(3200, 16, 32), V=at(1024), sv=S(3200, 16, 32), group=at(2048), pid=None,
             valid=None, O=at(4096), ldo=64, ws=at(1 << 16), bytes=BIG, stream=None)


def _cross(desc, **kw):
    return sf.lib().sf_cross_gqa_forward(C.byref(desc), *_with(CROSS, **kw).values())


def test_cross_refusals():
    L = sf.lib()
    f32 = sf.make_desc(2, 3, 64, 4, 2, 16, 64, dtype=F32)
    bf = sf.make_desc(2, 3, 128, 4, 2, 32, 64, dtype=BF)
    st = dict(sq=S(128, 32, 128), sk=S(6400, 32, 64), sv=S(6400, 32, 64), ldo=128)
    for kw in (dict(nH=0), dict(nG=0), dict(Lk=0), dict(Q=None), dict(K=None), dict(V=None), dict(group=None), dict(O=None), dict(ldo=63),
               dict(O=at(256)), dict(O=at(512)), dict(O=at(1024)), dict(Q=at(258)), dict(O=at(4098))):
        assert _cross(f32, **kw) == ARG, kw
    for kw in (dict(nH=65, ldo=65 * 16), dict(nG=65), dict(Lk=(1 << 30) + 1), dict(sq=S(-64, 16, 64)), dict(sk=S(3200, -16, 32)),
               dict(sv=S(3200, 16, (1 << 22) + 1))):
        assert _cross(f32, **kw) == SHAPE, kw
    for kw in (dict(ws=None), dict(bytes=255), dict(ws=at((1 << 16) + 64))):
        assert _cross(f32, Lk=1000, **kw) == WORKSPACE, kw       # few rows: the keys are split
    for kw in (dict(Q=at(264)), dict(K=at(520)), dict(V=at(1032)), dict(O=at(4104)), dict(ldo=132)):
        assert _cross(bf, **_with(st, **kw)) == ARG, kw
    for name in ("sq", "sk", "sv"):
        assert _cross(bf, **_with(st, **{name: S(6404, 32, 64)})) == SHAPE and _cross(bf, **_with(st, **{name: S(6400, 36, 64)})) == SHAPE
    assert _cross(sf.make_desc(2, 3, 64, 4, 2, 16, 64, dtype=BF)) == SHAPE                   # head dim of 16 in 16 bits
    assert _cross(sf.make_desc(2, 3, 544, 4, 2, 136, 64, dtype=F32), ldo=544) == SHAPE
    assert _cross(sf.make_desc(2, 3, 64, 4, 2, 16, 64, dtype=F16)) == UNSUPPORTED
    assert _cross(sf.make_desc(70000, 3, 64, 4, 2, 16, 64, dtype=F32)) == SHAPE
    size = L.sf_cross_gqa_workspace_bytes
    assert size(C.byref(f32), 0, 4, 2) == 0 and size(C.byref(f32), 100, 65, 2) == 0 and size(C.byref(f32), 100, 4, 0) == 0
    assert size(C.byref(f32), 1000, 4, 2) > 0
    many = sf.make_desc(64, 2048, 128, 4, 2, 32, 64, dtype=BF)
    assert size(C.byref(many), 2048, 4, 2) == 0                  # workgroups enough without splitting the keys


# ------------------------------------------------------------------------------------------------ MoE block of a few tokens
MOE = dict(n_experts=8, top_k=2, k_ffn_max=100, reserved=0, Wr=256, br=0, W1=512, b1=0, W2T=1024, b2x=0, ln_g=2048, ln_b=4096, k_ffn=8192)
MCALL = dict(X=at(1 << 16), pid=None, pre_ln=1, res=1, forced=None, Y=at(1 << 17), route=None, weight=None, logit=None, ws=at(1 << 18), bytes=BIG, stream=None)


def _moe_struct(**kw):
    m = sf.SfMoeCompact()
    names = [n for n, _ in sf.SfMoeCompact._fields_]
    for n, v in _with(MOE, **kw).items():
        if n in names:
            setattr(m, n, v)
    return m


@pytest.mark.parametrize("desc,moe,kw,code", [
    ({}, dict(n_experts=0), {}, ARG), ({}, dict(n_experts=65), {}, ARG), ({}, dict(top_k=0), {}, ARG), ({}, dict(top_k=9), {}, ARG),
    ({}, dict(n_experts=1, top_k=2), {}, ARG), ({}, dict(k_ffn_max=0), {}, ARG), ({}, dict(k_ffn_max=129), {}, ARG), ({}, dict(k_ffn=0), {}, ARG),
    (dict(d_ff=1 << 19), dict(k_ffn_max=(1 << 18) + 1), {}, SHAPE), (dict(B=13, L=5), {}, {}, SHAPE), (dict(d_model=68, dtype=F32), {}, {}, SHAPE),
    (dict(d_model=1032), {}, {}, SHAPE), (dict(P=513), {}, dict(pid=at(512)), SHAPE),
    ({}, {}, dict(X=None), ARG), ({}, {}, dict(Y=None), ARG), ({}, {}, dict(Y=at(1 << 16)), ARG), ({}, dict(Wr=0), {}, ARG), ({}, dict(W1=0), {}, ARG),
    ({}, dict(W2T=0), {}, ARG), ({}, dict(ln_g=0), {}, ARG), ({}, dict(ln_b=0), {}, ARG), (dict(P=2), {}, {}, ARG),
    ({}, dict(Wr=264), {}, ARG), ({}, dict(W1=520), {}, ARG), ({}, dict(W2T=1032), {}, ARG), ({}, dict(ln_g=2056), {}, ARG), ({}, {}, dict(X=at((1 << 16) + 8)), ARG),
    (dict(dtype=F16), {}, {}, UNSUPPORTED),
    ({}, {}, dict(ws=None), WORKSPACE), ({}, {}, dict(bytes=255), WORKSPACE), ({}, {}, dict(ws=at((1 << 18) + 16)), WORKSPACE),
])
def test_moe_few_refusals(desc, moe, kw, code):
    d, m = sf.make_desc(**_with(_with(DESC, B=4, L=2), **desc)), _moe_struct(**moe)
    assert sf.lib().sf_moe_ffn_few_forward(C.byref(d), C.byref(m), *_with(MCALL, **kw).values()) == code
    if code not in (WORKSPACE,) and (desc or moe) and code == SHAPE:
        assert sf.lib().sf_moe_ffn_few_workspace_bytes(C.byref(d), C.byref(m)) == 0


def test_moe_few_workspace():
    L = sf.lib()
    d = sf.make_desc(**_with(DESC, B=4, L=2))
    assert L.sf_moe_ffn_few_forward(C.byref(d), None, *MCALL.values()) == ARG
    assert L.sf_moe_ffn_few_workspace_bytes(C.byref(d), None) == 0
    assert L.sf_moe_ffn_few_workspace_bytes(C.byref(d), C.byref(_moe_struct())) >= 8 * 8 + 8 * 8 * 4 + 16 * 128 * 4
    assert L.sf_moe_ffn_few_workspace_bytes(C.byref(sf.make_desc(**_with(DESC, B=65, L=1))), C.byref(_moe_struct())) == 0


# ------------------------------------------------------------------------------------------------ Python functions
def test_rows_of_a_tensor():
    x = torch.zeros(6, 32)
    assert sf._rows_of(x, "x") == (6, 32) and sf._rows_of(x[:, :16], "x") == (6, 32) and sf._rows_of(x[::2], "x") == (3, 64)
    assert sf._rows_of(x[0], "x") == (1, 32) and sf._rows_of(x.view(2, 3, 32), "x") == (6, 32) and sf._rows_of(x[:0], "x") == (0, 32)
    assert sf._rows_of(x[:1].expand(1, 32), "x") == (1, 32)
    for bad in (x.t(), x[:1].expand(6, 32), x.view(2, 3, 32)[:, :2], torch.zeros(64).as_strided((4, 32), (8, 1))):
        with pytest.raises(AssertionError):
            sf._rows_of(bad, "x")


def test_strides_of_single_dimensions_say_nothing():
    s = sf._strides_of(torch.zeros(512).as_strided((1, 4, 1, 32), (7, 64, 3, 1)))
    assert (s.b, s.h, s.l) == (0, 64, 0)


def test_tensors_of_the_host_and_wrong_types_are_refused():
    bf, i8 = torch.bfloat16, torch.int8
    with pytest.raises(sf.SentryFuseError):
        sf.quantize_i8_rows(torch.zeros(2, 32))
    with pytest.raises(AssertionError):
        sf.quantize_i8_rows(torch.zeros(2, 32, dtype=torch.float64))
    with pytest.raises(AssertionError):
        sf.quantize_i8_rows(torch.zeros(2, 32), codes=torch.zeros(2, 32))
    with pytest.raises(AssertionError):
        sf.quantize_i8_rows(torch.zeros(2, 32), scale=torch.zeros(3))
    lin = sf.LinearI8(torch.zeros(8, 32, dtype=i8), torch.ones(8))
    with pytest.raises(sf.SentryFuseError):
        sf.linear_i8_forward(lin, torch.zeros(2, 32))
    for X, kw in ((torch.zeros(2, 16), {}), (torch.zeros(2, 32), dict(out=torch.zeros(2, 9))), (torch.zeros(2, 32), dict(residual=torch.zeros(3, 8))),
                  (torch.zeros(2, 32), dict(residual=torch.zeros(2, 8, dtype=bf))), (torch.zeros(2, 32, dtype=torch.float64), {})):
        with pytest.raises(AssertionError):
            sf.linear_i8_forward(lin, X, **kw)
    for codes, scale, bias in ((torch.zeros(8, 32), torch.ones(8), None), (torch.zeros(8, 32, dtype=i8), torch.ones(7), None),
                               (torch.zeros(8, 32, dtype=i8), torch.ones(8, dtype=bf), None), (torch.zeros(8, 32, dtype=i8), torch.ones(8), torch.zeros(9))):
        with pytest.raises(AssertionError):
            sf.LinearI8(codes, scale, bias)
    d = sf.make_desc(2, 3, 64, 4, 2, 16, 64, dtype=F32)
    Q, K, group = torch.zeros(2, 4, 3, 16), torch.zeros(2, 2, 10, 16), torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(sf.SentryFuseError):
        sf.cross_gqa_forward(d, Q, K, K, group)
    for kw in (dict(V=K[:, :1]), dict(head_group=group.long()), dict(head_group=group[:, :3]), dict(key_valid=torch.ones(2, 10)),
               dict(key_valid=torch.ones(2, 9, dtype=torch.uint8)), dict(pattern_id=torch.zeros(3, dtype=torch.int32)), dict(out=torch.zeros(2, 3, 63)),
               dict(out=torch.zeros(2, 5, 64)[:, :3]), dict(K=K.to(bf), V=K.to(bf)), dict(Q=Q[:, :, :2])):
        with pytest.raises(AssertionError):
            sf.cross_gqa_forward(d, **_with(dict(Q=Q, K=K, V=K, head_group=group), **kw))
    with pytest.raises(sf.SentryFuseError):                      # a single row of each sample: any distance between samples
        sf.cross_gqa_forward(sf.make_desc(2, 1, 64, 4, 2, 16, 64, dtype=F32), Q[:, :, :1], K, K, group, out=torch.zeros(2, 5, 64)[:, :1])
    with pytest.raises(AssertionError):
        sf.CompactFfnI8(sf.make_desc(**DESC), 100, W1q=torch.zeros(1, 128, 63, dtype=i8), device="cpu")
    ffn = sf.CompactFfnI8(sf.make_desc(**DESC), 100, s2=torch.ones(64), device="cpu")
    with pytest.raises(sf.SentryFuseError):
        sf.pruned_ffn_i8_forward(sf.make_desc(**DESC), ffn, torch.zeros(32, 64, dtype=bf), pre_ln=False)
    for X in (torch.zeros(32, 64), torch.zeros(31, 64, dtype=bf), torch.zeros(64, 32, dtype=bf).t()):
        with pytest.raises(AssertionError):
            sf.pruned_ffn_i8_forward(sf.make_desc(**DESC), ffn, X)
