"""Sizes of 8-bit integer products that take tiles of 256 x 256 (K from 1024 on, whole rounds of one tile per compute unit nearly full), and row
counts that give a wave several rows to quantise."""
from __future__ import annotations

import pytest
import torch

import test_gpu_i8 as i8
from paper_2604_08971_amd import binding as sf

pytestmark = pytest.mark.gpu


# whole tiles and ragged ones; an even and an odd number of stages, the last one in part; 16-byte rows and others
@pytest.mark.parametrize("dtype,rows,K,N,act,off", [("bf16", 16384, 1024, 1024, sf.SF_ACT_NONE, 0), ("f16", 16300, 1168, 1000, sf.SF_GELU_ERF, 0),
                                                    ("bf16", 32768, 1296, 500, sf.SF_RELU, 8), ("bf16", 65500, 1040, 256, sf.SF_ACT_NONE, 3)])
def test_linear(dtype, rows, K, N, act, off):
    i8.test_linear_of_wide_tiles(dtype, rows, K, N, act, off)


# samples of other patterns, their last tiles not whole
@pytest.mark.parametrize("dtype,act,B,L,d,F,keep,P", [("f16", sf.SF_GELU_ERF, 64, 479, 512, 1030, 1024, 11), ("bf16", sf.SF_RELU, 62, 256, 1008, 1300, 1250, 3)])
def test_pruned_ffn(dtype, act, B, L, d, F, keep, P):
    i8.test_pruned_ffn_of_many_rows(dtype, act, B, L, d, F, keep, P)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,n", [(16384, 8), (16385, 128), (16399, 136), (20001, 256), (16386, 264), (40003, 512), (32769, 520), (32768, 1024)])
def test_quantise_many_rows(dtype, rows, n):
    i8._say("quantise many", dtype, rows, n)
    x = i8._stream(i8._gen(rows + n), rows, n, i8.DT[dtype])
    x[1], x[rows - 1, 0], x[rows // 2, n - 1] = 0, float("nan"), float("-inf")
    with i8._half(dtype):
        codes = torch.full((rows + 1, n), 77, dtype=torch.int8, device="cuda")
        scale = torch.full((rows + 1,), -1.0, device="cuda")
        sf.quantize_i8_rows(x.cuda(), codes[:rows], scale[:rows])
    fine = torch.ones(rows, dtype=torch.bool)
    fine[[rows - 1, rows // 2]] = False
    q, s = i8._codes64(x[fine])
    c, sc = codes.cpu(), scale.cpu()
    assert torch.equal(c[:rows][fine].double(), q) and torch.equal(sc[:rows][fine], s.float()) and torch.isnan(sc[:rows][~fine]).all()
    assert not c[:rows][~fine].any() and torch.all(c[rows] == 77) and sc[rows] == -1
