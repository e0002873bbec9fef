"""Distillation by every kind of launch that its rules choose from: a wave per row of one, two and four chunks, alone and in one workgroup, a workgroup per row
of each size, rows that are cut where there are few of them and where there are many; and the second launch of the top logits of cut rows by each size of
workgroup.  At temperatures on both sides of the one that divides the ways.  Tolerances are those of test_gpu_distill.py."""
import pytest
import torch

from test_gpu_distill import agree, call, inputs, reference
from test_gpu_top_logits import check, logits

pytestmark = pytest.mark.gpu

SIZES = [(33, 65806, 764), (40, 135079, 6), (64, 131077, 100), (35, 300007, 64),      # many rows, cut
         (33, 66000, 50), (34, 131001, 70), (36, 65530, 3),                           # a workgroup of 1024 threads of sixteen chunks
         (5, 254, 2), (100, 505, 8), (2, 253, 2), (3, 511, 64), (4, 1000, 16), (1, 509, 1), (1, 1018, 36), (4, 2039, 64), (1592, 529, 8), (2000, 1000, 30), (1586, 1046, 29),
         (2000, 2040, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", SIZES)
def test_against_the_formulas(n, classes, k, dtype):
    for labels, temperature, alpha, ragged in ((False, 2.0, 1.0, True), (True, 4.0, 0.9, False), (True, 8.0, 0.3, True), (False, 8.0, 1.0, False)):
        x = inputs(n, classes, k, dtype, labels=labels, ragged=ragged)
        out = call(*x, temperature, alpha)
        agree(out, reference(*x, temperature, alpha), dtype)
        again = call(*x, temperature, alpha, inplace=True)
        assert all(torch.equal(again[w], out[w]) for w in out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(40, 135079, 6), (33, 66000, 50), (3, 511, 64), (2000, 1000, 30), (100, 505, 8)])
def test_rows_that_do_not_count(n, classes, k, dtype):
    for temperature in (2.0, 20.0):
        for labels, alpha in ((False, 1.0), (True, 0.5)):
            z, index, top, lab = inputs(n, classes, k, dtype, labels=labels, padded=True)
            z[::3] = float("nan")
            got = call(z, index, top, lab, temperature, alpha, ignore=-9)
            # (the definition's terms at T = 20 are 25 times those at 4 and its fp32 ones as much: sizes say so)
            agree(got, reference(torch.nan_to_num(z), index, top, lab, temperature, alpha, ignore=-9), dtype)
            assert (got["rows"][::3] == 0).all() and (got["dz"][::3] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(3, 356294, 683), (2, 327948, 56), (2, 338396, 189), (2, 329327, 299), (3, 328209, 47), (2339, 69983, 140), (3, 527948, 27)])
def test_top_logits_of_cut_rows(n, classes, k, dtype):
    check(logits(n, classes, dtype), k)
    check((2 * logits(n, classes, dtype)).round(), k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(1 << 20, 3, 2), (70001, 40, 5), (300000, 130, 100)])
def test_top_logits_of_many_rows(n, classes, k, dtype):
    check(logits(n, classes, dtype), k)
    check((2 * logits(n, classes, dtype)).round(), k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,k", [(1 << 20, 3, 2), (70001, 40, 40)])
def test_many_rows_at_a_high_temperature(n, classes, k, dtype):
    x = inputs(n, classes, k, dtype, labels=True)
    agree(call(*x, 8.0, 0.5), reference(*x, 8.0, 0.5), dtype)
