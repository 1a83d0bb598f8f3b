"""CPU tests of MXFP4 operands: the codes and scales of one cannot be replaced, and a
call refuses those that were resized since it was made (it would read by their old
sizes). No call reaches the library: the tensors are on the CPU, and what is wrong with
an operand is found before that."""
import pytest
import torch

import paper_2606_00735_amd as moe


def operand(lead, K):
    C = moe.mx4_chunks(K)
    return moe.Mx4Tensor(torch.zeros(lead + (128 * C,), dtype=torch.uint8),
                         torch.zeros(lead[:-1] + (C, lead[-1], 2), dtype=torch.int32), K)


def fewer_codes(t):
    t.codes.resize_(t.codes.shape[:-2] + (t.codes.shape[-2] // 2, t.codes.shape[-1]))


def no_codes(t):
    t.codes.resize_(0)


def other_codes(t):
    t.codes.set_(torch.zeros((3, 64), dtype=torch.uint8))


def strided_codes(t):
    t.codes.transpose_(-1, -2)


def fewer_scales(t):
    t.scales.resize_(t.scales.shape[:-1] + (1,))


def strided_scales(t):
    t.scales.set_(torch.zeros(t.scales.shape[:-1] + (4,), dtype=torch.int32)[..., ::2])


CHANGES = [fewer_codes, no_codes, other_codes, strided_codes, fewer_scales, strided_scales]


@pytest.mark.parametrize("change", CHANGES)
@pytest.mark.parametrize("which", range(4))
def test_resized_operands_are_refused(which, change):
    ops = [operand((4,), 256), operand((2, 128), 256), operand((2, 128), 256), operand((2, 256), 128)]
    off = torch.zeros(3, dtype=torch.int32)
    t = ops[which]
    change(t)
    calls = [lambda: moe.moe_mx4_dequantize(t), lambda: moe.moe_mx4_quantize(torch.zeros(t.shape), out=t)]
    if which == 0:
        calls.append(lambda: moe.moe_grouped_gemm_mx4(ops[0], ops[1], off))
        calls.append(lambda: moe.moe_grouped_swiglu_ffn_mx4(*ops, off))
    for call in calls:
        with pytest.raises(ValueError, match="codes must be|scales must be"):
            call()


@pytest.mark.parametrize("name", ["codes", "scales", "K", "shape", "ld"])
def test_operands_keep_what_they_were_made_of(name):
    t, u = operand((6,), 512), operand((9,), 512)
    with pytest.raises(AttributeError):
        setattr(t, name, getattr(u, name))
    with pytest.raises(AttributeError):
        t.row_count = 3
    assert t.shape == (6, 512) and t.ld == 256


def test_operands_on_the_cpu_are_refused():
    with pytest.raises(ValueError, match="GPU"):
        moe.moe_mx4_dequantize(operand((4,), 256))


@pytest.mark.parametrize("B,R,ld", [(3, 1, 160), (1, 1, 160), (1, 4, 160), (3, 4, 160), (3, 1, 128)])
def test_padded_rows(B, R, ld):
    """Rows ld bytes apart, in batches and matrices of one as well."""
    codes = torch.zeros((B, R, ld), dtype=torch.uint8)[..., :128]
    scales = torch.zeros((B, 1, R, 2), dtype=torch.int32)
    t = moe.Mx4Tensor(codes, scales, 256)
    assert t.shape == (B, R, 256) and t.ld == (ld if B * R > 1 else 128)


def test_rows_that_are_not_a_common_stride_apart_are_refused():
    with pytest.raises(ValueError, match="common stride"):  # matrices of one row that overlap
        moe.Mx4Tensor(torch.zeros(400, dtype=torch.uint8).as_strided((3, 1, 128), (100, 100, 1)),
                      torch.zeros((3, 1, 1, 2), dtype=torch.int32), 256)
    with pytest.raises(ValueError, match="common stride"):  # room between the matrices
        moe.Mx4Tensor(torch.zeros((3, 8, 128), dtype=torch.uint8)[:, :4], torch.zeros((3, 1, 4, 2), dtype=torch.int32), 256)
