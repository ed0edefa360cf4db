"""What the elements of the experts' floating-point operands may be: bfloat16 or raw 16-bit
integers, e4m3 or raw bytes, e8m0 or raw bytes.  A tensor of another format of the same size
is refused before anything is launched: its values would be taken for others."""
import pytest
import torch

import paper_2606_04101_amd as uep

BF16, F32, I64, U8 = torch.bfloat16, torch.float32, torch.int64, torch.uint8
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
OTHER8 = [torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.bool]


def t(n, dtype=torch.int32):
    return torch.zeros(n, dtype=dtype)


def calls():
    M, N, K = 4, 16, 32
    off, st = t(3, I64), t(1)
    return {
        "ultraep_expert_matmul_bf16": dict(
            x=t(M * K, BF16), M=M, w=t(2 * N * K, BF16), n_w=2, w_stride=N * K, N=N, K=K, trans=False, block_off=off,
            block_w=None, n_block=2, act=uep.ULTRAEP_SWIGLU, pre=t(M * N, BF16), y=t(M * N // 2, BF16), status=st),
        "ultraep_expert_weight_grad": dict(
            dy=t(M * N, BF16), x=t(M * K, BF16), M=M, N=N, K=K, block_off=off, block_w=None, n_block=2, n_w=2,
            dw_stride=N * K, accumulate=False, dw=t(2 * N * K, F32), ws=None, status=st),
        "ultraep_quant_blocks": dict(x=t(M * K, BF16), rows=M, K=K, ld=K, q=t(M * K, U8), ldq=K, scale=t(M * 4, U8)),
        "ultraep_expert_matmul_fp8": dict(
            xq=t(M * K, U8), x_scale=t(M * 4, U8), M=M, wq=t(2 * N * K, U8), w_scale=t(2 * N * 4, U8), n_w=2, N=N, K=K,
            block_off=off, block_w=None, n_block=2, act=0, y=t(M * N, BF16), status=st)}


BF16_ARGS = [("ultraep_expert_matmul_bf16", n) for n in ("x", "w", "pre")] + [("ultraep_expert_weight_grad", n) for n in ("dy", "x")]
E4M3_ARGS = [("ultraep_quant_blocks", "q"), ("ultraep_expert_matmul_fp8", "xq"), ("ultraep_expert_matmul_fp8", "wq")]
E8M0_ARGS = [("ultraep_quant_blocks", "scale"), ("ultraep_expert_matmul_fp8", "x_scale"), ("ultraep_expert_matmul_fp8", "w_scale")]
REFUSED = [(f, n, torch.float16) for f, n in BF16_ARGS] + [(f, n, d) for f, n in E4M3_ARGS for d in OTHER8 + [E8M0]] + \
    [(f, n, d) for f, n in E8M0_ARGS for d in OTHER8 + [E4M3]]
TAKEN = [(f, n, d) for f, n in BF16_ARGS for d in (torch.int16, torch.uint16)] + \
    [(f, n, d) for f, n in E4M3_ARGS for d in (torch.int8, E4M3)] + [(f, n, d) for f, n in E8M0_ARGS for d in (torch.int8, E8M0)]


@pytest.mark.parametrize("entry,name,dtype", REFUSED)
def test_other_formats_are_refused(entry, name, dtype):
    a = calls()[entry]
    a[name] = torch.zeros(a[name].numel(), dtype=U8).view(dtype) if a[name].element_size() == 1 else a[name].view(dtype)
    with pytest.raises(ValueError, match=f"{name}: .*{str(dtype).split('.')[1]}"):
        getattr(uep, entry)(*a.values())


@pytest.mark.parametrize("entry,name,dtype", TAKEN)
def test_raw_words_and_the_formats_own_types_pass(entry, name, dtype):
    """On the host every call ends at the check that its tensors are the device's."""
    a = calls()[entry]
    a[name] = a[name].view(dtype)
    with pytest.raises(ValueError, match="device tensor"):
        getattr(uep, entry)(*a.values())


@pytest.mark.gpu
@pytest.mark.parametrize("entry,name,dtype", REFUSED)
def test_both_halves_refuse_them_on_the_device(entry, name, dtype):
    a = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in calls()[entry].items()}
    assert getattr(uep._load_native(), entry.removeprefix("ultraep_"))(*a.values(), None) == 0
    a[name] = a[name].view(dtype)
    assert getattr(uep._load_native(), entry.removeprefix("ultraep_"))(*a.values(), None) is None
    with pytest.raises(ValueError, match=name):
        getattr(uep, entry)(*a.values())
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("entry,name,dtype", TAKEN)
def test_the_native_half_takes_the_others(entry, name, dtype):
    a = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in calls()[entry].items()}
    a[name] = a[name].view(dtype)
    assert getattr(uep._load_native(), entry.removeprefix("ultraep_"))(*a.values(), None) == 0
    torch.cuda.synchronize()
