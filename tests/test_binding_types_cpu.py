"""The binding refuses tensors of another type than a call computes in, also where their elements are as large: unsigned or
8-bit floating rows are no signed integers, fp16 rows no bf16. Checked on CPU tensors, which come last among the refusals."""
import numpy as np
import pytest
import torch

ppas = pytest.importorskip("paper_2608_15171_amd.ppas", reason="libppas.so not built")

BF, I8, F32 = torch.bfloat16, torch.int8, torch.float32


def t(dtype, *shape):
    return torch.zeros(shape, dtype=torch.uint8).to(dtype)


@pytest.mark.parametrize("dtype", [torch.uint8, torch.bool, torch.float8_e4m3fn, torch.float8_e5m2])
@pytest.mark.parametrize("which", [0, 2])
def test_products_take_signed_bytes(dtype, which):
    a = [t(I8, 4, 64), t(F32, 4), t(I8, 8, 64), t(F32, 8), t(BF, 4, 8)]
    a[which] = t(dtype, *a[which].shape)
    with pytest.raises(ValueError, match="int8"):
        ppas.gateup_proj_i8(*a)
    a[4] = t(BF, 4, 4)
    with pytest.raises(ValueError, match="int8"):
        ppas.gateup_act_i8(*a)


def test_products_write_bf16():
    with pytest.raises(ValueError, match="bf16"):
        ppas.gateup_proj_i8(t(I8, 4, 64), t(F32, 4), t(I8, 8, 64), t(F32, 8), t(torch.float16, 4, 8))


@pytest.mark.parametrize("x,xq,scale", [(torch.float16, I8, F32), (BF, torch.uint8, F32), (BF, torch.bool, F32),
                                        (BF, I8, torch.int32)])
def test_quantiser(x, xq, scale):
    with pytest.raises(ValueError, match="bf16|int8"):
        ppas.quant_i8(t(x, 4, 64), t(xq, 4, 64), t(scale, 4))


@pytest.mark.parametrize("x,y", [(torch.float16, BF), (BF, torch.float16)])
def test_rotary_rows(x, y, monkeypatch):
    # past the device check of x, whose turn comes first
    monkeypatch.setattr(ppas, "_heads", lambda v, name, f=ppas._heads: (0, 256) if v.dtype == BF else f(v, name))
    with pytest.raises(ValueError, match="bf16"):
        ppas.rope_rows(ppas.rope(), t(x, 4, 2, 128), t(torch.int32, 4), t(y, 4, 2, 128))


@pytest.mark.parametrize("dtype", [torch.uint32, torch.float32, torch.int64])
def test_positions(dtype, monkeypatch):
    monkeypatch.setattr(ppas, "_heads", lambda v, name: (0, 256))
    with pytest.raises(ValueError, match="positions must be int32"):
        ppas.rope_rows(ppas.rope(), t(BF, 4, 2, 128), t(dtype, 4), t(BF, 4, 2, 128))


DESC = np.array([[0, 1, 20]], np.int32)


def step_tensors():
    return {"out": t(BF, 1, 16, 128), "q": t(BF, 1, 16, 128), "k": t(BF, 4, 2, 16, 16, 8), "v": t(BF, 4, 2, 128, 16),
            "q_new": t(BF, 1, 16, 128), "k_new": t(BF, 1, 2, 128), "v_new": t(BF, 1, 2, 128), "bt": t(torch.int32, 1, 2),
            "ws": t(torch.uint8, 4096)}


@pytest.mark.parametrize("which,dtype,message", [
    ("out", torch.float16, "out must be bf16"), ("q", torch.float16, "q must be bf16"), ("k", torch.float16, "k_pages must be bf16"),
    ("v", torch.float16, "v_pages must be bf16"), ("bt", torch.float32, "block_table must be")])
def test_shared_attention(which, dtype, message, monkeypatch):
    a = step_tensors()
    a[which] = t(dtype, *a[which].shape)
    monkeypatch.setattr(ppas, "_dev", lambda v, name: 0)
    with pytest.raises(ValueError, match=message):
        ppas.attn_step_shared(ppas.make_shape(16, 2, 4), a["out"], a["q"], a["k"], a["v"], DESC, [(0, 1, 16)], a["bt"], a["ws"])


@pytest.mark.parametrize("which,dtype,message", [
    ("q", torch.float16, "q must be bf16"), ("k", torch.float16, "k_pages must be bf16"),
    ("v", torch.float16, "v_pages must be bf16"), ("q_new", torch.float16, "q_new must be"),
    ("k_new", torch.float16, "k_new must be"), ("v_new", torch.float16, "v_new must be"),
    ("bt", torch.float32, "block_table must be")])
def test_append(which, dtype, message, monkeypatch):
    a = step_tensors()
    a[which] = t(dtype, *a[which].shape)
    monkeypatch.setattr(ppas, "_dev", lambda v, name: 0)
    monkeypatch.setattr(ppas, "_heads", lambda v, name, f=ppas._heads: (0, 2048) if v.dtype == BF else f(v, name))
    with pytest.raises(ValueError, match=message):
        ppas.rope_qkv_append(ppas.make_shape(16, 2, 4), ppas.rope(), a["q"], a["k"], a["v"], a["q_new"], a["k_new"],
                             a["v_new"], DESC, a["bt"])
