"""CPU checks of what the rotation, the appends with it and the calls on a cache of 8 bits refuse."""
import pytest

from paper_2503_02356_amd import binding as B
from tests.test_paged_abi import COMMON, append, paged, refused

INVALID, OTHER = B.CF_EINVAL, B.CF_EUNSUPPORTED


def change(p, name, value):
    *path, last = name.split(".")
    for x in path:
        p = getattr(p, x)
    setattr(p, last, value)


def rotate(**c):
    p = B.RotateParams()
    p.head_dim, p.n_tokens, p.n_segments, p.cu_seqlens_q, p.cu_seqlens_k = 128, 10, 2, 4096, 4096
    p.rotation = B.Rotation(4096, 128, 0)
    p.q = B.RotateTensor(4, B.CF_BF16, B.CF_BF16, 1 << 20, 512, 128, 1 << 21, 512, 128)
    p.k = B.RotateTensor(2, B.CF_FP32, B.CF_BF16, 1 << 22, 256, 128, 1 << 23, 256, 128)
    for name, value in c.items():
        change(p, name.replace("__", "."), value)
    return p


def turn(**c):
    r = B.AppendRotation(B.Rotation(4096, 64, 1), 4, 0, 1 << 20, 512, 128, 1 << 21, 512, 128)
    for name, value in c.items():
        change(r, name.replace("__", "."), value)
    return r


def append8(**c):
    p = B.KvAppend8Params(append(), 4096, 4096, 8, 4)
    for name, value in c.items():
        change(p, name.replace("__", "."), value)
    return p


def attend8(**c):
    p = B.AttnPaged8Params(paged(), 4096, 4096, 8, 4)
    for name, value in c.items():
        change(p, name.replace("__", "."), value)
    return p


ROTATION = [("inv_freq", None, INVALID), ("inv_freq", 4098, INVALID), ("rot_dim", 0, INVALID), ("rot_dim", 24, INVALID), ("rot_dim", 144, INVALID),
            ("rot_dim", -16, INVALID)]
SCALES = [("k_scales", None, INVALID), ("v_scales", 4098, INVALID), ("scale_stride_page", 3, INVALID), ("scale_stride_head", 3, INVALID),
          ("scale_stride_head", -4, INVALID)]


@pytest.mark.parametrize("name,value,code", [("rotation__" + a, b, c) for a, b, c in ROTATION] + [
    ("head_dim", 96, OTHER), ("n_tokens", 0, INVALID), ("n_segments", 0, INVALID), ("n_segments", (1 << 30) + 1, INVALID), ("inverse", 2, INVALID),
    ("cu_seqlens_q", None, INVALID), ("cu_seqlens_k", 4098, INVALID), ("q__n_heads", -1, INVALID), ("q__n_heads", 65536, INVALID), ("q__dtype_in", 2, OTHER),
    ("q__dtype_out", B.CF_FP32, OTHER), ("k__dtype_out", -1, OTHER), ("q__x", None, INVALID), ("q__y", (1 << 21) + 8, INVALID), ("k__x_stride_tok", 258, INVALID),
    ("k__y_stride_head", 124, INVALID), ("q__x_stride_head", 120, INVALID), ("q__y_stride_tok", -512, INVALID)])
def test_rotate_refuses(name, value, code):
    refused(code, B.cf_rotate, rotate(**{name: value}))
    assert B.lib().cf_rotate(None, None) == INVALID


def test_rotate_in_place_needs_one_layout():
    refused(INVALID, B.cf_rotate, rotate(k__y=1 << 22))                                  # (fp32 to bf16)
    refused(INVALID, B.cf_rotate, rotate(q__y=1 << 20, q__y_stride_tok=1024))
    refused(INVALID, B.cf_rotate, rotate(q__n_heads=0, k__n_heads=0))


@pytest.mark.parametrize("name,value,code", [("rotation__" + a, b, c) for a, b, c in ROTATION] + [
    ("n_q_heads", 0, INVALID), ("q", (1 << 20) + 2, INVALID), ("q", None, INVALID), ("q_out", None, INVALID), ("q_out_stride_tok", 508, INVALID),
    ("q_out", 1 << 20, None), ("q_stride_head", 0, INVALID)])
def test_appends_refuse_a_rotation(name, value, code):
    for call, p in ((B.cf_kv_append_rotated, append()), (B.cf_kv_append8, append8())):
        if code is None:                             # in place, other strides
            with pytest.raises(B.CfError):
                call(p, turn(q_out=value, q_out_stride_tok=1024), stream=0)
        else:
            with pytest.raises(B.CfError) as e:
                call(p, turn(**{name: value}), stream=0)
            assert e.value.code == code and call.__name__ in str(e.value)


@pytest.mark.parametrize("name,value,code", COMMON + [("n_kv_heads", 0, INVALID), ("k", None, INVALID), ("v", 8, INVALID), ("page_stride_head", 4, INVALID),
                                                      ("page_stride_tok", 12, INVALID)])
def test_append_rotated_refuses(name, value, code):
    with pytest.raises(B.CfError) as e:
        B.cf_kv_append_rotated(append(**{name: value}), turn(), stream=0)
    assert e.value.code == code and "cf_kv_append_rotated" in str(e.value)
    assert B.lib().cf_kv_append_rotated(None, None, None) == INVALID


@pytest.mark.parametrize("name,value,code", [("a__" + a, b, c) for a, b, c in COMMON] + SCALES + [
    ("a__n_kv_heads", 0, INVALID), ("a__n_kv_heads", 65535, INVALID), ("a__k", None, INVALID), ("a__v", 8, INVALID), ("a__page_stride_head", 136, INVALID),
    ("a__page_stride_tok", 136, INVALID), ("a__page_stride", 64 * 256 + 8, INVALID)])
def test_append8_refuses(name, value, code):
    refused(code, B.cf_kv_append8, append8(**{name: value}))


def test_append8_refuses_more_blocks_than_a_launch_holds():
    refused(INVALID, B.cf_kv_append8, append8(a__n_tokens=1 << 27, a__n_seqs=1 << 29))      # (either one alone is less)
    assert B.lib().cf_kv_append8(None, None, None) == INVALID


@pytest.mark.parametrize("name,value,code", [("a__" + a, b, c) for a, b, c in COMMON] + SCALES + [
    ("a__n_q_heads", 5, INVALID), ("a__n_tokens", 1 << 30, INVALID), ("a__flags", 2, INVALID), ("a__max_kv_len", -1, INVALID), ("a__window", -1, INVALID),
    ("a__n_sinks", 1, INVALID), ("a__softmax_scale", float("nan"), INVALID), ("a__q", None, INVALID), ("a__o", 8, INVALID), ("a__q_stride_head", 64, INVALID),
    ("a__kv_stride_tok", 264, INVALID), ("a__kv_stride_head", 120, INVALID), ("a__page_stride", 64 * 256 + 8, INVALID), ("a__lse", 4098, INVALID)])
def test_attention_refuses(name, value, code):
    refused(code, B.cf_attn_paged8_fwd, attend8(**{name: value}))
    assert B.lib().cf_attn_paged8_fwd(None, None) == INVALID and B.lib().cf_attn_paged8_workspace_bytes(None) == INVALID


def test_workspace_sizes_need_no_pointers():
    p = attend8(a__cu_seqlens_q=None, a__kv_lens=None, a__block_table=None, a__q=None, a__k_pages=None, a__v_pages=None, a__o=None, k_scales=None)
    assert B.cf_attn_paged8_workspace_bytes(p) >= 0
