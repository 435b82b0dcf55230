"""What the paged cache's further operators refuse (host only): configurations in 4 bits, rotations, calls and tensors that do not fit."""
import ctypes

import pytest
import torch

from paper_2607_24788_b200 import build, glide
from tests.test_paged_host import binding, call, config


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    return glide.load_library()


def workspace(**kw):
    out = ctypes.c_size_t(0)
    cfg = config(**(dict(io_dtype=glide.GLIDE_BF16_CACHE4, weights=0) | kw))
    return glide.load_library().glide_paged_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out))


@pytest.mark.parametrize("kw,code", [
    (dict(), glide.GLIDE_OK), (dict(head_dim=64), glide.GLIDE_OK), (dict(page_size=16), glide.GLIDE_OK), (dict(page_size=256), glide.GLIDE_OK),
    (dict(weights=1), glide.GLIDE_ERR_UNSUPPORTED), (dict(io_dtype=2), glide.GLIDE_ERR_UNSUPPORTED), (dict(io_dtype=3), glide.GLIDE_ERR_UNSUPPORTED),
    (dict(head_dim=96), glide.GLIDE_ERR_UNSUPPORTED), (dict(page_size=8), glide.GLIDE_ERR_UNSUPPORTED),
    (dict(layer_stride=1 << 20, page_stride=1 << 14, head_stride=4352, row_stride=68), glide.GLIDE_OK),
    (dict(layer_stride=1 << 20, page_stride=1 << 14, head_stride=4368, row_stride=68), glide.GLIDE_OK),
    (dict(layer_stride=1 << 20, page_stride=1 << 14, head_stride=4360, row_stride=68), glide.GLIDE_ERR_INVALID_ARG),   # no multiple of 16 bytes
    (dict(layer_stride=1 << 20, page_stride=1 << 14, head_stride=4336, row_stride=68), glide.GLIDE_ERR_INVALID_ARG),   # shorter than a block
    (dict(layer_stride=1 << 20, page_stride=1 << 14, head_stride=4352, row_stride=64), glide.GLIDE_ERR_INVALID_ARG),
    (dict(layer_stride=(1 << 20) + 16, page_stride=1 << 14, head_stride=4352, row_stride=68), glide.GLIDE_ERR_INVALID_ARG)])
def test_configurations_in_4_bits(kw, code):
    assert workspace(**kw) == code


def test_the_strides_of_pages_in_4_bits_are_those_of_the_tensor():
    k = torch.empty(3, 10, 2, 32 * 36 + 16, dtype=torch.uint8)[..., :32 * 36]
    cfg = glide.make_paged_config(k, 4, 2, 100, head_dim=64, weights=False)
    assert (cfg.io_dtype, cfg.page_size, cfg.head_dim, cfg.row_stride) == (glide.GLIDE_BF16_CACHE4, 32, 64, 36)
    assert (cfg.layer_stride, cfg.page_stride, cfg.head_stride) == (10 * 2 * 1168, 2 * 1168, 1168)
    one = glide.make_paged_config(torch.empty(1, 1, 1, 16 * 68, dtype=torch.uint8), 4, 2, 100, head_dim=128, weights=False)
    assert workspace_of(one) == glide.GLIDE_OK
    for bad in (torch.empty(1, 10, 2, 32 * 36 + 1, dtype=torch.uint8), torch.empty(1, 10, 2, 32, 36, dtype=torch.uint8), torch.empty(1, 10, 2, 32 * 36),
                torch.empty(1, 10, 1, 32 * 36, dtype=torch.uint8).expand(1, 10, 2, 32 * 36)):
        with pytest.raises(AssertionError):
            glide.make_paged_config(bad, 4, 2, 100, head_dim=64)


def workspace_of(cfg):
    out = ctypes.c_size_t(0)
    return glide.load_library().glide_paged_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out))


def test_null_handles():
    lib, c = glide.load_library(), ctypes.byref(call())
    assert lib.glide_paged_append(None, c, None, None, 4096, 4096, None, None) == glide.GLIDE_ERR_INVALID_ARG
    assert lib.glide_paged_read(None, c, 4096, 4096, None) == glide.GLIDE_ERR_INVALID_ARG
    assert lib.glide_paged_bounds(None, c, 4096, None) == glide.GLIDE_ERR_INVALID_ARG
    assert lib.glide_paged_decode_sparse(None, c, 4096, None, None, 4096, None, 4096, 4, 4096, 4096, None) == glide.GLIDE_ERR_INVALID_ARG


def test_a_context_is_not_held_in_4_bits():
    cfg = glide.glide_config(n_layers=1, batch=1, n_q_heads=4, n_kv_heads=4, head_dim=64, io_dtype=glide.GLIDE_BF16_CACHE4, max_tokens=64,
                             windows=(ctypes.c_int64 * 1)(16))
    out = ctypes.c_size_t(0)
    assert glide.load_library().glide_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out)) != glide.GLIDE_OK


def test_angles_that_do_not_fit():
    cos = torch.zeros(10, 16)
    r = glide.glide_rotation.from_buffer_copy(glide.GlideRotation(cos, cos.clone(), neighbours=True).packed)
    assert (r.n_positions, r.stride, r.rot_dim, r.neighbours) == (10, 16, 32, 1)
    wide = torch.zeros(10, 40)
    r = glide.glide_rotation.from_buffer_copy(glide.GlideRotation(wide[:, :16], wide[:, 20:36]).packed)
    assert (r.stride, r.neighbours) == (40, 0)
    for a, b in ((cos, torch.zeros(9, 16)), (cos, cos.double()), (cos.t(), cos.t()), (cos[:1].expand(10, 16), cos[:1].expand(10, 16)), (cos[0], cos[0])):
        with pytest.raises(AssertionError):
            glide.GlideRotation(a, b)


def test_tensors_that_do_not_fit():
    h = binding()
    h.lib, h.n_pages, h.page_size, h.max_tokens = glide.load_library(), 8, 16, 64
    table, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    q, k = torch.zeros(2, 4, 64), torch.zeros(2, 2, 64)
    bounds, picks, scores = torch.zeros(8, 2, 2, 64), torch.zeros(2, 2, 3, dtype=torch.int32), torch.zeros(2, 2, 4, dtype=torch.float64)
    with pytest.raises(AssertionError):
        h.glide_paged_append(table, lens, None, q, k, k)                        # q without q_out
    with pytest.raises(AssertionError):
        h.glide_paged_append(table, lens, None, None, k[:1], k[:1])             # a row for each sequence
    with pytest.raises(AssertionError):
        h.glide_paged_read(table, lens, None, k[:1], k[:1])
    for b, p, s in ((bounds[:7], picks, scores), (bounds.double(), picks, scores), (bounds, picks[:1], scores), (bounds, picks.long(), scores),
                    (bounds, picks, scores.float()), (bounds, picks, scores[..., :3])):
        with pytest.raises(AssertionError):
            h.glide_paged_decode_sparse(table, lens, q, k, k, q, b, p, s)
