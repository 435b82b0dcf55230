"""What the paged attention refuses, and the workspace it asks for (host only)."""
import contextlib
import ctypes

import pytest
import torch

from paper_2607_24788_b200 import build, glide


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    return glide.load_library()


def config(**kw):
    d = dict(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=128, io_dtype=glide.GLIDE_BF16, page_size=64, n_pages=100, max_batch=4,
             max_tokens=1000, softmax_scale=0.0, weights=1)
    return glide.glide_paged_config(**(d | kw))


def workspace(**kw):
    out = ctypes.c_size_t(0)
    return glide.load_library().glide_paged_workspace_bytes(ctypes.byref(config(**kw)), ctypes.byref(out)), out.value


@pytest.mark.parametrize("kw,code", [
    (dict(), glide.GLIDE_OK), (dict(head_dim=64), glide.GLIDE_OK), (dict(io_dtype=glide.GLIDE_F32), glide.GLIDE_OK), (dict(max_batch=1024), glide.GLIDE_OK),
    (dict(n_layers=0), glide.GLIDE_ERR_INVALID_ARG), (dict(n_pages=0), glide.GLIDE_ERR_INVALID_ARG), (dict(max_batch=0), glide.GLIDE_ERR_INVALID_ARG),
    (dict(max_tokens=0), glide.GLIDE_ERR_INVALID_ARG), (dict(max_tokens=(1 << 30) + 1), glide.GLIDE_ERR_INVALID_ARG),
    (dict(softmax_scale=-1.0), glide.GLIDE_ERR_INVALID_ARG), (dict(softmax_scale=float("nan")), glide.GLIDE_ERR_INVALID_ARG),
    (dict(softmax_scale=float("inf")), glide.GLIDE_ERR_INVALID_ARG), (dict(weights=2), glide.GLIDE_ERR_INVALID_ARG),
    (dict(head_dim=96), glide.GLIDE_ERR_UNSUPPORTED), (dict(io_dtype=7), glide.GLIDE_ERR_UNSUPPORTED), (dict(n_q_heads=6), glide.GLIDE_ERR_UNSUPPORTED),
    (dict(n_q_heads=32), glide.GLIDE_ERR_UNSUPPORTED), (dict(n_q_heads=7), glide.GLIDE_ERR_UNSUPPORTED), (dict(page_size=8), glide.GLIDE_ERR_UNSUPPORTED),
    (dict(page_size=48), glide.GLIDE_ERR_UNSUPPORTED), (dict(page_size=512), glide.GLIDE_ERR_UNSUPPORTED), (dict(max_batch=1025), glide.GLIDE_ERR_UNSUPPORTED),
    (dict(max_tokens=1 << 30, max_batch=512), glide.GLIDE_ERR_UNSUPPORTED),
    (dict(layer_stride=1 << 24, page_stride=1 << 15, head_stride=1 << 13, row_stride=128), glide.GLIDE_OK),
    (dict(layer_stride=1 << 24, page_stride=1 << 15, head_stride=1 << 13, row_stride=132), glide.GLIDE_ERR_INVALID_ARG),
    (dict(layer_stride=1 << 24, page_stride=1 << 15, head_stride=1 << 13, row_stride=64), glide.GLIDE_ERR_INVALID_ARG),
    (dict(layer_stride=(1 << 24) + 128, page_stride=1 << 15, head_stride=1 << 13, row_stride=128), glide.GLIDE_ERR_INVALID_ARG),
    (dict(page_stride=1 << 15), glide.GLIDE_ERR_INVALID_ARG), (dict(layer_stride=-(1 << 24)), glide.GLIDE_ERR_INVALID_ARG)])
def test_configurations(kw, code):
    assert workspace(**kw)[0] == code


def test_workspace_holds_a_steps_scores_only_where_weights_are_kept():
    a, b = workspace(weights=1)[1], workspace(weights=0)[1]
    assert abs(a - b - 4 * 8 * 1000 * 4) <= 512
    assert workspace(max_tokens=4000)[1] - workspace(max_tokens=2000)[1] == pytest.approx(4 * 8 * 2000 * 4, abs=512)
    # beyond 1024 tokens: the records of prompts of few rows behind long caches
    assert workspace(weights=0, max_tokens=1025)[1] - workspace(weights=0, max_tokens=1024)[1] <= 16384 * (128 + 4) * 4


def call(**kw):
    d = dict(layer=0, batch=2, dev_table=4096, table_cols=4, table_stride=4, dev_lens=4096, window=-1, n_sink=0)
    return glide.glide_paged_call(**(d | kw))


@pytest.mark.parametrize("kw,ok", [
    (dict(), True), (dict(layer=1), True), (dict(batch=4), True), (dict(table_stride=100), True), (dict(dev_starts=4096, n_tokens=0), True),
    (dict(window=0), True), (dict(window=1 << 60), True), (dict(n_sink=1 << 30), True), (dict(q_stride=8 * 128 + 8), True),
    (dict(dev_weight=4096, track_stride=256), True),
    (dict(layer=2), False), (dict(layer=-1), False), (dict(batch=0), False), (dict(batch=5), False), (dict(dev_table=None), False),
    (dict(table_cols=0), False), (dict(table_stride=3), False), (dict(dev_lens=None), False), (dict(n_sink=-1), False),
    (dict(dev_starts=4096, n_tokens=-1), False), (dict(q_stride=8 * 128 - 8), False), (dict(q_stride=8 * 128 + 4), False),
    (dict(kv_stride=2 * 128 - 8), False), (dict(out_stride=4), False), (dict(dev_weight=4096, track_stride=255), False), (dict(dev_pos=4096), False)])
def test_calls(kw, ok):
    got = glide.load_library().glide_paged_check_call(ctypes.byref(config()), ctypes.byref(call(**kw)))
    assert got == (glide.GLIDE_OK if ok else glide.GLIDE_ERR_INVALID_ARG)


def test_null_arguments():
    lib = glide.load_library()
    out = ctypes.c_void_p()
    assert lib.glide_paged_workspace_bytes(None, None) == glide.GLIDE_ERR_INVALID_ARG
    assert lib.glide_paged_check_call(ctypes.byref(config()), None) == glide.GLIDE_ERR_INVALID_ARG
    assert lib.glide_paged_create(ctypes.byref(config()), 4096, 4096, None, 1 << 30, None, ctypes.byref(out)) == glide.GLIDE_ERR_INVALID_ARG
    assert lib.glide_paged_create(ctypes.byref(config()), 4096, 4096, 4096, 1, None, ctypes.byref(out)) == glide.GLIDE_ERR_WORKSPACE_TOO_SMALL
    assert lib.glide_paged_create(ctypes.byref(config()), 4096, 4100, 4096, 1 << 40, None, ctypes.byref(out)) == glide.GLIDE_ERR_INVALID_ARG
    assert lib.glide_paged_create(ctypes.byref(config()), 4096, 4096, 4097, 1 << 40, None, ctypes.byref(out)) == glide.GLIDE_ERR_INVALID_ARG
    assert not out.value
    for f in (lib.glide_paged_prefill, lib.glide_paged_decode):
        assert f(None, ctypes.byref(call()), 4096, None, None, 4096, None, None) == glide.GLIDE_ERR_INVALID_ARG
    assert lib.glide_paged_weights(None, ctypes.byref(call()), 4096, 4096, None) == glide.GLIDE_ERR_INVALID_ARG
    assert lib.glide_paged_evict(None, ctypes.byref(call()), 1, 0, 4096, 4096, 4096, None) == glide.GLIDE_ERR_INVALID_ARG
    assert lib.glide_paged_device_status(None, None, None) == glide.GLIDE_ERR_INVALID_ARG
    assert lib.glide_paged_destroy(None) == glide.GLIDE_ERR_INVALID_ARG


def test_the_pages_strides_are_those_of_the_tensor():
    k = torch.empty(3, 10, 32, 2, 64).transpose(2, 3)
    cfg = glide.make_paged_config(k, 4, 2, 100)
    assert (cfg.layer_stride, cfg.page_stride, cfg.head_stride, cfg.row_stride) == (40960, 4096, 64, 128)
    assert (cfg.n_layers, cfg.n_pages, cfg.n_kv_heads, cfg.page_size, cfg.head_dim) == (3, 10, 2, 32, 64)


def binding(H=4, Hkv=2, d=64):
    """A GlidePaged without a handle, whose tensors live on the host: what it checks and packs before the library is called."""
    h = object.__new__(glide.GlidePaged)
    h.device, h._index, h.dtype, h.H, h.Hkv, h.d, h._h = torch.device("cpu"), -1, torch.float32, H, Hkv, d, None
    return h


def test_rows_that_share_memory_are_refused():
    """A token stride of 0 (an expanded view) says "side by side" to the library, which would read and write behind the tensor."""
    h = binding()
    row = torch.zeros(1, 4, 64)
    assert h._rows(row, 1, 4, "q")[1] == 0
    assert h._rows(row.expand(1, 4, 64), 1, 4, "q")[1] == 0
    assert h._rows(torch.zeros(5, 6, 64)[:, :4], 5, 4, "q")[1] == 6 * 64
    assert h._rows(torch.zeros(5, 4, 64)[:, ::4], 5, 1, "k")[1] == 4 * 64
    for shared in (row.expand(5, 4, 64), torch.zeros(9 * 64).as_strided((5, 4, 64), (64, 64, 1))):
        with pytest.raises(AssertionError):
            h._rows(shared, 5, 4, "q")
    with pytest.raises(AssertionError):
        h._rows(torch.zeros(1, 1, 64).expand(5, 1, 64), 5, 1, "k")
    with pytest.raises(AssertionError):
        h._qkv(torch.zeros(5, 4, 64), None, None, row.expand(5, 4, 64), 5)


def test_pages_that_share_memory_are_refused():
    """Strides that are all 0 say "side by side" too."""
    row = torch.zeros(64)
    for shape in ((1, 8, 2, 16, 64), (3, 8, 2, 16, 64)):
        with pytest.raises(AssertionError):
            glide.make_paged_config(row.expand(shape), 4, 2, 100)


def test_calls_of_one_object_from_two_threads():
    """A second thread's call that comes while the library reads the first one's fields does not change them."""
    import threading
    h = binding()
    lens, seen = torch.zeros(2, dtype=torch.int32), []
    tables = [torch.zeros(2, 3 + i, dtype=torch.int32) for i in range(2)]
    q, k = torch.zeros(2, 4, 64), torch.zeros(2, 2, 64)

    def step(i):
        h.glide_paged_decode(tables[i], lens, q, k, k, q, layer=i, stream=type("Stream", (), dict(cuda_stream=0))())

    class Library:
        @staticmethod
        def glide_paged_decode(handle, call, *rest):
            if not seen:
                seen.append(None)
                other = threading.Thread(target=step, args=(1,))
                other.start()
                other.join()
            address = call if isinstance(call, int) else ctypes.cast(ctypes.c_char_p(call), ctypes.c_void_p).value
            fields = glide.glide_paged_call.from_buffer_copy(ctypes.string_at(address, ctypes.sizeof(glide.glide_paged_call)))
            seen.append((fields.layer, fields.table_cols, fields.dev_table))
            return 0

    h.lib, h._index = Library, -1
    current = glide._current_device
    glide._current_device = lambda: -1
    try:
        step(0)
    finally:
        glide._current_device = current
    assert seen[1:] == [(1, 4, tables[1].data_ptr()), (0, 3, tables[0].data_ptr())]


def test_the_status_is_that_of_the_stream_it_is_asked_for(monkeypatch):
    """Read on another stream, it could come before the calls have recorded anything, and clear what they record."""
    h, asked = binding(), []

    class Library:
        @staticmethod
        def glide_paged_device_status(handle, stream, out):
            asked.append(stream)
            return 0

    h.lib = Library
    monkeypatch.setattr(glide.torch.cuda, "device", lambda _: contextlib.nullcontext())
    assert h.glide_paged_device_status(stream=type("Stream", (), dict(cuda_stream=77))()) == 0
    assert asked == [77]
