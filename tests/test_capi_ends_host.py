"""CPU tests of the entry points at both ends of the model: what they refuse
before they touch a device, and the workspaces they ask for."""
import ctypes
import struct

import pytest

from paper_2607_20652_gb300 import build, dpb

INVALID, UNSUPPORTED = 1, 2
BF16, F32 = 1, 0
MOST = (1 << 31) - 256


@pytest.fixture(scope="module")
def lib():
    build.build()
    return dpb.load()


def packed(form, defaults, kw):
    assert set(kw) <= set(defaults)
    return ctypes.create_string_buffer(struct.pack(form, *(defaults | kw).values()))


def loss_config(**kw):
    return packed("=qiiqiiii", dict(tokens=300, vocab=700, dim=64, ignore_index=-100, index_bytes=8, dtype=BF16, grad_stride=1,
                                    status_slot=0), kw)


def embedding_config(**kw):
    return packed("=qiiiifi", dict(tokens=300, vocab=700, dim=64, index_bytes=8, dtype=BF16, scale=1.0, status_slot=0), kw)


def norm_config(**kw):
    return packed("=qiifi", dict(tokens=300, dim=64, dtype=BF16, eps=1e-6, reserved=0), kw)


def at(buf):
    return ctypes.addressof(buf)


def rows(data, stride):
    return ctypes.create_string_buffer(struct.pack("=Qq", data, stride))


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), INVALID), (dict(vocab=0), INVALID), (dict(dim=0), INVALID), (dict(dim=60), UNSUPPORTED),
    (dict(tokens=(1 << 24) + 1), UNSUPPORTED), (dict(vocab=(1 << 28) + 1), UNSUPPORTED),
    (dict(tokens=1 << 24, vocab=1 << 20), UNSUPPORTED), (dict(dtype=F32), UNSUPPORTED), (dict(index_bytes=2), INVALID), (dict(grad_stride=2), INVALID), (dict(grad_stride=-1), INVALID), (dict(status_slot=-1), INVALID),
    (dict(status_slot=257), INVALID)])
def test_loss_refuses(lib, change, status):
    c, n = loss_config(**change), ctypes.c_size_t()
    for backward in (0, 1):
        assert lib.dpb_linear_cross_entropy_workspace_size(at(c), backward, n) == status
    assert lib.dpb_linear_cross_entropy_forward(at(c), *[None] * 7, 0, None) == status
    assert lib.dpb_linear_cross_entropy_backward(at(c), *[None] * 8, 0, None) == status
    assert lib.dpb_last_error()


def test_loss_refuses_missing_rows_and_strides(lib):
    c = loss_config()
    assert lib.dpb_linear_cross_entropy_workspace_size(None, 0, ctypes.c_size_t()) == INVALID
    assert lib.dpb_linear_cross_entropy_workspace_size(at(c), 0, None) == INVALID
    good = rows(256, 64)
    for bad in (None, rows(0, 64), rows(8, 64), rows(256, 56), rows(256, 68), rows(256, -64)):
        b = None if bad is None else at(bad)
        assert lib.dpb_linear_cross_entropy_forward(at(c), b, at(good), 256, 256, 256, None, None, 0, None) == INVALID
        assert lib.dpb_linear_cross_entropy_forward(at(c), at(good), b, 256, 256, 256, None, None, 0, None) == INVALID
        assert lib.dpb_linear_cross_entropy_backward(at(c), b, at(good), 256, 256, 256, at(good), None, None, 0, None) == INVALID
        if bad is not None:
            assert lib.dpb_linear_cross_entropy_backward(at(c), at(good), at(good), 256, 256, 256, b, None, None, 0, None) == INVALID
            assert lib.dpb_linear_cross_entropy_backward(at(c), at(good), at(good), 256, 256, 256, None, b, None, 0, None) == INVALID
    wide = rows(256, 1 << 38)
    assert lib.dpb_linear_cross_entropy_forward(at(c), at(wide), at(good), 256, 256, 256, None, None, 0, None) == UNSUPPORTED
    for k in range(3):  # targets, loss, lse
        p = [256, 256, 256]
        for bad in (0, 258):
            p[k] = bad
            assert lib.dpb_linear_cross_entropy_forward(at(c), at(good), at(good), *p, None, None, 0, None) == INVALID
    # the workspace: none, at an odd address, too small
    n = ctypes.c_size_t()
    assert lib.dpb_linear_cross_entropy_workspace_size(at(c), 0, n) == 0
    for ws, size in ((None, n.value), (128, n.value), (256, n.value - 1)):
        for slot in (0, 3):
            c = loss_config(status_slot=slot)
            assert lib.dpb_linear_cross_entropy_forward(at(c), at(good), at(good), 256, 256, 256, None, ws, size, None) == INVALID
            assert b"workspace" in lib.dpb_last_error()


def test_loss_workspace(lib):
    def size(backward, **kw):
        n = ctypes.c_size_t()
        assert lib.dpb_linear_cross_entropy_workspace_size(at(loss_config(**kw)), backward, n) == 0
        return n.value

    # far below the tokens x vocabulary scores, in bf16, of a training step
    step = dict(tokens=65536, vocab=50257, dim=768)
    assert size(0, **step) < 65536 * 50257 * 2 / 8 and size(1, **step) < 65536 * 50257 * 2 / 3
    assert size(1, tokens=1 << 24, vocab=50257, dim=1 << 13) > (1 << 39)  # nothing overflows
    assert size(0, tokens=0) >= 256


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), INVALID), (dict(vocab=0), INVALID), (dict(dim=0), INVALID), (dict(tokens=1 << 31), UNSUPPORTED),
    (dict(vocab=MOST + 1), UNSUPPORTED), (dict(dim=(1 << 20) + 1), UNSUPPORTED), (dict(dtype=2), INVALID),
    (dict(index_bytes=1), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(status_slot=300), INVALID)])
def test_embedding_refuses(lib, change, status):
    c = embedding_config(**change)
    assert lib.dpb_embedding_workspace_size(at(c), ctypes.c_size_t()) == status
    assert lib.dpb_embedding(at(c), None, None, None, None, 0, None) == status
    assert lib.dpb_embedding_backward(at(c), None, None, None, None, 0, None) == status


def test_embedding_refuses_missing_rows_and_strides(lib):
    c, good = embedding_config(), rows(256, 64)
    for bad in (None, rows(0, 64), rows(257, 64), rows(256, 63)):
        b = None if bad is None else at(bad)
        for f in (lib.dpb_embedding, lib.dpb_embedding_backward):
            assert f(at(c), b, 256, at(good), None, 0, None) == INVALID
            assert f(at(c), at(good), 256, b, None, 0, None) == INVALID
    n = ctypes.c_size_t()
    assert lib.dpb_embedding_workspace_size(at(c), n) == 0
    for f, need in ((lib.dpb_embedding, 256), (lib.dpb_embedding_backward, n.value)):
        for ids in (0, 260):
            assert f(at(c), at(good), ids, at(good), 256, need, None) == INVALID
        assert f(at(c), at(good), 256, at(good), 256, need - 1, None) == INVALID
    assert lib.dpb_embedding_workspace_size(at(embedding_config(tokens=MOST, dim=1 << 20)), n) == 0
    assert n.value > MOST * 16 + (MOST // 256 << 22)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), INVALID), (dict(dim=0), INVALID), (dict(dim=16385), UNSUPPORTED), (dict(tokens=(1 << 40) + 1), UNSUPPORTED),
    (dict(dtype=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("inf")), INVALID), (dict(eps=float("nan")), INVALID)])
def test_norm_refuses(lib, change, status):
    c = norm_config(**change)
    assert lib.dpb_norm_workspace_size(at(c), ctypes.c_size_t()) == status
    assert lib.dpb_add_norm(at(c), *[None] * 6) == status
    assert lib.dpb_add_norm_backward(at(c), *[None] * 7, 0, None) == status


def test_norm_refuses_missing_rows_and_strides(lib):
    c, good = norm_config(), rows(256, 64)
    for bad in (None, rows(0, 64), rows(257, 64), rows(256, 63)):
        b = None if bad is None else at(bad)
        assert lib.dpb_add_norm(at(c), b, None, None, at(good), None, None) == INVALID
        assert lib.dpb_add_norm(at(c), at(good), None, None, b, None, None) == INVALID
        assert lib.dpb_add_norm_backward(at(c), b, at(good), None, None, at(good), None, None, 0, None) == INVALID
        assert lib.dpb_add_norm_backward(at(c), at(good), b, None, None, at(good), None, None, 0, None) == INVALID
        assert lib.dpb_add_norm_backward(at(c), at(good), at(good), None, None, b, None, None, 0, None) == INVALID
        if bad is not None:
            assert lib.dpb_add_norm(at(c), at(good), b, None, at(good), None, None) == INVALID
            assert lib.dpb_add_norm(at(c), at(good), None, None, at(good), b, None) == INVALID
            assert lib.dpb_add_norm_backward(at(c), at(good), at(good), b, None, at(good), None, None, 0, None) == INVALID
    assert lib.dpb_add_norm(at(c), at(good), None, 257, at(good), None, None) == INVALID
    # the weight's gradient needs its address and a workspace
    assert lib.dpb_add_norm_backward(at(c), at(good), at(good), None, None, at(good), 258, 256, 1 << 20, None) == INVALID
    assert lib.dpb_add_norm_backward(at(c), at(good), at(good), None, None, at(good), 256, None, 0, None) == INVALID


def test_the_model_refuses_what_the_operators_do():
    from paper_2607_20652_gb300.transformer import ParityTransformer
    import torch
    at = dict(layers=1, d=64, heads=4, d_mlp=128, vocab=97, context=32)
    for kw in (dict(ends="other"), dict(ends="dpb", dtype=torch.float32), dict(ends="dpb", d=60)):
        with pytest.raises(ValueError):
            ParityTransformer(**(at | kw))
    plain = ParityTransformer(**at)
    assert plain.ends == "torch" and ParityTransformer(**at, ends="dpb").state_dict().keys() == plain.state_dict().keys()


def test_functions_want_cuda_tensors():
    import torch
    x, ids = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.long)
    for f in (lambda: dpb.embedding(x, ids), lambda: dpb.embedding_backward(x, ids, 9), lambda: dpb.add_norm(x),
              lambda: dpb.add_norm_backward(x, x), lambda: dpb.linear_cross_entropy_forward(x, x, ids),
              lambda: dpb.linear_cross_entropy_backward(x, x, ids, x, x)):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            f()


@pytest.mark.parametrize("dim", [(1 << 20) + 8, 1 << 24, (1 << 31) - 1024, (1 << 31) - 8])
def test_loss_refuses_rows_that_are_too_wide(lib, dim):
    """A unit's products over such a row would outlast the waits for them, and the last of these sizes overflow its tiles."""
    n = ctypes.c_size_t()
    c, good = loss_config(tokens=1, vocab=1, dim=dim), rows(256, dim)
    for backward in (0, 1):
        assert lib.dpb_linear_cross_entropy_workspace_size(at(c), backward, n) == UNSUPPORTED
    assert lib.dpb_linear_cross_entropy_forward(at(c), at(good), at(good), 256, 256, 256, None, 256, 1 << 62, None) == UNSUPPORTED
    assert lib.dpb_linear_cross_entropy_backward(at(c), at(good), at(good), 256, 256, 256, at(good), at(good), 256, 1 << 62,
                                                 None) == UNSUPPORTED
    assert b"columns" in lib.dpb_last_error()
    for backward in (0, 1):
        assert lib.dpb_linear_cross_entropy_workspace_size(at(loss_config(tokens=1, vocab=1, dim=1 << 20)), backward, n) == 0


def test_a_workspace_of_another_place_is_refused():
    """Memory of the host or with repeats: its address and size would not be what the kernels write to."""
    import torch
    there, ws = torch.device("cuda", 0), torch.zeros(1 << 10, dtype=torch.uint8)
    with pytest.raises(ValueError, match="workspace"):
        dpb._space(ws, there)
    for bad in (ws[:1].expand(1 << 20), ws[::2]):
        with pytest.raises(ValueError, match="workspace"):
            dpb._space(bad, ws.device)
    assert dpb._space(None, there) == (None, 0) and dpb._space(ws, ws.device) == (ws.data_ptr(), 1 << 10)


@pytest.mark.parametrize("tokens", [1, 33, 512, 1000, 4096, 8192, 65536, 262144])
@pytest.mark.parametrize("vocab", [50, 1000, 5003, 9001, 12288, 50257, 1 << 20])
def test_the_gradients_scratch_is_what_is_said(lib, tokens, vocab):
    """dz of three pieces, 192 MB or 24 KB a token, or 3/160 of a large vocabulary, and never more than all of it; beside
    it rows of the tokens (closed up, bf16; sums in fp32, apart for up to 160 pieces where all of dz is held, which is where
    dz has 192 MB at most) and sums of dW for parts of the tokens, of fewer tiles than half the multiprocessors."""
    dim, n = 768, ctypes.c_size_t()
    assert lib.dpb_linear_cross_entropy_workspace_size(at(loss_config(tokens=tokens, vocab=vocab, dim=dim)), 1, n) == 0
    T, V, mb = -(-tokens // 256) * 256, -(-vocab // 256) * 256, 1 << 20
    piece = max(12288, -(-3 * vocab // 160) + 768)
    dz = min(max(192 * mb, 2 * T * min(V, piece)), 2 * T * V * (2 if T <= 512 else 1))
    held = 2 * T * V <= 192 * mb
    tiles = (T // 256) * 3
    # pieces whose sums are apart: two units a pair of blocks, each unit a tile of fp32 sums
    sums = min(152 * 256 * 1024 + tiles * 256 * 1024, 160 * tiles * 256 * 1024) if held else T * dim * 4
    parts = 76 * 256 * 1024 + V * dim * 4
    assert n.value <= dz + sums + parts + T * (dim * 2 + 20) + 64 * 1024
