"""CPU tests of the training step's entry points: what they refuse before they
touch a device, with the message's words, and the workspaces they ask for."""
import ctypes
import struct

import pytest

from paper_2607_20652_gb300 import build, dpb

INVALID, UNSUPPORTED = 1, 2
BF16, F32 = 1, 0


@pytest.fixture(scope="module")
def lib():
    build.build()
    return dpb.load()


def attention_config(**kw):
    c = dict(total_q=300, total_k=300, seqs=1, max_q=300, max_k=300, heads_q=4, heads_kv=2, head_dim=64, causal=1, dtype=BF16,
             scale=0.125, reserved=0)
    assert set(kw) <= set(c)
    c.update(kw)
    return ctypes.create_string_buffer(struct.pack("=qq8ifi", *c.values()))


def rope_config(**kw):
    c = dict(tokens=10, heads_q=4, heads_k=2, head_dim=64, rot_dim=64, interleaved=0, normalise=1, positions_n=10, dtype=BF16,
             eps=1e-6, reserved=0)
    assert set(kw) <= set(c)
    c.update(kw)
    return ctypes.create_string_buffer(struct.pack("=q8ifi", *c.values()))


def at(buf):
    return ctypes.addressof(buf)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=F32), UNSUPPORTED), (dict(seqs=-1), INVALID), (dict(total_q=-1), INVALID), (dict(max_k=-1), INVALID),
    (dict(total_k=1 << 31), UNSUPPORTED), (dict(heads_kv=0), INVALID), (dict(heads_q=3), INVALID), (dict(heads_q=0), INVALID),
    (dict(head_dim=4), UNSUPPORTED), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=136), UNSUPPORTED),
    (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID),
])
def test_attention_refuses(lib, change, status):
    c, n = attention_config(**change), ctypes.c_size_t()
    assert lib.dpb_attention_workspace_size(at(c), n) == status
    assert lib.dpb_last_error()
    assert lib.dpb_attention_forward(at(c), *[None] * 8, 0, None) == status
    assert lib.dpb_attention_backward(at(c), *[None] * 12, 0, None) == status


def test_attention_refuses_missing_rows_and_strides(lib):
    c = attention_config()
    assert lib.dpb_attention_workspace_size(None, ctypes.c_size_t()) == INVALID
    assert lib.dpb_attention_workspace_size(at(c), None) == INVALID
    assert lib.dpb_attention_forward(at(c), *[None] * 8, 0, None) == INVALID
    assert b"q is NULL" in lib.dpb_last_error()
    for data, token, head in ((0, 256, 64), (8, 256, 64), (256, 0, 64), (256, 260, 64), (256, 256, 60), (256, 256, -64)):
        q = ctypes.create_string_buffer(struct.pack("=Qqq", data, token, head))
        assert lib.dpb_attention_forward(at(c), at(q), *[None] * 7, 0, None) == INVALID, (data, token, head)
    q = ctypes.create_string_buffer(struct.pack("=Qqq", 256, 1 << 40, 64))
    assert lib.dpb_attention_forward(at(c), at(q), *[None] * 7, 0, None) == UNSUPPORTED


def test_attention_workspace(lib):
    def size(**kw):
        n = ctypes.c_size_t()
        assert lib.dpb_attention_workspace_size(at(attention_config(**kw)), n) == 0
        return n.value

    # rows too short to be shared out: the status word, the lists, fp32 delta
    short = size()
    assert 256 + 300 * 4 * 4 <= short < 256 + 300 * 4 * 4 + 4096
    # long ones: room for the sums of 304 parts of [128][2 x 64] (heads to 64) or [128][2 x 128] fp32
    long = dict(total_q=5000, total_k=5000, max_q=5000, max_k=5000)
    for dim, parts in ((64, 304 * 128 * 128 * 4), (72, 304 * 128 * 256 * 4)):
        assert parts < size(head_dim=dim, **long) < parts + 256 + 5000 * 4 * 4 + (1 << 17)
    # the largest token count does not overflow
    most = (1 << 31) - 256
    assert size(total_q=most, total_k=most, max_q=(1 << 31) - 1, max_k=(1 << 31) - 1) > 4 * 4 * most
    assert size(total_q=0, total_k=0) >= 256


@pytest.mark.parametrize("change", [dict(tokens=-1), dict(heads_q=-1), dict(head_dim=0), dict(rot_dim=65), dict(rot_dim=66),
                                    dict(dtype=7), dict(eps=-1.0), dict(eps=float("nan"))])
def test_norm_and_rotation_refuse(lib, change):
    c = rope_config(**change)
    assert lib.dpb_rope_workspace_size(at(c), ctypes.c_size_t()) in (INVALID, UNSUPPORTED)
    assert lib.dpb_qk_norm_rope(at(c), *[None] * 10, 0, None) in (INVALID, UNSUPPORTED)
    assert lib.dpb_last_error()


@pytest.mark.parametrize("change", [dict(lr=-1.0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0),
                                    dict(weight_decay=float("inf")), dict(step=0), dict(dtype=3), dict(state_bits=16)])
def test_adamw_refuses(lib, change):
    c = dpb.AdamWConfig(1e-3, 0.9, 0.95, 1e-8, 0.1, 1, 0, None, F32, 32)
    for k, v in change.items():
        setattr(c, k, v)
    assert lib.dpb_adamw_step(c, None, 0, None) == INVALID
    assert lib.dpb_last_error()


def test_adamw_refuses_bad_tensors(lib):
    c = dpb.AdamWConfig(1e-3, 0.9, 0.95, 1e-8, 0.1, 1, 0, None, F32, 8)
    assert lib.dpb_adamw_step(c, None, 0, None) == 0  # no tensors: nothing to do
    assert lib.dpb_adamw_step(c, None, 1, None) == INVALID
    assert lib.dpb_adamw_step(c, None, -1, None) == INVALID
    good = [256, 512, 768, 1024, 1280, 1536, 5]
    for i, bad in [(6, -1), (0, 0), (1, 514), (2, 0), (4, 0), (5, 1538)]:
        t = list(good)
        t[i] = bad
        buf = ctypes.create_string_buffer(struct.pack("=6Qq", *t))
        assert lib.dpb_adamw_step(c, ctypes.addressof(buf), 1, None) == INVALID, (i, bad)


def test_status_slots(lib):
    word = ctypes.c_void_p()
    for slot in (-1, 0, 257):
        assert lib.dpb_status_word(slot, word) == INVALID
    assert lib.dpb_status_word(1, None) == INVALID
    for slot in (-1, 257):
        assert lib.dpb_attention_workspace_size(at(attention_config(reserved=slot)), ctypes.c_size_t()) == INVALID
        assert lib.dpb_rope_workspace_size(at(rope_config(reserved=slot)), ctypes.c_size_t()) == INVALID
    rows = ctypes.create_string_buffer(struct.pack("=Qqq", 256, 256, 64))
    forward = [at(rows)] * 3 + [None, None, at(rows), 256]
    # the gradient's scratch is the caller's with any slot, the forward needs a workspace for the status alone
    assert lib.dpb_attention_forward(at(attention_config()), *forward, None, 0, None) == INVALID
    assert b"workspace is NULL" in lib.dpb_last_error()
    backward = [at(rows)] * 4 + [256, at(rows), None, None] + [at(rows)] * 3
    assert lib.dpb_attention_backward(at(attention_config(reserved=1)), *backward, None, 0, None) == INVALID
    assert b"workspace is NULL" in lib.dpb_last_error()


def test_calls_without_a_workspace_share_no_scratch(monkeypatch):
    """Each call's scratch is its own: two threads on one stream, or a graph and a later call, cannot meet in it."""
    assert not hasattr(dpb, "_shared_workspace")
    monkeypatch.setattr(dpb, "_slots", {})
    monkeypatch.setattr("torch._C._cuda_isCurrentStreamCapturing", lambda: False, raising=False)
    import torch
    one, two = dpb._status_slot(torch.device("cuda", 0), 7), dpb._status_slot(torch.device("cuda", 0), 8)
    assert one != two and one == dpb._status_slot(torch.device("cuda", 0), 7) and dpb._GRAPH_SLOT not in (one, two)
    for i in range(300):  # more streams than words: the last is shared
        assert 1 < dpb._status_slot(torch.device("cuda", 1), i) <= dpb.STATUS_SLOTS
    monkeypatch.setattr("torch._C._cuda_isCurrentStreamCapturing", lambda: True, raising=False)
    monkeypatch.setattr(dpb, "_captured", set())
    assert dpb._status_slot(torch.device("cuda", 0), 7) == dpb._GRAPH_SLOT
