"""The paged 8-bit cache on the CPU: the oracle's pieces against other ways to say the same, and what the library refuses."""
import ctypes
import functools
import os

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O
from paper_2503_18773_amd import binding as B

needs_lib = pytest.mark.skipif(not os.path.exists(B._LIB_PATH), reason="libbitdecode.so not built")


def test_rounding_to_e4m3_and_halves():
    y = np.concatenate([np.linspace(-460, 460, 40001), np.linspace(-0.05, 0.05, 40001), np.float64(2.0) ** np.arange(-14, 9) * 1.0625])
    assert np.array_equal(O.round_e4m3(y.astype(np.float32)), torch.from_numpy(np.clip(y, -448, 448).astype(np.float32)).to(torch.float8_e4m3fn).double().numpy())
    x = np.random.default_rng(0).standard_normal(20000) * 10.0 ** np.random.default_rng(1).integers(-9, 4, 20000)
    for dtype, t in (("fp16", torch.float16), ("bf16", torch.bfloat16)):
        assert np.array_equal(O.round_half(x, dtype), torch.from_numpy(x).float().to(t).double().numpy())


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_relative_angles(interleaved):
    rng = np.random.default_rng(2)
    t = B.Rotation.table(64, 32, device="cpu").numpy()
    assert t.shape == (64, 32) and np.allclose(t[:, :16] ** 2 + t[:, 16:] ** 2, 1, atol=1e-6)
    x = rng.standard_normal((1, 1, 48)).astype(np.float16).astype(np.float64)
    y = rng.standard_normal((1, 1, 48)).astype(np.float16).astype(np.float64)
    turn = lambda z, p: O.rotate(z, t[p:p + 1, :16], t[p:p + 1, 16:], interleaved, "fp16")   # noqa: E731
    assert np.array_equal(turn(x, 0), x) and np.array_equal(turn(x, 9)[..., 32:], x[..., 32:])
    dots = [float((turn(x, p + 7) * turn(y, p)).sum()) for p in (0, 11, 50)]   # of the distance alone
    assert np.ptp(dots) < 48 * 2 ** -10 * np.linalg.norm(x) * np.linalg.norm(y) / 7


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_appending_in_pieces_is_appending_at_once(code):
    rng = np.random.default_rng(3)
    k, v = (rng.standard_normal((700, 2, 64)).astype(np.float16) for _ in range(2))
    caches = []
    for pieces in ([700], [1, 126, 1, 1, 300, 128, 143]):
        c = O.Cache(1, 2, 64, code, "fp16", 6, [[5, 0, 3, 2, 1, 4]])
        for n in pieces:
            at = c.lens[0]
            c.append(0, k[at:at + n], v[at:at + n])
            c.lens[0] += n
        caches.append(c)
    a, b = caches
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        assert np.array_equal(getattr(a, name), getattr(b, name), equal_nan=True)
    x, _, there = a.values(0, 700)
    assert there.all() and np.array_equal(x[:, 640:], k[640:].transpose(1, 0, 2).astype(np.float64))
    step = np.abs(k[:640].astype(np.float64)).max() / O.MOST[code] * (0.5 if code == "int8" else 16)
    assert np.abs(x[:, :640] - k[:640].transpose(1, 0, 2)).max() <= step * 1.0001


def test_attention_against_softmax_of_the_whole():
    rng = np.random.default_rng(4)
    c = O.Cache(1, 2, 64, "int8", "fp16", 3, [[2, 0, 1]])
    k, v = (rng.standard_normal((300, 2, 64)).astype(np.float16) for _ in range(2))
    c.append(0, k, v)
    q = rng.standard_normal((5, 4, 64)).astype(np.float16)
    kv, vv, _ = c.values(0, 300)
    out, spread, _, _ = O.attention(c, 0, q, 295, 0.125)
    s = torch.from_numpy(np.einsum("thd,hjd->htj", q.astype(np.float64), kv.repeat(2, 0))) * 0.125
    s = s.masked_fill(torch.arange(300)[None] > torch.arange(295, 300)[:, None], -np.inf)
    want = torch.softmax(s, -1).numpy() @ vv.repeat(2, 0)
    assert np.allclose(out, want.transpose(1, 0, 2), atol=1e-12) and (spread >= np.abs(out) - 1e-12).all()
    # a window of one sees itself alone; a prefix is seen by all; nothing there: zeros
    out, _, _, _ = O.attention(c, 0, q, 295, 0.125, window=1)
    assert np.allclose(out, vv.repeat(2, 0)[:, 295:].transpose(1, 0, 2))
    a = O.attention(c, 0, q, 295, 0.125, prefix=300, window=1)[0]
    assert np.allclose(a, O.attention(c, 0, q, 295, 0.125, prefix=299)[0], atol=0.5) and not np.allclose(a, out)
    c.table = np.array([[-1, 3, 99]])
    c.lens[0] = 0
    assert (O.attention(c, 0, q[:1], 255, 0.125)[0] == 0).all()


def _desc(**kw):
    d = dict(batch=4, n_q_heads=8, n_kv_heads=2, head_dim=128, code_type=0, elem_type=0, num_pages=16, max_pages_per_seq=4)
    d.update(kw)
    c = B.bd_paged8_cache(**d)
    for name in ("k_codes", "v_codes", "k_scales", "v_scales", "k_res", "v_res", "block_table", "seq_lens"):
        setattr(c, name, 4096)   # (never read: every call here is refused before a launch)
    return c


@needs_lib
def test_sizes_and_splits():
    c = _desc()
    assert [B.bd_paged8_cache_bytes(c, i) for i in range(9)] == [16 * 2 * 128 * 128] * 2 + [16 * 2 * 4] * 2 + [4 * 2 * 128 * 128 * 2] * 2 + [64, 16, 0]
    for bad in (dict(head_dim=96), dict(head_dim=256), dict(code_type=2), dict(elem_type=-1), dict(n_q_heads=7), dict(batch=0), dict(num_pages=0),
                dict(max_pages_per_seq=-1), dict(batch=65536), dict(n_q_heads=32768)):
        assert B.bd_paged8_cache_bytes(_desc(**bad), 0) == 0
    assert B.bd_paged8_cache_bytes(c, -1) == 0
    # counters, then a row and split each: of few rows for every sequence, in up to 128 splits
    size = lambda *a: B.bd_paged8_workspace_bytes(c, *a) - 65536   # noqa: E731
    assert B.bd_paged8_workspace_bytes(c, 10, 4, 1) == B.bd_paged8_workspace_bytes(c, 0, 4, 3) == B.bd_paged8_workspace_bytes(c, 9, 0, 3) == 0
    assert size(4, 1, 3) >= 3 * 4 * 2 * 4 * 130 * 4 and size(20, 5, 3) >= 3 * 4 * 2 * 20 * 130 * 4
    wide = _desc(n_q_heads=34)   # (17 a group: without cu_tokens the rows are few, whatever is said of max_tokens)
    assert B.bd_paged8_workspace_bytes(wide, 4, 100, 3) - 65536 >= 3 * 4 * 2 * 17 * 130 * 4
    assert size(4, 1, 128) == size(4, 1, 9999) == 128 * 32 * 130 * 4 and size(500, 200, 3) == 3 * 500 * 8 * 130 * 4
    assert "#define BD_PAGED8_COUNTER_BYTES 65536\n" in open(os.path.join(os.path.dirname(B._LIB_PATH), "..", "include", "bitdecode.h")).read()
    for tokens in (1, 3, 17, 300, 5000):
        for length in (1, 128, 129, 5000, 1 << 20, 2 ** 31 - 1):
            assert 1 <= B.bd_paged8_choose_splits(c, tokens, length) <= (length + 127) // 128
    assert B.bd_paged8_choose_splits(c, 0, 100) == B.bd_paged8_choose_splits(c, 1, 0) == 1


@needs_lib
def test_what_is_refused_before_anything_is_launched():
    L, c = B.lib(), _desc()
    ok = B.bd_rows(4096, 1024, 128)
    rot = B.bd_rotation(4096, None, 100, 64, 0)

    def append(c=c, k=ok, v=ok, q=None, q_out=None, cu=4096, total=4, most=4, rot=None):
        r = lambda x: None if x is None else ctypes.byref(x)   # noqa: E731
        return L.bd_paged8_append(r(c), r(k), r(v), r(q), r(q_out), cu, total, most, r(rot), None)

    rows = lambda *a: B.bd_rows(*a)   # noqa: E731
    assert append(c=None) == append(k=None) == append(v=rows(None, 8, 8)) == -1
    assert append(total=-1) == append(most=0) == append(cu=None, total=3) == -1
    assert append(k=rows(4096, -8, 8)) == append(q=ok, q_out=None, rot=rot) == append(q=ok, q_out=ok) == append(q_out=ok, rot=rot) == -1
    assert append(k=rows(4100, 8, 8)) == append(v=rows(4096, 12, 8)) == append(v=rows(4096, 8, 4)) == append(cu=4098) == -3
    assert append(q=ok, q_out=rows(4096, 0, 128), rot=rot) == append(q=ok, q_out=rows(4096, 1024, 64), rot=rot) == -1   # rows on top of each other
    for bad in (dict(cos_sin=None), dict(n_positions=0), dict(rotary_dim=0), dict(rotary_dim=24), dict(rotary_dim=144), dict(interleaved=2)):
        r = B.bd_rotation(4096, None, 100, 64, 0)
        for name, x in bad.items():
            setattr(r, name, x)
        assert append(rot=r) == -1, bad
    assert append(rot=B.bd_rotation(4100, None, 100, 64, 0)) == append(rot=B.bd_rotation(4096, 4098, 100, 64, 0)) == -3
    assert append(total=2 ** 31 - 1, most=2 ** 31 - 1) == -2   # beyond a launch
    assert append(total=0, k=None, v=None) == 0                # nothing to do
    assert append(c=_desc(head_dim=32)) == -2
    for name, status in (("k_codes", -1), ("v_scales", -1), ("seq_lens", -1), ("block_table", -1), ("k_res", -1)):
        d = _desc()
        setattr(d, name, None)
        assert append(c=d) == status
        setattr(d, name, 4098)
        assert append(c=d) == -3
    d = _desc()
    d.status = 4097
    assert append(c=d) == -3

    def attn(c=c, q=ok, cu=4096, total=4, most=4, scale=0.1, cap=0.0, slopes=None, prefix=None, window=0, splits=1, ws=None, out=4096, scores=True):
        s = B.bd_scores(scale, cap, slopes, prefix, window)
        return L.bd_paged8_attn(ctypes.byref(c), None if q is None else ctypes.byref(q), cu, total, most, ctypes.byref(s) if scores else None, splits, ws,
                                out, None)

    assert attn(q=None) == attn(out=None) == attn(scores=False) == attn(splits=0) == attn(splits=2) == attn(window=-1) == -1
    assert attn(cap=-1.0) == attn(cap=float("nan")) == attn(cu=None, total=5) == attn(total=-2) == attn(most=0) == -1
    assert attn(out=4100) == attn(splits=2, ws=4104) == attn(slopes=4098) == attn(prefix=4098) == attn(q=rows(4096, 8, 12)) == -3
    assert attn(cap=1025.0) == -2
    assert attn(splits=65536, ws=4096) == attn(total=2 ** 31 - 1, most=2 ** 31 - 1) == -2
    assert attn(total=0, q=None, out=None) == 0
    assert L.bd_paged8_advance(ctypes.byref(c), None, 3, 1, None) == L.bd_paged8_advance(None, 4096, 3, 1, None) == -1
    assert L.bd_paged8_advance(ctypes.byref(c), 4096, 0, 1, None) == 0


@needs_lib
@pytest.mark.parametrize("call", ["ctypes", "module"])
def test_the_class_checks_its_tensors(call, monkeypatch):
    """Both ways that the class calls the library (the C module may not have been built)."""
    if call == "ctypes":
        monkeypatch.setattr(B, "_call", B._CtypesCall)
    stream = type("", (), {"cuda_stream": 0})
    c = B.PagedKV8Cache(2, 4, 2, "int8", 6, [[0, 1, 2], [3, 4, 5]], head_dim=64, device="cpu")   # (a description; nothing is launched)
    assert c.max_len == 4 * 128 - 1 and c.k_codes.numel() == 6 * 2 * 128 * 64
    k, q, out = (torch.zeros(2, h, 64, dtype=torch.float16) for h in (2, 4, 4))
    append, attn = functools.partial(c.append, stream=stream), functools.partial(c.attn, stream=stream)
    for bad in (lambda: append(k.float(), k), lambda: append(k[:, :1], k), lambda: append(k, k[:1]), lambda: append(k, k, q=q),
                lambda: append(k, k, q=q, q_out=out[:1]), lambda: append(k.transpose(0, 2).contiguous().transpose(0, 2), k),
                lambda: append(k, k, cu_tokens=torch.zeros(2, dtype=torch.int32)), lambda: append(k, k, cu_tokens=torch.zeros(3, dtype=torch.int64)),
                lambda: attn(q, 1.0, out[:1]), lambda: attn(q, 1.0, torch.zeros(2, 4, 128, dtype=torch.float16)[..., :64]),
                lambda: attn(q, 1.0, out, slopes=torch.zeros(2)), lambda: attn(q, 1.0, out, prefix_lens=torch.zeros(2)),
                lambda: append(k, k, rotation=B.Rotation(torch.zeros(9, 32), positions=torch.zeros(3, dtype=torch.int32))),
                lambda: B.Rotation(torch.zeros(9, 32).double()), lambda: B.Rotation(torch.zeros(9, 32), positions=torch.zeros(3)),
                lambda: B.PagedKV8Cache(2, 4, 2, "int4", 6, [[0], [1]], device="cpu"), lambda: B.PagedKV8Cache(2, 4, 2, "int8", 6, [[0]], device="cpu"),
                lambda: B.PagedKV8Cache(2, 4, 2, "int8", 6, [[0], [1]], dtype=torch.float32, device="cpu"),
                lambda: B.PagedKV8Cache(2, 4, 2, "int8", 6, [[0], [1]], device="cpu", seq_lens=torch.zeros(2)),
                lambda: B.PagedKV8Cache(2, 4, 2, "int8", 6, [[0], [1]], device="cpu", buffers=[torch.zeros(4)] * 6)):
        with pytest.raises(ValueError):
            bad()
    # memory on another device than the current one (named by its number; there need not be one here)
    c._layout = c._layout[:7] + (3,) + c._layout[8:]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device is 0"):
        c.advance(stream=stream)
    with pytest.raises(ValueError, match="current device is 0"):
        B._stream_on(stream, 3)
    assert B._stream_on(stream, 0) == B._stream_on(stream, -1) == 0
    c._layout = c._layout[:7] + (-1,) + c._layout[8:]
    with pytest.raises(B.BitDecodeError):
        B.PagedKV8Cache(2, 4, 3, "int8", 6, [[0], [1]], device="cpu")
    with pytest.raises(B.BitDecodeError):
        c.append(k, k, rotation=B.Rotation(torch.zeros(9, 24)), stream=stream)
