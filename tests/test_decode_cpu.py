"""The decode-step entry points' host checks (nothing is launched on any of
these paths), and the reference that the GPU tests use, on known values."""
import ctypes
import os

import numpy as np
import pytest

import paper_2609_15359_amd as maps
from tests import decode_ref as ref

FAKE = ctypes.c_void_p(0x1000)    # never read: every call below fails its host checks
ODD = ctypes.c_void_p(0x1001)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(maps.LIBRARY):
        pytest.fail("libmaps.so is not built; run __graft_entry__.build()")
    return maps.library()


def test_page_bytes(lib):
    assert lib.maps_kv_page_bytes(16, 128) == 2 * 16 * (64 + 4)
    assert lib.maps_kv_page_bytes(256, 64) == 2 * 256 * (32 + 2)
    for S, D in ((0, 128), (8, 128), (24, 128), (512, 128), (16, 96), (16, 0), (-16, 128)):
        assert lib.maps_kv_page_bytes(S, D) == 0
    assert maps.KVCache.bytes_per_token(8, 128) == 8 * 2 * 68
    with pytest.raises(maps.MapsError):
        maps.KVCache.page_bytes(16, 100)


def _block_step(lib, B=4, max_blocks=8, S=16, N=32, T=10, **null):
    names = ("grow", "lens", "held", "table", "ring", "ring_pos", "lens_out", "held_out", "ring_pos_out", "tok_off",
             "slots")
    p = {k: None if k in null else FAKE for k in names + ("granted", "dev_err")}
    return lib.maps_block_step(B, max_blocks, S, N, None, *(p[k] for k in names), T, p["granted"], p["dev_err"], None)


def test_block_step(lib):
    for bad in (dict(B=0), dict(B=maps.decode.MAX_STEP_REQUESTS + 1), dict(max_blocks=0), dict(S=0), dict(N=0),
                dict(T=-1), dict(T=2**31), dict(B=4096, max_blocks=2**20)):
        assert _block_step(lib, **bad) == -2, bad
    for name in ("grow", "lens", "held", "table", "ring", "ring_pos", "lens_out", "held_out", "ring_pos_out", "tok_off",
                 "slots", "granted", "dev_err"):
        assert _block_step(lib, **{name: None}) == -1, name


def test_append_and_read(lib):
    def append(cache=FAKE, n=4, S=16, H=2, D=128, k=FAKE, v=FAKE, ty=0, T=3, slots=FAKE, err=FAKE):
        return lib.maps_kv_append(cache, n, S, H, D, k, v, ty, T, 256, 128, 256, 128, slots, err, None)

    def read(cache=FAKE, n=4, S=16, H=2, D=128, k=FAKE, v=FAKE, ty=0, T=3, slots=FAKE, err=FAKE):
        return lib.maps_kv_read(cache, n, S, H, D, slots, T, k, v, ty, err, None)

    for f in (append, read):
        for bad in (dict(n=0), dict(S=8), dict(S=48), dict(S=512), dict(H=0), dict(D=96), dict(T=-1), dict(T=2**31)):
            assert f(**bad) == -2, bad
        for bad in (dict(cache=None), dict(k=None), dict(v=None), dict(slots=None), dict(err=None)):
            assert f(**bad) == -1, bad
        assert f(ty=3) == -8 and f(ty=-1) == -8
        assert f(cache=ctypes.c_void_p(0x1008)) == -9
        assert f(k=ODD) == -9 and f(v=ODD) == -9
        assert f(T=0) == 0
    assert read(k=ctypes.c_void_p(0x1008)) == -9


def test_attend(lib):
    def attend(cache=FAKE, n=4, S=16, H=2, D=128, q=FAKE, ty=0, T=3, Hq=8, st=1024, sh=128, table=FAKE, B=3, mb=5,
               lens=FAKE, off=FAKE, max_q=1, window=0, out=FAKE, err=FAKE, ws=FAKE, short=0):
        need = lib.maps_kv_attend_workspace_size(B, T, Hq, H, D, max_q)
        return lib.maps_kv_attend(cache, n, S, H, D, q, ty, T, Hq, st, sh, table, B, mb, lens, off, max_q, 0.1, window,
                                  out, None, err, ws, max(0, need - short), None)

    for bad in (dict(n=0), dict(S=20), dict(H=0), dict(H=3), dict(D=80), dict(T=-1), dict(T=2**31), dict(Hq=0), dict(B=0),
                dict(B=maps.decode.MAX_STEP_REQUESTS + 1), dict(mb=0), dict(max_q=0), dict(window=-1),
                dict(B=4096, mb=2**20)):
        assert attend(**bad) == -2, bad
    for bad in (dict(cache=None), dict(q=None), dict(table=None), dict(lens=None), dict(off=None), dict(out=None),
                dict(err=None)):
        assert attend(**bad) == -1, bad
    assert attend(ty=2) == -8 and attend(ty=7) == -8
    for bad in (dict(cache=ODD), dict(q=ctypes.c_void_p(0x1008)), dict(out=ODD), dict(st=1028), dict(sh=100), dict(ws=ODD)):
        assert attend(**bad) == -9, bad
    assert attend(T=0) == 0


def test_attend_needs_no_stride_of_one_row(lib):
    """Strides of axes of size 1 are free (what is refused is the workspace, which comes behind the alignment), and a
    workspace that is missing or a byte short is refused; the tables are wide enough for all workgroups."""
    def attend(T, Hq, st, sh, ws=FAKE, short=1):
        need = lib.maps_kv_attend_workspace_size(3, T, Hq, 1, 128, 4)
        return lib.maps_kv_attend(FAKE, 4096, 16, 1, 128, FAKE, 0, T, Hq, st, sh, FAKE, 3, 2**20, FAKE, FAKE, 4, 0.1, 0, FAKE,
                                  None, FAKE, ws, need - short, None)

    assert attend(1, 8, 1001, 128) == -4 and attend(1, 1, 3, 5) == -4 and attend(4, 1, 128, 129) == -4
    assert attend(2, 8, 1001, 128) == -9 and attend(1, 8, 1024, 129) == -9 and attend(4, 1, 130, 129) == -9
    assert attend(4, 8, 1024, 128) == -4 and attend(4, 8, 1024, 128, None, 0) == -1


def test_verify(lib):
    def verify(B=3, K=2, V=100, target=FAKE, ty=2, tokens=FAKE, n=FAKE, u=FAKE, noise=FAKE, out=FAKE, acc=FAKE, err=FAKE,
               ws=FAKE, short=0):
        need = lib.maps_verify_drafts_workspace_size(B, V)
        return lib.maps_verify_drafts(B, K, V, target, 300, 100, None, 0, 0, ty, tokens, n, u, noise, 100, out, acc, err,
                                      ws, need - short if need else 0, None)

    for bad in (dict(B=0), dict(K=-1), dict(K=maps.decode.MAX_DRAFTS + 1), dict(V=0)):
        assert verify(**bad) == -2, bad
    for name in ("target", "tokens", "n", "u", "noise", "out", "acc", "err", "ws"):
        assert verify(**{name: None}) == -1, name
    assert verify(ty=3) == -8
    assert verify(short=1) == -4
    assert verify(ws=ODD) == -9
    assert lib.maps_verify_drafts_workspace_size(0, 5) == 0 and lib.maps_verify_drafts_workspace_size(5, 0) == 0


def test_workspace_sizes_follow_the_device(monkeypatch):
    """Attention's workspace depends on the device's compute units: a size that one device gave is no other's."""
    import torch

    class Library:
        device = 0

        def maps_kv_attend_workspace_size(self, *sizes):
            return 1000 * (self.device + 1)

    lib = Library()
    monkeypatch.setattr(maps.decode, "library", lambda: lib)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: lib.device)
    maps.decode._size.cache_clear()
    try:
        for lib.device in (0, 1, 0, 3):
            assert maps.decode.kv_attend_workspace_bytes(3, 5, 8, 2, 128, 1) == 1000 * (lib.device + 1)
    finally:
        maps.decode._size.cache_clear()


def test_binding_refuses_host_tensors_and_shapes():
    import torch
    i32 = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(maps.MapsError, match="device tensor"):
        maps.block_step(i32, i32.reshape(4, 1), i32, i32, i32, i32[:2], 16, 4)
    with pytest.raises(maps.MapsError, match="device tensor"):
        maps.KVCache(torch.zeros((2, 1, 2176), dtype=torch.uint8), 16, 128)
    with pytest.raises(maps.MapsError, match="device tensor"):
        maps.verify_drafts(torch.zeros((2, 2, 5)), i32[:2].reshape(2, 1), i32[:2], torch.zeros(2, 1), torch.zeros(2, 5))


def test_reference_number_format():
    """All 16 codes, ties to the even code, the limit, the scale of a block."""
    assert ref.dequantise(np.arange(16).repeat(2), np.array([127])).reshape(16, 2)[:, 0].tolist() == [
        0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6]
    x = np.zeros(32)
    x[:11] = [4, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 7.9, -.2500001, 5.0001]
    code, byte = ref.quantise(x)
    assert byte.tolist() == [127]
    assert ref.dequantise(code, byte)[:11].tolist() == [4, 0, 1, 1, 2, 2, 4, 4, 6, -.5, 6]
    for amax, want in ((1.0, 125), (1.99, 125), (2.0, 126), (0.0, 2), (2.0 ** -130, 2), (2.0 ** 127, 252), (np.inf, 255)):
        assert ref.quantise(np.full(32, amax))[1].tolist() == [want], amax


def test_reference_pages():
    rng = np.random.RandomState(0)
    for S, D in ((16, 64), (32, 128), (16, 256)):
        page = np.zeros(2 * S * (D // 2 + D // 32), np.uint8)
        k, v = rng.standard_normal((2, S, D))
        for t in range(S):
            ref.write_token(page, t, k[t], v[t], S, D)
        got = ref.read_tokens(np.broadcast_to(page, (S, page.size)), np.arange(S), S, D)
        for g, x in zip(got, (k, v)):
            assert np.array_equal(g, ref.dequantise(*ref.quantise(x)))
