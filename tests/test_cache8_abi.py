"""Host-side checks of the 8-bit cache's entry points that need no GPU: sizes and refusals before any device work."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def laga():
    from paper_2607_17644_b200 import build
    build.build()
    from paper_2607_17644_b200 import laga as _laga
    _laga.lib()
    return _laga


P = ctypes.c_void_p


def at(i):
    """Distinct, aligned addresses far apart; never dereferenced on these paths."""
    return P((i + 1) << 36)


def test_append_refusals(laga):
    def call(kv=at(0), pitch=576, gamma=at(1), beta=None, eps=1e-5, pos=at(2), fr=at(3), M=4, layout=1, ms=1.0, cache=at(4), pages=8, page=64, slots=at(5)):
        return laga.lib().laga_cache8_append(kv, pitch, gamma, beta, eps, pos, fr, M, layout, ms, cache, pages, page, slots, None)

    bad = laga.ERR_INVALID_ARG
    for name in ("kv", "gamma", "pos", "fr", "cache", "slots"):
        assert call(**{name: None}) == bad, name
    assert call(M=0) == bad and call(M=(1 << 30) + 1) == bad and call(pages=0) == bad and call(eps=-1.0) == bad and call(eps=float("nan")) == bad
    for page in (0, 8, 24, 2048, -64):
        assert call(page=page) == bad
    assert call(pitch=568) == bad and call(pitch=580) == bad and call(pitch=(1 << 30) + 8) == bad
    assert call(layout=2) == bad and call(ms=float("nan")) == bad
    assert call(pages=(1 << 24) + 1) == bad                       # rows past 2^30
    for name in ("kv", "gamma", "cache"):
        assert call(**{name: P((9 << 36) + 8)}) == bad, name
    assert call(slots=P((9 << 36) + 2)) == bad and call(beta=P(8)) == bad
    for i in (0, 1, 2, 3, 5):                                     # the cache apart from every input
        assert call(cache=at(i)) == bad, i
    assert call(slots=P((5 << 36) + 8 * 64 * 644 - 4)) == bad


def test_read_refusals(laga):
    def call(cache=at(0), pages=8, page=64, slots=at(1), M=4, latent=at(2), k_pe=at(3)):
        return laga.lib().laga_cache8_read(cache, pages, page, slots, M, latent, k_pe, None)

    bad = laga.ERR_INVALID_ARG
    for name in ("cache", "slots", "latent", "k_pe"):
        assert call(**{name: None}) == bad, name
    assert call(M=0) == bad and call(M=(1 << 30) + 1) == bad and call(pages=0) == bad and call(page=48) == bad and call(pages=(1 << 24) + 1) == bad
    for name in ("cache", "latent", "k_pe"):
        assert call(**{name: P((9 << 36) + 8)}) == bad, name
    assert call(slots=P((9 << 36) + 1)) == bad
    assert call(latent=at(0)) == bad and call(k_pe=at(1)) == bad and call(k_pe=at(2)) == bad and call(k_pe=P((3 << 36) + 4 * 1024 - 16)) == bad


def test_decode_refusals_and_sizes(laga):
    lib = laga.lib()

    def call(q=at(0), w=at(1), cache=at(2), pages=16, page=64, table=at(3), columns=4, lens=at(4), B=2, h=16, dc=512, dn=128, dr=64, dv=128,
             scale=0.07, out=at(5), lse=None, ws=at(6), ws_bytes=1 << 40, flags=0):
        return lib.laga_paged_decode8(q, w, cache, pages, page, table, columns, lens, B, h, dc, dn, dr, dv, scale, out, lse, ws, ws_bytes, flags, None)

    bad = laga.ERR_INVALID_ARG
    for name in ("q", "w", "cache", "table", "lens", "out", "ws"):
        assert call(**{name: None}) == bad, name
    assert call(B=0) == bad and call(h=0) == bad and call(pages=0) == bad and call(columns=0) == bad
    assert call(page=8) == bad and call(page=96) == bad and call(page=2048) == bad
    assert call(scale=0.0) == bad and call(scale=float("nan")) == bad and call(flags=1) == bad
    assert call(ws=P((7 << 36) + 16)) == bad and call(q=P(24)) == bad and call(lens=P(6)) == bad and call(cache=P((9 << 36) + 8)) == bad
    assert call(dc=256) == laga.ERR_UNSUPPORTED and call(dr=32) == laga.ERR_UNSUPPORTED
    assert call(pages=(1 << 24) + 1) == bad and call(columns=(1 << 24) + 1) == bad and call(B=1 << 22, h=32) == bad
    assert call(ws_bytes=1024) == laga.ERR_WORKSPACE_TOO_SMALL
    for i in (0, 1, 2, 3, 4):
        assert call(out=at(i)) == bad and call(ws=at(i)) == bad and call(lse=at(i)) == bad, i
    assert call(lse=at(5)) == bad and call(out=at(6)) == bad
    size = lib.laga_paged_decode8_workspace_bytes
    assert size(0, 16, 512, 128, 64, 128) == 0 and size(4, 0, 512, 128, 64, 128) == 0 and size(4, 16, 256, 128, 64, 128) == 0
    # the status, two rows of 640 codes and a factor for each padded head, and the pieces: 512 + 2 words for each of (CTAs + B) x heads
    assert size(4, 16, 512, 128, 64, 128) == 1024 + 4 * 16 * 1280 + 1024 + (148 + 4) * 16 * (512 + 2) * 4
    assert laga.paged_decode_workspace_bytes(4, 16, cache8=True) == size(4, 16, 512, 128, 64, 128) != laga.paged_decode_workspace_bytes(4, 16)


def test_cache_of_eight_bits_or_sixteen():
    from paper_2607_17644_b200 import LatentCache
    with pytest.raises(ValueError, match="bits"):
        LatentCache(4, 2, 64, bits=4, device="cpu")
    eight, sixteen = LatentCache(4, 2, 64, page_size=16, device="cpu", bits=8), LatentCache(4, 2, 64, page_size=16, device="cpu")
    assert eight.pages[0].numel() == 4 * 16 * 644 and sixteen.pages[0].numel() * 2 == 4 * 16 * 1152
