"""Host-side checks of the rotary, cache and decode entry points that need no GPU: sizes, refusals before any device
work, and the frequencies of the rotation plan."""
import ctypes
import math

import pytest
import torch


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
    return P((i + 1) << 32)


def test_rope_refusals(laga):
    lib = laga.lib()

    def call(x=at(0), xp=3 * 192, pos=at(1), fr=at(2), M=4, h=3, d=192, begin=128, rot=64, layout=1, ms=1.0, y=at(3), yp=3 * 192):
        return lib.laga_rope(x, xp, pos, fr, M, h, d, begin, rot, layout, ms, 0, y, yp, None)

    bad = laga.ERR_INVALID_ARG
    assert call(x=None) == bad and call(pos=None) == bad and call(fr=None) == bad and call(y=None) == bad
    assert call(M=0) == bad and call(h=0) == bad
    assert call(x=P((1 << 32) + 8)) == bad                       # not 16-byte aligned
    assert call(xp=3 * 192 - 8) == bad and call(yp=3 * 192 + 4) == bad
    assert call(d=190) == bad and call(d=2048, xp=1 << 13, yp=1 << 13) == bad
    assert call(rot=24) == bad and call(rot=512, d=512, begin=0, xp=1536, yp=1536) == bad
    assert call(begin=136) == bad and call(begin=-8) == bad and call(begin=4) == bad
    assert call(layout=2) == bad
    assert call(ms=float("nan")) == bad
    assert call(y=at(0), yp=4 * 192) == bad                      # in place needs one pitch
    assert call(y=P((1 << 32) + 384)) == bad                     # overlaps x without being x
    assert call(y=at(1)) == bad and call(y=at(2)) == bad


def test_latent_norm_rope_refusals(laga):
    lib = laga.lib()

    def fwd(kv=at(0), pitch=576, gamma=at(1), beta=None, eps=1e-5, pos=at(2), fr=at(3), M=4, D=512, R=64, layout=0, lat=at(4), kpe=at(5),
            mean=at(6), rstd=at(7), cache=None, slots=None, n_slots=0):
        return lib.laga_latent_norm_rope(kv, pitch, gamma, beta, eps, pos, fr, M, D, R, layout, 1.0, lat, kpe, mean, rstd, cache, slots,
                                         n_slots, None)

    bad = laga.ERR_INVALID_ARG
    assert fwd(kv=None) == bad and fwd(gamma=None) == bad and fwd(pos=None) == bad and fwd(fr=None) == bad
    assert fwd(M=0) == bad and fwd(D=516) == bad and fwd(D=2048, pitch=4096) == bad and fwd(R=8) == bad
    assert fwd(pitch=568) == bad and fwd(pitch=580) == bad
    assert fwd(eps=-1.0) == bad
    assert fwd(lat=None) == bad and fwd(kpe=None) == bad          # one of the two
    assert fwd(lat=None, kpe=None) == bad                         # no destination at all
    assert fwd(cache=at(8)) == bad and fwd(slots=at(8)) == bad
    assert fwd(cache=at(8), slots=at(9), n_slots=0) == bad
    assert fwd(beta=P(8)) == bad
    assert fwd(M=(1 << 30) + 1) == bad and fwd(pitch=(1 << 30) + 8) == bad
    for name in ("lat", "kpe", "mean", "rstd"):                   # outputs apart from inputs ...
        for i in (0, 1, 2, 3):
            assert fwd(**{name: at(i)}) == bad, (name, i)
    assert fwd(cache=at(0), slots=at(9), n_slots=4) == bad and fwd(cache=at(8), slots=at(8), n_slots=4) == bad
    assert fwd(rstd=at(6)) == bad and fwd(kpe=P((5 << 32) + 4 * 512 * 2 - 16)) == bad      # ... and from one another
    assert fwd(cache=at(4), slots=at(9), n_slots=4) == bad

    def bwd(dl=at(0), ws=at(9), ws_bytes=1 << 30, M=4, D=512, R=64, pitch=576):
        return lib.laga_latent_norm_rope_backward(dl, at(1), at(2), pitch, at(3), at(4), at(5), at(6), at(7), M, D, R, 0, 1.0, at(8), at(10),
                                                  None, ws, ws_bytes, None)

    assert bwd(dl=None) == bad and bwd(ws=None) == bad and bwd(M=0) == bad and bwd(D=20) == bad and bwd(R=20) == bad and bwd(pitch=512) == bad
    assert bwd(M=(1 << 30) + 1) == bad and bwd(pitch=(1 << 30) + 8) == bad
    assert bwd(dl=at(8)) == bad and bwd(ws=at(2)) == bad and bwd(ws=at(10)) == bad and bwd(dl=P((10 << 32) + 1024)) == bad
    assert bwd(ws_bytes=16) == laga.ERR_WORKSPACE_TOO_SMALL
    size = lib.laga_latent_norm_rope_backward_workspace_bytes
    assert size(1, 512) == 4096 and size(1 << 20, 512) == 296 * 4096 and size(0, 512) == 0 and size(5, 2048) == 0


def test_cache_plan_refusals(laga):
    lib = laga.lib()

    def call(seq=at(0), new=at(1), n=4, page=64, table=at(2), columns=8, free=at(3), cap=32, n_free=at(4), rows=16, slots=at(5), pos=at(6),
             cu=at(7), seq_out=at(8), free_out=at(9), word=at(10)):
        return lib.laga_cache_plan(seq, new, n, page, table, columns, free, cap, n_free, rows, slots, pos, cu, seq_out, free_out, word, None)

    bad = laga.ERR_INVALID_ARG
    for name in ("seq", "new", "table", "free", "n_free", "slots", "pos", "cu", "seq_out", "free_out", "word"):
        assert call(**{name: None}) == bad
    assert call(n=0) == bad and call(n=8193) == bad and call(columns=0) == bad and call(cap=0) == bad and call(rows=0) == bad
    for page in (0, 1, 8, 48, 100, 2048, -64):
        assert call(page=page) == bad
    assert call(page=1024, columns=(1 << 20) + 1) == bad and call(rows=(1 << 30) + 1) == bad
    assert call(seq_out=at(0)) == bad                             # outputs apart from inputs ...
    assert call(free_out=at(4)) == bad
    assert call(slots=P((4 << 32) + 4)) == bad                    # (inside the free stack)
    assert call(pos=P((6 << 32) + 32)) == bad                     # ... and from one another


def test_paged_decode_refusals_and_sizes(laga):
    lib = laga.lib()

    def call(q=at(0), w=at(1), cache=at(2), pages=16, page=64, table=at(3), columns=4, lens=at(4), B=2, h=16, dc=512, dn=128, dr=64, dv=128,
             scale=0.07, out=at(5), lse=None, ws=at(6), ws_bytes=1 << 40, flags=0):
        return lib.laga_paged_decode(q, w, cache, pages, page, table, columns, lens, B, h, dc, dn, dr, dv, scale, out, lse, ws, ws_bytes,
                                     flags, None)

    bad = laga.ERR_INVALID_ARG
    for name in ("q", "w", "cache", "table", "lens", "out", "ws"):
        assert call(**{name: None}) == bad
    assert call(B=0) == bad and call(h=0) == bad and call(pages=0) == bad and call(columns=0) == bad
    assert call(page=8) == bad and call(page=96) == bad and call(page=2048) == bad
    assert call(scale=0.0) == bad and call(scale=float("nan")) == bad and call(flags=1) == bad
    assert call(ws=P((7 << 32) + 16)) == bad and call(q=P(24)) == bad and call(lens=P(6)) == bad
    assert call(pages=(1 << 24) + 1) == bad and call(columns=(1 << 24) + 1) == bad
    assert call(columns=1 << 24, B=65) == bad                     # tiles counted in 32 bits
    for i in (0, 1, 2, 3, 4):                                     # outputs and workspace apart from inputs and from one another
        assert call(out=at(i)) == bad and call(lse=at(i)) == bad and call(ws=at(i)) == bad, i
    assert call(lse=at(5)) == bad and call(ws=at(5)) == bad and call(lse=P((7 << 32) + 64)) == bad
    assert call(dc=256) == laga.ERR_UNSUPPORTED and call(dv=64) == laga.ERR_UNSUPPORTED
    assert call(ws_bytes=4096) == laga.ERR_WORKSPACE_TOO_SMALL
    size = laga.paged_decode_workspace_bytes
    assert size(1, 16) % 1024 == 0 and size(0, 16) == 0 and size(4, 16, d_c=256) == 0
    for B, h in ((1, 1), (64, 16), (7, 40), (8, 128), (300, 200)):
        heads = 16 if h <= 16 else 32 if h <= 32 else 64
        groups = -(-h // heads)
        slots = max(1, 148 // groups) + B
        assert size(B, h) >= slots * groups * heads * (512 * 4 + 8) + B * h * 512 * 2 + 1024


def test_binding_refuses_cpu_tensors_and_wrong_types(laga):
    rope = laga.rope_plan(64, device="cpu")
    x = torch.zeros(4, 2, 192, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        laga.rope(x, torch.zeros(4, dtype=torch.int32), rope)
    kv = torch.zeros(4, 576, dtype=torch.bfloat16)
    gamma = torch.ones(512, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        laga.latent_norm_rope(kv, gamma, None, torch.zeros(4, dtype=torch.int32), rope)
    with pytest.raises(ValueError):
        laga.latent_norm_rope(kv, gamma, None, torch.zeros(4, dtype=torch.int32), rope, cache=kv)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        laga.cache_plan(i, i, i.view(4, 1), i, i[:1], 64, 4)
    with pytest.raises(ValueError):
        laga.paged_decode(x, torch.zeros(512, 512, dtype=torch.bfloat16), torch.zeros(2, 64, 576, dtype=torch.bfloat16), i.view(4, 1), i)


def test_binding_refuses_what_is_no_tensor_or_no_plan(laga):
    rope = laga.rope_plan(64, device="cpu")
    x, i = torch.zeros(4, 2, 192, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: laga.rope(None, i, rope), lambda: laga.rope(x.tolist(), i, rope), lambda: laga.latent_norm_rope(x, x, 3, i, rope),
                 lambda: laga.cache_append(x, None, None, i, rope, i, x), lambda: laga.paged_decode(x, x, x, None, i),
                 lambda: laga.cache_plan(i, i, None, i, i, 64, 4)):
        with pytest.raises(TypeError):
            call()
    from paper_2607_17644_b200 import _binding
    for entry in ("rope", "latent_norm_rope", "latent_norm_rope_backward", "cache_plan", "paged_decode", "bind"):
        with pytest.raises(TypeError):
            getattr(_binding, entry)(x)


def test_rope_plan_frequencies(laga):
    j = torch.arange(32, dtype=torch.float64)
    plain = laga.rope_plan(64, device="cpu")
    assert plain.mscale == 1.0 and plain.interleaved and plain.freqs.dtype == torch.float64
    assert torch.allclose(plain.freqs, torch.exp(-j / 32 * math.log(10000.0)), rtol=1e-14)
    assert torch.equal(laga.rope_plan(64, scaling={"type": "linear", "factor": 8}, device="cpu").freqs, plain.freqs / 8)
    ntk = laga.rope_plan(64, scaling={"type": "ntk", "factor": 4}, device="cpu").freqs
    assert ntk[0] == 1.0 and math.isclose(float(ntk[-1]), float(plain.freqs[-1]) / 4, rel_tol=1e-12)
    yarn = laga.rope_plan(64, scaling={"type": "yarn", "factor": 40, "original_length": 4096}, interleaved=False, device="cpu")
    turns = 4096 * plain.freqs / (2 * math.pi)
    assert torch.equal(yarn.freqs[turns >= 33], plain.freqs[turns >= 33])                # fast pairs kept
    assert torch.allclose(yarn.freqs[turns <= 0.7], plain.freqs[turns <= 0.7] / 40, rtol=1e-14)      # slow pairs stretched
    assert bool((yarn.freqs <= plain.freqs).all() and (yarn.freqs >= plain.freqs / 40).all() and (yarn.freqs.diff() < 0).all())
    assert math.isclose(yarn.mscale, 0.1 * math.log(40) + 1) and not yarn.interleaved
    for wrong in ({"type": "cubic", "factor": 2}, {"type": "linear", "factor": 0.5}, {"type": "linear", "factor": 2, "beta_fast": 3}):
        with pytest.raises(ValueError):
            laga.rope_plan(64, scaling=wrong, device="cpu")
    with pytest.raises(ValueError):
        laga.rope_plan(63, device="cpu")
