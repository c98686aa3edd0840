"""Guard bands for the 8-bit cache's entry points: outputs, pages and workspaces carved out of one arena and fenced by a known byte pattern, run
on ragged sizes, then (1) the status words are clean, (2) results agree with the float64 references, (3) no guard byte changed.  Run as a script by
test_gpu_cache8_guard.py, once against the normal library and once against the checked build (LAGA_DEBUG=1).  Prints GUARD_BANDS_OK on success."""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "tests"))

import cache8_reference as c8  # noqa: E402
from guard_band_run import Arena  # noqa: E402
from paper_2607_17644_b200 import laga  # noqa: E402
from test_gpu_cache8 import check_rows, expected, inputs  # noqa: E402
from test_gpu_decode8 import case  # noqa: E402

BF16, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


def decode(lens, h, page):
    tensors = case(lens, h, page, seed=9)
    q, w, pages, table, n = (t.cuda() for t in tensors)
    B = len(lens)
    need = laga.paged_decode_workspace_bytes(B, h, cache8=True)
    arena = Arena(need + B * h * 300 + pages.numel() + (1 << 17))
    held = arena.take(pages.numel(), U8, pages.shape)
    held.copy_(pages)
    out = arena.take(B * h * 256, BF16, (B, h, 128))
    lse = arena.take(B * h * 4, F32, (B, h))
    ws = arena.take(need)
    laga.paged_decode(q, w, held, table, n, out=out, lse=lse, workspace=ws)
    laga.check_status(ws, where=f"decode {lens} {h} {page}")
    want, want_lse, b_out, b_lse = c8.decode(*tensors, 192 ** -0.5)
    err = (out.double().cpu() - want).abs()
    assert not torch.isnan(out.float()).any() and float((err - b_out).max()) <= 0, (lens, h, page)
    live = tensors[4] > 0
    assert float(((lse.double().cpu() - want_lse)[live].abs() - b_lse[live]).max()) <= 0
    assert torch.equal(held, pages) and arena.guards_intact(), ("decode", lens, h, page)


def append_and_read(M, page):
    kv, gamma, beta, pos = inputs(M)
    n = -(-M // page) + 1
    arena = Arena(n * page * 644 + M * 1400 + (1 << 17))
    pages = arena.take(n * page * 644, U8, (n, page * 644))
    latent, k_pe = arena.take(M * 1024, BF16, (M, 512)), arena.take(M * 128, BF16, (M, 64))
    slots = torch.randperm(n * page, generator=torch.Generator().manual_seed(M))[:M].to(torch.int32)
    slots[-1] = n * page if M > 1 else slots[-1]                # one row outside
    for interleaved in (True, False):
        rope = laga.rope_plan(64, interleaved=interleaved)
        laga.cache_append(kv.cuda(), gamma.cuda(), beta.cuda(), pos.cuda(), rope, slots.cuda(), pages)
        laga.cache_read(pages, slots.cuda(), latent=latent, k_pe=k_pe)
        m = M - 1 if M > 1 else M
        rows, slack = expected(kv, gamma, beta, pos, rope)
        check_rows(pages.cpu(), slots[:m], rows[:m], slack[:m])
        assert M == m or not bool(latent[-1].any() | k_pe[-1].any())
        assert arena.guards_intact(), ("append", M, page)


if __name__ == "__main__":
    for args in (([1], 1, 16), ([65, 0, 7, 1000], 16, 16), ([130, 511], 40, 64), ([700, 129], 20, 32), ([3000, 1, 64], 130, 32), ([17] * 21, 8, 128),
                 ([100] * 40, 30, 1024), ([3, 90, 0] * 45 + [1200], 70, 16), ([20] * 129, 64, 64)):
        decode(*args)
    for args in ((1, 16), (77, 64), (1025, 1024), (4099, 32)):
        append_and_read(*args)
    print("GUARD_BANDS_OK")
