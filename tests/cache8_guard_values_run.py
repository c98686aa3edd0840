"""The decode over the 8-bit cache between guard bands, with results that start as NaN and have to be the float64 reference's in the mean square: a load or a store that the
checked build left out would show.  Run as a script by test_gpu_cache8_guard_values.py, against the normal library and the checked build (LAGA_DEBUG=1).
Prints GUARD_VALUES_OK on success."""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "tests"))

from guard_band_run import Arena  # noqa: E402
from paper_2607_17644_b200 import laga  # noqa: E402
from test_gpu_decode8 import case, check  # noqa: E402
from test_gpu_decode8_apart import sinks  # noqa: E402

BF16, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


def decode(tensors, l2=5e-3):
    q, w, pages, table, n = (t.cuda() for t in tensors)
    B, h = q.shape[:2]
    need = laga.paged_decode_workspace_bytes(B, h, cache8=True)
    arena = Arena(need + B * h * 300 + pages.numel() + (1 << 17))
    held = arena.take(pages.numel(), U8, pages.shape)
    held.copy_(pages)
    out, lse, ws = arena.take(B * h * 256, BF16, (B, h, 128)), arena.take(B * h * 4, F32, (B, h)), arena.take(need)
    out.fill_(float("nan"))
    lse.fill_(float("nan"))
    laga.paged_decode(q, w, held, table, n, out=out, lse=lse, workspace=ws)
    laga.check_status(ws, where=f"decode {B} {h}")
    check(tensors, out, lse, l2=l2)
    assert torch.equal(held, pages) and arena.guards_intact(), ("decode", B, h)


if __name__ == "__main__":
    for lens, h, page in (([1], 1, 16), ([65, 0, 7, 1000], 16, 16), ([130, 511], 40, 64), ([700, 129], 20, 32), ([3000, 1, 64], 130, 32), ([17] * 21, 8, 128),
                          ([100] * 40, 30, 1024), ([3, 90, 0] * 45 + [1200], 70, 16), ([20] * 129, 64, 64)):
        decode(case(lens, h, page, seed=9))
    for lens, h, page in (([100, 0, 700, 30], 16, 16), ([129, 64] * 60, 30, 64), ([300] * 20 + [2], 70, 32)):
        decode(sinks(lens, h, page, [0, 5, 40], 12.0, 1.0, seed=10), l2=7.5e-3)     # weights that stand apart, kept in the workspace
    print("GUARD_VALUES_OK")
