"""Guard bands for the rotary, cache and decode entry points: every output, table and workspace carved out of one arena and
fenced by a known byte pattern, run on ragged sizes, then (1) the status words are clean, (2) results agree with the float64
references, (3) no guard byte and no cache row outside the slots changed.  Run as a script by test_gpu_serving_guard.py, once
against the normal library and once against the checked build (LAGA_DEBUG=1).  Prints GUARD_BANDS_OK on success."""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "tests"))

import serving_reference as ref  # noqa: E402
from guard_band_run import Arena  # noqa: E402
from paper_2607_17644_b200 import laga  # noqa: E402
from test_gpu_decode import case  # noqa: E402

BF16, I32, F32 = torch.bfloat16, torch.int32, torch.float32
SIZE = {BF16: 2, I32: 4, F32: 4}


def within(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    assert not torch.isnan(got.double()).any() and float((err - bound).max()) <= 0, (what, float(err.max()))


def decode(lens, h, page):
    tensors = case(lens, h, page, seed=9)
    q, w, cache, table, n = (t.cuda() for t in tensors)
    B = len(lens)
    need = laga.paged_decode_workspace_bytes(B, h)
    arena = Arena(need + B * h * 300 + (1 << 17))
    out = arena.take(B * h * 256, BF16, (B, h, 128))
    lse = arena.take(B * h * 4, F32, (B, h))
    ws = arena.take(need)
    laga.paged_decode(q, w, cache, table, n, out=out, lse=lse, workspace=ws)
    laga.check_status(ws, where=f"decode {lens} {h} {page}")
    want, want_lse, b_out, b_lse = ref.decode(*tensors, 192 ** -0.5)
    within(out, want, b_out, "out")
    live = tensors[4] > 0
    assert float(((lse.double().cpu() - want_lse)[live].abs() - b_lse[live]).max()) <= 0
    assert arena.guards_intact(), ("decode", lens, h, page)


def rope_and_latent(M, h):
    g = torch.Generator().manual_seed(M)
    x = torch.randn(M, h, 192, generator=g).to(BF16)
    kv = torch.randn(M, 576, generator=g).to(BF16)
    gamma = torch.ones(512, dtype=BF16)
    pos = torch.randint(0, 100000, (M,), generator=g, dtype=I32)
    arena = Arena(2 * M * h * 384 + M * 4096 + (1 << 20))
    take = lambda dtype, *shape: arena.take(torch.Size(shape).numel() * SIZE[dtype], dtype, shape)  # noqa: E731
    for interleaved in (True, False):
        rope = laga.rope_plan(64, interleaved=interleaved)
        fr = rope.freqs.cpu()
        y = take(BF16, M, h, 192)
        laga.rope(x.cuda(), pos.cuda(), rope, y=y)
        within(y, *ref.rotate(x.double(), pos, fr, 1.0, interleaved), "rope")
    latent, k_pe, pages = take(BF16, M, 512), take(BF16, M, 64), take(BF16, M + 9, 576)
    pages.fill_(5.0)
    slots = torch.randperm(M + 9, generator=g)[:M].to(I32)
    slots[-1] = M + 9                                       # one row outside
    _, _, mean, rstd = laga.latent_norm_rope(kv.cuda(), gamma.cuda(), None, pos.cuda(), rope, latent=latent, k_pe=k_pe, cache=pages,
                                             slots=slots.cuda())
    want = torch.full((M + 9, 576), 5.0, dtype=BF16)
    want[slots[:-1].long()] = torch.cat([latent, k_pe], 1).cpu()[:-1]
    assert torch.equal(pages.cpu(), want)
    dkv = take(BF16, M, 576)
    need = int(laga.lib().laga_latent_norm_rope_backward_workspace_bytes(M, 512))
    ws = arena.take(need)
    laga.latent_norm_rope_backward(latent.clone(), k_pe.clone(), kv.cuda(), gamma.cuda(), mean, rstd, pos.cuda(), rope, dkv_a=dkv, workspace=ws)
    assert not torch.isnan(dkv.float()).any()
    assert arena.guards_intact(), ("latent", M, h)


def plan(n, page, rows):
    lens = torch.randint(0, 100, (n,), generator=torch.Generator().manual_seed(n), dtype=I32)
    new = torch.randint(0, rows // n + 1, (n,), generator=torch.Generator().manual_seed(n + 1), dtype=I32)
    columns = (100 + rows // n) // page + 1
    arena = Arena((2 * rows + n * (columns + 4) + 4000) * 4 + (1 << 17))
    take = lambda size: arena.take(size * 4, I32, (size,))  # noqa: E731
    out = laga.CachePlan(take(rows), take(rows), take(n + 1), take(n), take(1), take(1))
    table = arena.take(n * columns * 4, I32, (n, columns))
    table.fill_(0)
    free = torch.arange(n * columns, dtype=I32, device="cuda")
    laga.cache_plan(lens.cuda(), new.cuda(), table, free, torch.tensor([n * columns], dtype=I32, device="cuda"), page, rows, out=out)
    laga.check_status(out.status)
    torch.cuda.synchronize()
    assert out.cu_new_lens[-1].item() == int(new.sum()) and arena.guards_intact(), ("plan", n, page, rows)


if __name__ == "__main__":
    for args in (([1], 1, 16), ([65, 0, 7, 1000], 16, 16), ([130, 511], 40, 64), ([3000, 1, 64], 130, 32), ([17] * 21, 8, 128)):
        decode(*args)
    for args in ((1, 1), (77, 3), (1025, 16)):
        rope_and_latent(*args)
    for args in ((1, 16, 1), (37, 64, 1000), (1000, 16, 5000)):
        plan(*args)
    print("GUARD_BANDS_OK")
