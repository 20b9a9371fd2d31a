"""Packed weights made by a context on a stream of its own (GPU)."""
import pytest
import torch

from paper_2602_04929_amd import pipeline

pytestmark = pytest.mark.gpu


def test_packed_on_another_stream(lib):
    """pack_attention_block and pack_mlp of a context on a stream of its own, called from another one that is still writing the layers."""
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    a, b = lib.Context(), lib.Context(stream=side)
    try:
        g = torch.Generator().manual_seed(1)
        made = {n: dict(codes=torch.randint(0, 16, (512, 1024), generator=g, dtype=torch.uint8).cuda(), scales=torch.rand(512, 8, generator=g).cuda(), zeros=torch.randint(0, 16, (512, 8), generator=g).float().cuda())
                for n in ("q", "k", "v", "o", "gate", "up", "down")}
        layers = {n: {k: torch.zeros_like(t) for k, t in l.items()} for n, l in made.items()}
        want = {**pipeline.pack_attention_block(a, made, 4, 128), **pipeline.pack_mlp(a, made, 4, 128)}
        torch.cuda.synchronize()
        busy = torch.randn(4096, 4096, device="cuda")
        for _ in range(3):
            for l in layers.values():
                for t in l.values():
                    t.zero_()
            torch.cuda.synchronize()
            for _ in range(20):
                busy = torch.mm(busy, busy).clamp_(-1, 1)
            for n, l in layers.items():
                for k, t in l.items():
                    t.copy_(made[n][k])
            got = {**pipeline.pack_attention_block(b, layers, 4, 128), **pipeline.pack_mlp(b, layers, 4, 128)}
            junk = [torch.full((1536, 1024), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]      # what the packing has read may be given away now, not before
            side.synchronize()
            main.synchronize()
            del junk
            for n, p in want.items():
                assert torch.equal(got[n].packed, p.packed) and torch.equal(got[n].scales, p.scales) and torch.equal(got[n].zeros, p.zeros), n
    finally:
        a.close()
        b.close()
