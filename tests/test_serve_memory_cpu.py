"""What a decoder keeps on the device beside the cache (no GPU: nothing is launched)."""

import torch

from paper_2506_03781_gb300 import api, serve, synth
from paper_2506_03781_gb300.recon import _rotary


def test_a_decoder_keeps_no_more_than_its_tokens_need():
    shape = synth.BLOCKS["tiny"]
    p = serve.PagePool(4096, shape.kv_heads, shape.head_dim, page_size=64, sequences=2, device="cpu")
    d = serve.BlockDecoder(shape, {}, 64, p)
    kept = lambda: sum(t.numel() * t.element_size() for t in vars(d).values() if isinstance(t, torch.Tensor))
    single = api.paged_attn_workspace(shape.heads, shape.kv_heads, shape.head_dim, "cpu").nbytes
    assert kept() == single
    s = p.open()
    for n in (1, 1023, 1, 4000, 10000):
        p.append([s], [n])
        rope, have = d._rotations(), p.length[s]
        assert rope is d.rope and have <= len(rope) <= max(1024, 2 * have) and kept() == single + rope.nbytes
        x = torch.randn(have, shape.head_dim, generator=torch.Generator().manual_seed(n))
        (a, b), (cos, sin) = x.chunk(2, -1), rope[:have].unbind(-1)
        assert torch.equal(torch.cat([a * cos - b * sin, a * sin + b * cos], -1), _rotary(x, shape.theta))
