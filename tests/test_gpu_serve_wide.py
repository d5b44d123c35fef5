"""A deployed block with heads of 256 channels: a long prompt in one go, whose rows are read back, and the same tokens in chunks
and one by one."""

import dataclasses

import pytest
import torch

from paper_2506_03781_gb300 import recon, serve, synth
from tests.test_gpu_serve_rows import FMT, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def block():
    shape = dataclasses.replace(synth.BLOCKS["tiny"], name="wide", head_dim=256)
    weights = {n: raw for n, (raw, _) in synth.block_weights(shape, 1).items()}
    return recon.BlockReconstructor(shape, weights, q=3, g=64, G=4, T=2)


@pytest.mark.parametrize("fmt", sorted(FMT))
def test_long_prompts_in_one_go_and_in_chunks(block, fmt):
    pool = serve.PagePool(60, block.shape.kv_heads, 256, page_size=16, fmt=FMT[fmt], sequences=2)
    dec = serve.BlockDecoder.of(block, pool)
    X = torch.randn(303, block.shape.d, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    a, b = pool.open(), pool.open()
    whole = torch.cat([dec.prefill(a, X[:300]), *(dec.decode([a], X[i:i + 1]) for i in range(300, 303))])
    parts = torch.cat([dec.extend([b], X[:130], [130]), dec.extend([b], X[130:299], [169]), *(dec.decode([b], X[i:i + 1]) for i in range(299, 303))])
    same(whole, parts, X, fmt)
    assert pool.length[a] == pool.length[b] == 303
