"""ss_paged_forward behind thousands of cached positions, where the attention of a model's rows (two planes in bf16) goes round its ring and workgroups have
pieces of several heads: beside ss_verify_forward over the contiguous cache."""
import pytest
import torch

import paper_2311_04951_amd as sv
import seeded_inputs as si
from gpu_util import dev, maxabs, tol, weights_to_device
from paper_2311_04951_amd.paged import PagedCache

pytestmark = pytest.mark.gpu
# heads of 128, 64 and 32; fp32
SHAPES = [si.DecoderShape(2, 256, 2, 128, 512, 1000, dtype="bf16"), si.DecoderShape(2, 256, 4, 64, 512, 1000, dtype="bf16"),
          si.DecoderShape(1, 256, 8, 32, 512, 1000, dtype="bf16"), si.TINY_TARGET]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("M", [1, 4])
def test_long_contexts_beside_the_contiguous_cache(shape, M):
    batch, max_pos = 16, 16400
    gm = sv.Model(shape, weights_to_device(si.decoder_weights(shape, 11)), max_rows=batch * M, max_pos=max_pos)
    lengths = [max_pos - M - 1000 * b - 7 * b for b in range(batch)]
    block = 256 if shape.dtype == "bf16" else 128
    assert sum(-(-n // block) for n in lengths) * shape.n_heads // 256 >= 128 // shape.head_dim + 2     # blocks of a workgroup: more than the ring's stages
    contiguous = sv.KVCache(gm, batch, max_pos)
    cache = PagedCache(gm, batch, sum(-(-(n + M) // 64) for n in lengths), 64, -(-max_pos // 64), weights=False)
    g = torch.Generator(device="cuda")
    g.manual_seed(12)
    for b, n in enumerate(lengths):
        cache.resize(b, n)
        one = cache.one(b)
        for layer in range(shape.n_layers):
            k, v = (torch.randn((n, shape.n_heads, shape.head_dim), generator=g, device="cuda").to(cache.kv.k.dtype) for _ in range(2))
            sv.ss_kv_cache_append(contiguous, layer, b, 0, k, v)
            sv.ss_paged_append(one, layer, k[None], v[None])
        sv.ss_paged_advance(one, n)
    sv.ss_kv_cache_set_len(contiguous, lengths)
    toks = si.token_ids(11, "rows", (batch, M), shape.vocab).to(dev())
    for b, n in enumerate(lengths):
        cache.resize(b, n + M)
    got = sv.ss_paged_forward(gm, cache.kv, toks, M, max_len=max(lengths) + M)
    want = sv.ss_verify_forward(gm, contiguous, toks, M)
    assert maxabs(got, want.cpu().numpy()) < tol(shape)
    assert int(cache.kv.status[0]) == 0 and cache.kv.length.tolist() == [n + M for n in lengths]
