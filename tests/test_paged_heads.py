"""The binding's calls take a config of the heads that the pages and scales have, and no other: the kernels would read and
write past the pool.  On the CPU; calls that are in order have nothing to do."""
from types import SimpleNamespace

import pytest
import torch

from paper_2404_09529_amd import prepack as pp

STREAM = SimpleNamespace(cuda_stream=0)


def _cfg(H, Hkv, D, dtype):
    return pp.PPConfig(n_layers=1, d_model=512, n_heads=H, n_kv_heads=Hkv, head_dim=D, ffn_dim=1024, vocab=1000, dtype=dtype,
                       rms_eps=1e-5, rope_theta=1e4)


def _cache(kv, Hkv, D, k=0, scale_heads=None):
    pages = torch.zeros((3, 4, Hkv * D), dtype={pp.PP_KV_F32: torch.float32, pp.PP_KV_BF16: torch.bfloat16, pp.PP_KV_I8: torch.int8}[kv])
    scale = torch.zeros((3, 4, scale_heads or Hkv)) if kv == pp.PP_KV_I8 else None
    return pp.PagedCache(kv, torch.zeros((k, 2), dtype=torch.int32), pages, pages.clone(), scale, None if scale is None else scale.clone())


def _calls(cfg, cache):
    w = cfg.n_kv_heads * cfg.head_dim
    qw, all_ = cfg.n_heads * cfg.head_dim, (cfg.n_heads + 2 * cfg.n_kv_heads) * cfg.head_dim
    return [lambda: pp.pp_paged_write(cfg, cache, None, None, 0, None, w, None, w, stream=STREAM),
            lambda: pp.pp_paged_read(cfg, cache, None, None, 0, None, w, None, w, stream=STREAM),
            lambda: pp.pp_paged_append(cfg, cache, None, None, all_, None, qw, stream=STREAM),
            lambda: pp.pp_paged_attention_workspace_size(cfg, cache),
            lambda: pp.pp_paged_attention(cfg, cache, None, None, qw, None, None, stream=STREAM)]


KINDS = [(pp.PP_F32, pp.PP_KV_F32), (pp.PP_F32, pp.PP_KV_I8), (pp.PP_BF16, pp.PP_KV_BF16), (pp.PP_BF16, pp.PP_KV_I8)]


@pytest.mark.parametrize("dtype,kv", KINDS)
def test_heads_of_the_pages(dtype, kv):
    cache = _cache(kv, 2, 128)
    for call in _calls(_cfg(4, 2, 128, dtype), cache):
        call()
    others = [(4, 4, 128), (4, 1, 128), (8, 8, 128)] + ([(4, 2, 64), (4, 1, 64)] if dtype == pp.PP_F32 else [])
    for heads in others:
        for call in _calls(_cfg(*heads, dtype), cache):
            with pytest.raises(ValueError):
                call()


def test_heads_of_the_scales():
    """256 values a token are two heads of 128 or four of 64; scales of other heads are another layout."""
    for scale_heads in (1, 4):
        cache = _cache(pp.PP_KV_I8, 2, 128, scale_heads=scale_heads)
        for call in _calls(_cfg(4, 2, 128, pp.PP_F32), cache):
            with pytest.raises(ValueError):
                call()
    for call in _calls(_cfg(4, 4, 64, pp.PP_F32), _cache(pp.PP_KV_I8, 2, 128, scale_heads=4)):
        call()
    table, codes, two, four = torch.zeros((0, 2), dtype=torch.int32), torch.zeros((3, 4, 256), dtype=torch.int8), torch.zeros((3, 4, 2)), torch.zeros((3, 4, 4))
    for scales in [(two, four), (torch.zeros((3, 4, 0)),) * 2, (torch.zeros((3, 4, 3)),) * 2, (torch.zeros((3, 4)),) * 2]:
        with pytest.raises(ValueError):
            pp.PagedCache(pp.PP_KV_I8, table, codes, codes.clone(), *scales)
