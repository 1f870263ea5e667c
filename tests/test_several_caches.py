"""Caches of different shapes that live side by side and share kernels."""
import pytest
import torch

from paper_2512_04857_b200 import lar

DEV = "cuda:0"


def _config(dtype, batch, hkv, line_width, budget_lines, flags=0):
    return lar.make_config(n_layers=1, batch=batch, n_q_heads=4 * hkv, n_kv_heads=hkv, head_dim=128, dtype=dtype, cond_len=1, line_width=line_width,
                           n_lines=12, anchor_len=line_width, recent_lines=1, budget_lines=budget_lines, flags=flags)


def _generate(cache, lines, seed):
    cfg, g = cache.cfg, torch.Generator(DEV).manual_seed(seed)
    td = torch.bfloat16 if cfg.dtype == lar.LAR_BF16 else torch.float32
    rand = lambda h: torch.randn(cfg.batch, h, 128, device=DEV, generator=g).to(td)
    k, v = rand(cfg.n_kv_heads).view(cfg.batch, cfg.n_kv_heads, 1, 128), rand(cfg.n_kv_heads).view(cfg.batch, cfg.n_kv_heads, 1, 128)
    cache.append_kv(0, k, v, 1)
    outs = []
    for line in range(lines):
        for _ in range(cfg.line_width):
            q = rand(cfg.n_q_heads)
            outs.append(torch.empty_like(q))
            cache.decode_step(0, q, rand(cfg.n_kv_heads), rand(cfg.n_kv_heads), outs[-1])
        cache.line_end_score_evict(0)
    assert cache.poll_device_status() == 0
    return torch.stack(outs)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("flags", [0, lar.LAR_FLAG_SCORE_CACHE_NORM])
def test_a_cache_goes_on_after_another_is_created(dtype, flags):
    """The kernels' limits of shared memory are those of all caches, not of the one that was created last."""
    first, again = (lar.Cache(_config(dtype, 1, 1, 24, 6, flags)) for _ in range(2))
    want = _generate(first, 8, 3)
    others = [lar.Cache(_config(dtype, 16, 32, 8, 4, flags)), lar.Cache(_config(dtype, 2, 2, 8, 4, flags)), lar.Cache(_config(dtype, 64, 4, 8, 4, flags))]
    assert torch.equal(_generate(again, 8, 3), want)
    for c in others:
        _generate(c, 6, 4)
    for c in (first, again, *others):
        c.close()
