"""Group norm over sequences with many narrow groups (instance norm), where a workgroup has hundreds of groups at once.  References
and tolerances are those of test_gpu_group_norm.py (the formulas in 64 bits)."""
import pytest

from test_gpu_group_norm import _check, g  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("items,length,channels,groups", [(2, 600, 1024, 1024), (1, 520, 768, 768), (1, 1000, 1536, 768), (1, 600, 516, 516), (1, 700, 1544, 1544), (1, 530, 2048, 1024),
                                                          (1, 300, 1944, 648), (1, 600, 512, 512), (1, 515, 513, 513), (1, 513, 2100, 2100)])
def test_hundreds_of_narrow_groups(g, dtype, items, length, channels, groups):  # noqa: F811
    _check(g, dtype, items, length, channels, groups, "silu", seed=groups)


def test_every_group_has_its_own_statistics(g):  # noqa: F811
    """Channel c holds c or c + 1, half of the time each: mean c + 0.5, variance 0.25, all exact."""
    import torch
    for dtype, C in ((torch.float32, 2048), (torch.bfloat16, 256), (torch.float16, 1024)):
        x = torch.arange(C, device="cuda", dtype=torch.float32).expand(1, 600, C).clone()
        x[:, ::2] += 1
        if dtype == torch.bfloat16:  # whole numbers up to 256
            x = x.repeat(1, 1, 5)
        x = x.to(dtype)
        _, mean, rstd = g.group_norm(x, x.shape[-1], eps=0.0, want_stats=True)
        assert torch.equal(mean[0], x[0, 1].float() + 0.5) and torch.equal(rstd, torch.full_like(rstd, 2.0))
