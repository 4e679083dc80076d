"""The cases by which the 8-bit attention's few rows are held to their weights tell a weight's parts apart: emulated on the host."""
import pytest
import torch

from paged8_weights import bounds, case, weights


def emulate(pool, q, live, dtype, how):
    """Outputs from weights against a maximum that is up to 2^8 below (as the running one may be), in the parts of `how`."""
    w, v, _ = weights(pool, q, live)
    p = (w / w.amax(-1, keepdim=True) * 1.37).float()
    hi = p.bfloat16().float()
    rest = (p - hi).bfloat16().float()
    low = (p - hi - rest).bfloat16().float()
    rows = torch.arange(p.shape[0] * p.shape[1]).view(p.shape[:2])
    parts = {"kept": hi + rest, "three": hi.double() + rest + low, "lost": hi, "turned": hi - rest,
             "lost in one row": torch.where((rows == rows.max() // 2)[..., None], hi, hi + rest)}[how]
    out = parts.double() @ v / p.double().sum(-1, keepdim=True)
    return out.to(torch.bfloat16 if dtype == "bf16" else torch.float32).double()


SHAPES = [(n, m, H) for n in (8, 40, 900, 9000) for m, H in ((1, 4), (1, 16), (1, 17), (2, 9), (1, 32), (4, 8))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,m,H", SHAPES)
def test_bound_tells_parts_apart(n, m, H, dtype):
    pool, q, live = case(n, m, H, dtype)
    ref, tol = bounds(pool, q, live, m, H, dtype)
    worst = lambda how: float(((emulate(pool, q, live, dtype, how) - ref).abs() / tol).max())
    assert worst("kept" if dtype == "bf16" else "three") <= 1
    assert worst("lost") > 1.5 and worst("turned") > 1.5 and worst("lost in one row") > 1.5
