"""The weights' gradients of the head norms over so many tokens that thousands of workgroups leave sums to be added up (GPU)."""
import pytest
import torch

from paper_2604_04215_amd import binding as dlm
from gpu_util import DEV

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8
BF16, EPS = torch.bfloat16, 1e-6


def grads(dy, x, w):
    """Of one part in 64 bits, some tokens at a time: (dx, what is added up for it, sum of dz n, sum of |dz n|)."""
    dw, size, dx, add = 0, 0, [], []
    for a, b in zip(dy.split(4096), x.split(4096)):
        a, b, wide = a.double(), b.double(), w.double()
        r = (b.square().mean(-1, keepdim=True) + EPS).rsqrt()
        n, g = b * r, a * wide
        dw, size = dw + (a * n).sum((0, 1)), size + (a * n).abs().sum((0, 1))
        dx.append((r * (g - n * (g * n).mean(-1, keepdim=True))).float())
        add.append((r * (g.abs() + n.abs() * (g * n).abs().mean(-1, keepdim=True))).float())
    return torch.cat(dx), torch.cat(add), dw, size


@pytest.mark.parametrize("T,Hq,Hkv,d,least", [(20000, 32, 2, 128, 900), (66000, 64, 1, 64, 4096), (33000, 64, 2, 128, 4096), (140000, 64, 1, 64, 8193), (70000, 64, 2, 128, 8193)])
def test_sums_of_thousands_of_workgroups(T, Hq, Hkv, d, least):
    """Upstream gradients that go along with the heads, so that every workgroup's row adds to a sum of one sign: one that is left out or added twice shows.  Bounds as in the
    tests of the gradient: 400 u of what is added up, and for a head's gradient a rounding to bf16."""
    gen = torch.Generator(device=DEV).manual_seed(T)
    normal = lambda *shape: torch.randn(shape, generator=gen, device=DEV, dtype=BF16)
    x = [normal(T, h, d) for h in (Hq, Hkv)]
    dy = [t + normal(*t.shape) * 0.5 for t in x]
    w = [(1 + 0.2 * normal(d).float()).to(BF16) for _ in range(2)]
    dx, dw = [torch.empty_like(t) for t in x], [torch.full((d,), 5.0, device=DEV) for _ in range(2)]
    ws = torch.empty(dlm.qk_norm_rope_bwd_workspace_bytes(T, Hq, Hkv, d), dtype=torch.uint8, device=DEV)
    groups = ws.numel() // (4 * d)
    assert groups > least
    call = lambda: dlm.qk_norm_rope_bwd(dy[0], dy[1], dx[0], dx[1], q=x[0], k=x[1], q_weight=w[0], k_weight=w[1], d_q_weight=dw[0], d_k_weight=dw[1], eps=EPS, workspace=ws)
    call()
    for got, got_w, g, t, wt in zip(dx, dw, dy, x, w):
        want, add, want_w, size = grads(g, t, wt)
        bound = 400 * U * size
        assert (want_w / groups > bound).all()                  # (a workgroup's share is more than the bound)
        assert ((got_w - want_w).abs() <= bound).all(), ((got_w - want_w).abs() / bound).max()
        assert ((got - want).abs() <= H * want.abs() * (1 + H) + 400 * U * add * (1 + H) + 2.0 ** -133).all()
    again = [t.clone() for t in dx + dw]
    call()
    assert all(torch.equal(a, b) for a, b in zip(again, dx + dw))
