"""The 8-bit rollout example's autograd function without a GPU: what it asks of the library's calls, which are replaced by their formulas."""
import pytest
import torch

from examples import rollout_8bit as E


@pytest.fixture
def asked(monkeypatch):
    """The calls replaced; a list of what each backward call was asked for."""
    calls = []

    def z_of(x, w, cos_sin, positions):
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + E.EPS) * (1.0 if w is None else w)
        c, s = cos_sin[positions.long()][:, None].chunk(2, -1)
        a, b = y.chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    def forward(q, k, qw, kw, cos_sin, positions, eps, q_out, k_out):
        assert eps == E.EPS
        with torch.no_grad():
            q_out.copy_(z_of(q, qw, cos_sin, positions)), k_out.copy_(z_of(k, kw, cos_sin, positions))
        return q_out, k_out

    def backward(dq_out, dk_out, q, k, qw, kw, cos_sin, positions, eps, dq, dk, dqw, dkw, ws):
        assert dq_out.is_contiguous() and dk_out.is_contiguous()
        calls.append((dqw is not None, dkw is not None))
        for dz, x, w, dx, dw in ((dq_out, q, qw, dq, dqw), (dk_out, k, kw, dk, dkw)):
            with torch.enable_grad():
                leaf = [t.detach().clone().requires_grad_() for t in ((x,) if w is None else (x, w))]
                g = torch.autograd.grad(z_of(leaf[0], None if w is None else leaf[1], cos_sin, positions), leaf, dz.detach())
            dx.copy_(g[0])
            if dw is not None:
                assert w is not None
                dw.copy_(g[1])
        return dq, dk, dqw, dkw

    monkeypatch.setattr(E.B, "marl_qk_norm_rope", forward)
    monkeypatch.setattr(E.B, "marl_qk_norm_rope_backward", backward)
    return calls


def operands(seed=0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    q, k, qw, kw = rnd(5, 3, E.D), rnd(5, 2, E.D), 1 + rnd(E.D) / 8, 1 + rnd(E.D) / 8
    angle = rnd(9, E.D // 2)
    return [t.requires_grad_() for t in (q, k, qw, kw)], torch.cat([angle.cos(), angle.sin()], 1), torch.tensor([0, 8, 3, 4, 4], dtype=torch.int32)


def test_all_gradients(asked):
    leaves, cs, pos = operands()
    q_out, k_out = E.QkNormRope.apply(*leaves, cs, pos)
    (q_out.sum() + (k_out * 2).sum()).backward()
    assert asked == [(True, True)] and all(t.grad is not None and bool(t.grad.any()) for t in leaves)


def test_heads_without_weights(asked):
    (q, k, qw, _), cs, pos = operands()
    q_out, k_out = E.QkNormRope.apply(q, k, None, None, cs, pos)
    (q_out.sum() + k_out.sum()).backward()
    assert asked == [(False, False)] and bool(q.grad.any()) and bool(k.grad.any())
    q_out, k_out = E.QkNormRope.apply(q, k, qw, None, cs, pos)
    (q_out.sum() + k_out.sum()).backward()
    assert asked[1:] == [(True, False)] and bool(qw.grad.any())


def test_only_what_is_wanted(asked):
    (q, k, qw, kw), cs, pos = operands()
    q_out, k_out = E.QkNormRope.apply(q, k.detach(), qw.detach(), kw, cs, pos)
    (q_out.sum() + k_out.sum()).backward()
    assert asked == [(False, True)] and q.grad is not None and kw.grad is not None and qw.grad is None and k.grad is None


def test_no_second_derivative(asked):
    leaves, cs, pos = operands()
    q_out, _ = E.QkNormRope.apply(*leaves, cs, pos)
    dq, = torch.autograd.grad((q_out * q_out).sum(), leaves[0], create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (dq.sum() + leaves[0].sum()).backward()     # (else the first term would be left out without a word)
