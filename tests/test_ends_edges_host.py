"""What autograd keeps of the operators at the ends of a model.  Nothing here needs a GPU: the library's calls are left out."""
import pytest
import torch


@pytest.fixture
def prism(monkeypatch):
    """The binding on tensors of the host, whose results hold anything: checks and allocations only."""
    from paper_2601_22137_amd import prism as P
    monkeypatch.setattr(P, "lib", lambda: type("Nothing", (), {"__getattr__": lambda self, name: None})())
    monkeypatch.setattr(P, "_device", lambda t: t.get_device())
    monkeypatch.setattr(P, "_scratch", lambda *a: (b"", None))
    monkeypatch.setattr(P, "_on", lambda *a: None)
    return P


@pytest.mark.parametrize("gradient", [False, True])
def test_results_of_the_loss_are_tensors_of_their_own(prism, gradient):
    r = prism.policy_loss(torch.randn(2, 3, 7), torch.zeros(2, 3, dtype=torch.int64), gradient=gradient)
    rows = r.logp, r.lse, r.dlogp
    assert all(t.shape == (2, 3) and t.is_contiguous() and t.dtype is torch.float32 and t.untyped_storage().nbytes() == 24 for t in rows)
    r.logp.neg_()
    assert [t._version for t in rows] == [1, 0, 0]


def test_log_probabilities_may_be_written_to_before_the_backward_pass(prism):
    from paper_2601_22137_amd import layers
    z = torch.randn(5, 7, requires_grad=True)
    loss, logp = layers.policy_loss(z, torch.zeros(5, dtype=torch.int64))
    logp.clamp_(max=0.0)
    logp.detach().mul_(0.5)
    loss.backward()
    assert z.grad.shape == z.shape


def test_tangents_are_not_lost(prism):
    """no_grad does not turn forward mode off: an argument with a tangent, for which the operators have no derivative, is an error there too."""
    from paper_2601_22137_amd import layers
    import torch.autograd.forward_ad as forward
    x, w, tokens = torch.randn(3, 8), torch.ones(8), torch.zeros(3, dtype=torch.int64)
    heads, freq = torch.randn(1, 3, 2, 8), torch.ones(4)
    norm_rope = lambda q=heads, k=heads, qw=w, kw=w, f=freq: layers.norm_rope(q, k, qw, kw, inv_freq=f)   # noqa: E731
    calls = [(layers.embedding, (tokens, x), 1)] + [(lambda *a: layers.layer_norm(*a), (x, w, w, x), i) for i in range(4)] + [(norm_rope, (heads, heads, w, w, freq), i) for i in range(5)]
    with forward.dual_level():
        for call, args, i in calls:
            dual = list(args)
            dual[i] = forward.make_dual(args[i], torch.ones_like(args[i]))
            with torch.no_grad():
                call(*args)
                with pytest.raises((NotImplementedError, layers.prism.PrismError), match="jvp|inv_freq"):
                    call(*dual)
            with torch.inference_mode():                 # where forward mode is off
                call(*dual)
