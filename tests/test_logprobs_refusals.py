"""What the log probabilities of tokens refuse, before anything reaches a GPU."""
import pytest
import torch
from torch.autograd import forward_ad
from torch.fx.experimental.proxy_tensor import make_fx

from paper_1412_1576_b200 import binding as b
from paper_1412_1576_b200 import rows

P = 4096      # an address that is never looked at


def logp(logits=P, dtype=b.LDA_F32, rows=2, V=10, stride=10, tokens=P, top=3, tau=1.0, lp=P, entropy=P, stats=P, ids=P, alternatives=P):
    return b.lda_token_logprobs(logits, dtype, rows, V, stride, tokens, top, tau, lp, entropy, stats, ids, alternatives)


def grad(logits=P, dtype=b.LDA_F32, rows=2, V=10, stride=10, tokens=P, stats=P, w=P, h=P, tau=1.0, g=P + 4096, gs=10):
    return b.lda_token_logprobs_grad(logits, dtype, rows, V, stride, tokens, stats, w, h, tau, g, gs)


BOTH = [dict(dtype=3), dict(dtype=-1), dict(V=0), dict(rows=-1), dict(stride=-1), dict(logits=None), dict(logits=P + 2), dict(tokens=None), dict(tokens=P + 2),
        dict(stats=P + 1), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")), dict(tau=1e7), dict(tau=1e-7)]


@pytest.mark.parametrize("call", [logp, grad])
@pytest.mark.parametrize("bad", BOTH, ids=str)
def test_bad_rows_are_refused(call, bad):
    assert call(**bad) == b.LDA_EINVAL


@pytest.mark.parametrize("bad", [dict(top=-1), dict(lp=None), dict(entropy=None), dict(ids=None), dict(alternatives=None), dict(lp=P + 2), dict(entropy=P + 1),
                                 dict(ids=P + 2), dict(alternatives=P + 1)], ids=str)
def test_bad_outputs_are_refused(bad):
    assert logp(**bad) == b.LDA_EINVAL


@pytest.mark.parametrize("bad", [dict(stats=None), dict(g=None), dict(g=P + 2), dict(gs=9), dict(g=P, gs=12), dict(w=P + 2), dict(h=P + 1)], ids=str)
def test_bad_gradients_are_refused(bad):
    assert grad(**bad) == b.LDA_EINVAL


def test_sizes_beyond_the_limits_are_refused():
    for call in (logp, grad):
        assert call(rows=1 << 31) == call(stride=(1 << 31) + 1) == b.LDA_ERANGE
        assert call(V=b.LDA_ROW_MAX_V + 1, stride=1 << 21, **({} if call is logp else {"gs": 1 << 21})) == b.LDA_ERANGE
    assert logp(top=b.LDA_TOP_MAX + 1) == grad(gs=(1 << 31) + 1) == b.LDA_ERANGE


def test_no_rows_is_nothing_to_do():
    assert logp(rows=0, logits=None, tokens=None, lp=None, entropy=None, ids=None, alternatives=None) == b.LDA_OK
    assert grad(rows=0, logits=None, tokens=None, stats=None, g=None) == b.LDA_OK


def test_tensors_of_another_kind_are_refused(monkeypatch):
    x, tokens = torch.zeros(2, 10), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        rows.token_logprobs(x, tokens)
    with pytest.raises(ValueError, match="CUDA"):
        rows.token_logprobs_grad(x, tokens, torch.zeros(2, 3))
    with pytest.raises(RuntimeError, match="traced"):
        make_fx(lambda x: rows.token_logprobs(x, tokens))(x)
    monkeypatch.setattr(rows, "_cuda", lambda x, name: x.device)
    calls = []
    monkeypatch.setattr(rows, "_call", lambda name, device, *args: calls.append(name))
    got = rows.token_logprobs(x, tokens, top=3)
    assert calls == ["lda_token_logprobs"] and got.ids.shape == got.alternatives.shape == (2, 3) and got.stats.shape == (2, 3)
    assert rows.token_logprobs(x, tokens).ids is None
    for args, error in (((x.double(), tokens), TypeError), ((x[0], tokens), ValueError), ((x, tokens.long()), TypeError), ((x, tokens[:1]), ValueError),
                        ((x, tokens, -1), ValueError), ((x, tokens, b.LDA_TOP_MAX + 1), ValueError), ((x.t(), tokens), ValueError)):
        with pytest.raises(error):
            rows.token_logprobs(*args)
    stats, w = got.stats, torch.zeros(2)
    rows.token_logprobs_grad(x, tokens, stats, w, w)
    for kwargs, error in ((dict(stats=stats[:1]), ValueError), (dict(stats=stats.double()), TypeError), (dict(stats=torch.zeros(3, 2).t()), ValueError),
                          (dict(logprob_weights=w[:1]), ValueError), (dict(entropy_weights=w.double()), TypeError), (dict(grad=x.half()), ValueError),
                          (dict(grad=torch.zeros(2, 9)), ValueError), (dict(grad=x.clone().requires_grad_()), ValueError)):
        with pytest.raises(error):
            rows.token_logprobs_grad(x, tokens, **dict(dict(stats=stats), **kwargs))
    with forward_ad.dual_level():
        with pytest.raises(NotImplementedError):
            rows.token_logprobs(forward_ad.make_dual(x, x), tokens)


def test_a_second_derivative_is_refused(monkeypatch):
    monkeypatch.setattr(rows, "_cuda", lambda x, name: x.device)
    monkeypatch.setattr(rows, "_call", lambda name, device, *args: None)
    x = torch.zeros(2, 10, requires_grad=True)
    got = rows.token_logprobs(x, torch.zeros(2, dtype=torch.int32))
    grad, = torch.autograd.grad(got.logprobs.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()
