"""What the operators on rows refuse, before anything reaches a GPU (the statuses of the C ABI, the binding's checks)."""
import pytest
import torch
from torch.autograd import forward_ad
from torch.fx.experimental.proxy_tensor import make_fx

from paper_1412_1576_b200 import binding as b
from paper_1412_1576_b200 import rows

P = 4096      # an address that is never looked at


def top(logits=P, dtype=b.LDA_F32, rows=2, V=10, stride=10, top=3, tau=1.0, ids=P, values=P, lse=P):
    return b.lda_top_logits(logits, dtype, rows, V, stride, top, tau, ids, values, lse)


def loss(logits=P, dtype=b.LDA_F32, rows=2, V=10, stride=10, ids=P, values=P, vt=b.LDA_F32, top=3, ls=3, lse=None, tau=1.0, out=P):
    return b.lda_distill_loss(logits, dtype, rows, V, stride, ids, values, vt, top, ls, lse, tau, out)


def grad(logits=P, dtype=b.LDA_F32, rows=2, V=10, stride=10, ids=P, values=P, vt=b.LDA_F32, top=3, ls=3, lse=None, tau=1.0, w=None,
         out=None, g=P + 4096, gs=10):
    return b.lda_distill_grad(logits, dtype, rows, V, stride, ids, values, vt, top, ls, lse, tau, w, out, g, gs)


def verify(off=P, n=2, drafts=P, nd=3, p=P, ps=10, q=P, qs=10, dtype=b.LDA_F32, V=10, au=P, du=P, tok=P, acc=P):
    return b.lda_verify_drafts(off, n, drafts, nd, p, ps, q, qs, dtype, V, au, du, tok, acc)


ROWS = [dict(dtype=3), dict(dtype=-1), dict(V=0), dict(V=-5), dict(rows=-1), dict(stride=-1), dict(logits=None), dict(logits=P + 2),
        dict(logits=P + 1, dtype=b.LDA_BF16), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")), dict(tau=float("inf")),
        dict(tau=1e-7), dict(top=0), dict(top=-1)]
TOO_LARGE = [dict(V=b.LDA_ROW_MAX_V + 1, stride=1 << 21), dict(rows=1 << 31), dict(stride=(1 << 31) + 1), dict(top=b.LDA_TOP_MAX + 1)]


@pytest.mark.parametrize("call", [top, loss, grad])
@pytest.mark.parametrize("bad", ROWS, ids=str)
def test_bad_rows_are_refused(call, bad):
    assert call(**bad) == b.LDA_EINVAL


@pytest.mark.parametrize("call", [top, loss, grad])
@pytest.mark.parametrize("bad", TOO_LARGE, ids=str)
def test_rows_beyond_the_limits_are_refused(call, bad):
    if call is grad and "V" in bad:
        bad = dict(bad, gs=bad["stride"])
    assert call(**bad) == b.LDA_ERANGE


@pytest.mark.parametrize("bad", [dict(ids=None), dict(values=None)], ids=str)
def test_lists_are_needed(bad):
    assert top(**bad) == loss(**bad) == grad(**bad) == b.LDA_EINVAL


@pytest.mark.parametrize("bad", [dict(vt=3), dict(ls=-1), dict(values=P + 2), dict(values=P + 1, vt=b.LDA_F16)], ids=str)
def test_bad_lists_are_refused(bad):
    assert loss(**bad) == grad(**bad) == b.LDA_EINVAL


def test_outputs_of_the_loss_are_needed():
    assert loss(out=None) == b.LDA_EINVAL
    assert grad(g=None) == b.LDA_EINVAL
    assert grad(gs=9) == b.LDA_EINVAL                          # rows of the gradient would overlap
    assert grad(g=P, stride=11, gs=10) == b.LDA_EINVAL         # in place: row for row
    assert grad(ls=(1 << 31) + 1) == b.LDA_ERANGE


@pytest.mark.parametrize("bad", [dict(off=None), dict(drafts=None), dict(p=None), dict(au=None), dict(du=None), dict(tok=None),
                                 dict(acc=None), dict(n=-1), dict(nd=-1), dict(V=0), dict(ps=-1), dict(qs=-1), dict(dtype=9),
                                 dict(p=P + 1), dict(q=P + 2), dict(n=0)], ids=str)
def test_bad_verifications_are_refused(bad):
    assert verify(**bad) == b.LDA_EINVAL


@pytest.mark.parametrize("bad", [dict(n=1 << 31), dict(nd=1 << 31), dict(V=b.LDA_ROW_MAX_V + 1), dict(qs=(1 << 31) + 1)], ids=str)
def test_verifications_beyond_the_limits_are_refused(bad):
    assert verify(**bad) == b.LDA_ERANGE


def test_misaligned_pointers_are_refused():
    assert top(ids=P + 2) == top(values=P + 2) == top(lse=P + 1) == b.LDA_EINVAL
    assert top(dtype=b.LDA_BF16, values=P + 1) == b.LDA_EINVAL
    for call in (loss, grad):
        assert call(ids=P + 1) == call(lse=P + 2) == call(out=P + 3) == b.LDA_EINVAL
    assert grad(w=P + 2) == grad(g=P + 2) == b.LDA_EINVAL
    assert verify(off=P + 4) == verify(drafts=P + 2) == verify(au=P + 1) == verify(du=P + 2) == verify(tok=P + 2) == verify(acc=P + 3) == b.LDA_EINVAL


def test_no_rows_is_nothing_to_do():
    assert top(rows=0, logits=None, ids=None, values=None, lse=None) == b.LDA_OK
    assert loss(rows=0, logits=None, ids=None, values=None, out=None) == b.LDA_OK
    assert grad(rows=0, logits=None, ids=None, values=None, g=None) == b.LDA_OK
    assert verify(n=0, nd=0, off=None, drafts=None, p=None, q=None, au=None, du=None, tok=None, acc=None) == b.LDA_OK


def test_tensors_of_the_host_are_refused():
    x = torch.zeros(2, 10)
    ids = torch.zeros(2, 3, dtype=torch.int32)
    values = torch.zeros(2, 3)
    with pytest.raises(ValueError, match="CUDA"):
        rows.top_logits(x, 3)
    with pytest.raises(ValueError, match="CUDA"):
        rows.distill_loss(x, ids, values)
    with pytest.raises(ValueError, match="CUDA"):
        rows.distill_loss(x.clone().requires_grad_(), ids, values)
    with pytest.raises(ValueError, match="CUDA"):
        rows.distill_loss_and_grad(x, ids, values)
    with pytest.raises(ValueError, match="CUDA"):
        rows.verify_drafts(torch.zeros(2, dtype=torch.int64), ids[0, :0], x[:1], None, x[0, :0], x[0, :1])


def test_a_gradient_over_saved_logits_is_noticed(monkeypatch):
    # (no GPU: the library's calls are left out, the tensors' bookkeeping is torch's)
    monkeypatch.setattr(rows, "_cuda", lambda x, name: x.device)
    monkeypatch.setattr(rows, "_call", lambda name, device, *args: None)
    x = torch.zeros(2, 10, requires_grad=True)
    ids, values = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)
    kept = rows.distill_loss(x, ids, values)
    rows.distill_loss_and_grad(x, ids, values)
    kept.sum().backward()
    lost = rows.distill_loss(x, ids, values)
    rows.distill_loss_and_grad(x, ids, values, grad=x.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        lost.sum().backward()


@pytest.mark.parametrize("shape", [(), (2, 2)], ids=str)
def test_drafts_that_are_no_vector_are_refused(monkeypatch, shape):
    monkeypatch.setattr(rows, "_cuda", lambda x, name: x.device)
    drafts = torch.zeros(shape, dtype=torch.int32)
    n = drafts.numel()
    with pytest.raises(ValueError, match="drafts"):
        rows.verify_drafts(torch.tensor([0, n]), drafts, torch.zeros(n + 1, 10), None, torch.zeros(n), torch.zeros(1))


def test_forward_mode_is_refused(monkeypatch):
    # (a tensor with a tangent need not require a gradient; no GPU: the library's calls are left out)
    monkeypatch.setattr(rows, "_cuda", lambda x, name: x.device)
    monkeypatch.setattr(rows, "_call", lambda name, device, *args: None)
    x, ids, values = torch.zeros(2, 10), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)
    with forward_ad.dual_level():
        for primal in (x, x.clone().requires_grad_()):
            dual = forward_ad.make_dual(primal, torch.ones(2, 10))
            with pytest.raises(NotImplementedError):
                rows.distill_loss(dual, ids, values)
            with torch.no_grad(), pytest.raises(NotImplementedError):
                rows.distill_loss(dual, ids, values)
        assert rows.distill_loss(x, ids, values).shape == (2,)      # without a tangent nothing is lost


def calls():
    """Each entry point as a function of one matrix of the host."""
    ids, values = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)
    offsets, drafts, u = torch.tensor([0, 1]), torch.zeros(1, dtype=torch.int32), torch.zeros(1)
    return [lambda x: rows.top_logits(x, 3), lambda x: rows.distill_loss(x, ids, values),
            lambda x: rows.distill_loss(x.detach().requires_grad_(), ids, values),
            lambda x: rows.distill_loss_and_grad(x, ids, values), lambda x: rows.verify_drafts(offsets, drafts, x, None, u, u)]


@pytest.mark.parametrize("which", range(5))
def test_tracing_is_refused(which):
    """A traced graph would hold the outputs' allocation alone."""
    call, x = calls()[which], torch.zeros(2, 10)
    with pytest.raises(RuntimeError, match="traced"):
        torch.jit.trace(call, x, check_trace=False)
    for before in (False, True):
        with pytest.raises(RuntimeError, match="traced"):
            make_fx(call, pre_dispatch=before)(x)
    with pytest.raises(ValueError, match="CUDA"):      # (and nothing of it is left)
        call(x)


@pytest.mark.parametrize("which", ["lse", "weights", "draft_probs"])
def test_tensors_without_memory_are_refused(monkeypatch, which):
    """What functionalize hands on has the address 0, which stands for `not given` in the library."""
    monkeypatch.setattr(rows, "_cuda", lambda x, name: x.device)
    monkeypatch.setattr(rows, "_call", lambda name, device, *args: None)
    x, ids, values = torch.zeros(2, 10), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3)
    offsets, drafts, u = torch.tensor([0, 1]), torch.zeros(1, dtype=torch.int32), torch.zeros(1)
    call, given = {"lse": (lambda t: rows.distill_loss(x, ids, values, t), torch.zeros(2)),
                   "weights": (lambda t: rows.distill_loss_and_grad(x, ids, values, weights=t), torch.zeros(2)),
                   "draft_probs": (lambda t: rows.verify_drafts(offsets, drafts, x, t, u, u), torch.zeros(1, 10))}[which]
    call(given)
    with pytest.raises(ValueError, match="memory"):
        torch.func.functionalize(call)(given)


def test_tokens_over_a_saved_index_are_noticed(monkeypatch):
    monkeypatch.setattr(rows, "_cuda", lambda x, name: x.device)
    monkeypatch.setattr(rows, "_call", lambda name, device, *args: None)
    table = torch.ones(5, 4, requires_grad=True)
    target, u = torch.zeros(3, 10), torch.zeros(3)
    offsets, drafts = torch.tensor([0, 1, 2]), torch.zeros(2, dtype=torch.int32)
    for name, n in (("tokens", 4), ("accepted", 2)):
        given = torch.zeros(n, dtype=torch.int32)
        kept = torch.nn.functional.embedding(given, table)
        rows.verify_drafts(offsets, drafts, torch.zeros(4, 10), None, u[:2], u[:2])
        kept.sum().backward()
        lost = torch.nn.functional.embedding(given, table)
        rows.verify_drafts(offsets, drafts, torch.zeros(4, 10), None, u[:2], u[:2], **{name: given})
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            lost.sum().backward()
