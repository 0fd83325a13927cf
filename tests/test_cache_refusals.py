"""What the operators on a paged cache refuse, before anything reaches a GPU (the statuses of the C ABI, the binding's checks)."""
import pytest
import torch
from torch.fx.experimental.proxy_tensor import make_fx

from paper_1412_1576_b200 import binding as b
from paper_1412_1576_b200 import cache, rows

P = 4096      # an address that is never looked at
GOOD = dict(keys=P, values=P, dtype=b.LDA_BF16, kv_heads=2, dim=64, page_size=16, pages=5, key_steps=(2048, 128, 64), value_steps=(2048, 128, 64), table=P,
            table_stride=4, n_seqs=2, starts=P, offsets=P, width=4)


def paged(**other):
    d = dict(GOOD, **other)
    return b.lda_paged_cache(d["keys"], d["values"], d["dtype"], d["kv_heads"], d["dim"], d["page_size"], d["pages"], d["key_steps"], d["value_steps"], d["table"],
                             d["table_stride"], d["n_seqs"], d["starts"], d["offsets"], d["width"])


def append(of=None, tokens=3, k=P, ks=(128, 64), v=P, vs=(128, 64), positions=None, freq=P, rotated=64, q=P, qs=(256, 64), heads=4, out=P + 4096,
           os=(256, 64), **c):
    return b.lda_append_cache(of or paged(**c), tokens, k, *ks, v, *vs, positions, freq, rotated, 0, q, *qs, heads, out, *os)


def attend(of=None, tokens=3, q=P, qs=(256, 64), heads=4, mask=P, ms=1, words=1, scale=0.125, out=P + 4096, os=(256, 64), space=P, size=1 << 40, **c):
    return b.lda_tree_attention(of or paged(**c), tokens, q, *qs, heads, mask, ms, words, scale, out, *os, space, size)


def tree(parents=P, offsets=P, n=2, tokens=3, starts=P, words=1, mask=P, positions=P):
    return b.lda_tree_mask(parents, offsets, n, tokens, starts, words, mask, positions)


BAD = [dict(dtype=b.LDA_F32), dict(dtype=7), dict(kv_heads=0), dict(dim=0), dict(dim=60), dict(dim=-8), dict(page_size=0), dict(pages=-1),
       dict(n_seqs=-1), dict(width=-1), dict(keys=None), dict(values=None), dict(keys=P + 8), dict(values=P + 2), dict(key_steps=(2048, 128, 63)),
       dict(value_steps=(2044, 128, 64)), dict(key_steps=(-8, 128, 64)), dict(table=None), dict(table=P + 2), dict(table_stride=-1), dict(starts=None),
       dict(starts=P + 1), dict(offsets=None), dict(offsets=P + 4), dict(tokens=-1)]
LARGE = [dict(dim=b.LDA_HEAD_MAX_DIM + 8), dict(kv_heads=b.LDA_HEADS_MAX + 1, heads=2 * b.LDA_HEADS_MAX + 2), dict(pages=1 << 31), dict(n_seqs=1 << 31),
         dict(tokens=1 << 31), dict(width=1 << 27), dict(key_steps=((1 << 31) + 8, 128, 64)), dict(value_steps=(8, 1 << 32, 64)), dict(table_stride=(1 << 31) + 1)]


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("bad", BAD, ids=str)
def test_bad_caches_are_refused(call, bad):
    assert call(**bad) == b.LDA_EINVAL


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("bad", LARGE, ids=str)
def test_caches_beyond_the_limits_are_refused(call, bad):
    assert call(**bad) == b.LDA_ERANGE
    assert b.lda_tree_attention_workspace(paged(**{k: v for k, v in bad.items() if k in GOOD}), bad.get("tokens", 3), bad.get("heads", 4)) == b.LDA_ERANGE


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(ks=(127, 64)), dict(vs=(128, -8)), dict(q=None),
                                 dict(out=None), dict(qs=(256, 60)), dict(os=(-256, 64)), dict(out=P, os=(512, 64)), dict(heads=-1),
                                 dict(rotated=63), dict(rotated=66), dict(rotated=-2), dict(freq=None), dict(freq=P + 2),
                                 dict(positions=P + 2)], ids=str)
def test_bad_appending_is_refused(bad):
    assert append(**bad) == b.LDA_EINVAL


def test_appending_beyond_the_limits_is_refused():
    assert append(heads=b.LDA_HEADS_MAX + 1) == append(qs=(1 << 32, 64)) == append(ks=(128, 1 << 32)) == b.LDA_ERANGE


@pytest.mark.parametrize("bad", [dict(q=None), dict(out=None), dict(q=P + 8), dict(out=P + 4), dict(qs=(256, 4)), dict(os=(-8, 64)), dict(heads=0),
                                 dict(heads=3), dict(heads=-2), dict(mask=P + 4), dict(words=0), dict(ms=-1), dict(scale=0.0), dict(scale=-1.0),
                                 dict(scale=float("nan")), dict(scale=1e7), dict(space=None), dict(space=P + 8), dict(size=1000)], ids=str)
def test_bad_attention_is_refused(bad):
    assert attend(**bad) == b.LDA_EINVAL


def test_attention_beyond_the_limits_is_refused():
    assert attend(heads=2 * b.LDA_HEADS_MAX) == attend(words=b.LDA_MASK_MAX_WORDS + 1) == attend(ms=1 << 32) == attend(qs=(1 << 32, 64)) == b.LDA_ERANGE


@pytest.mark.parametrize("bad", [dict(parents=None), dict(offsets=None), dict(mask=None), dict(parents=P + 2), dict(offsets=P + 4), dict(mask=P + 4),
                                 dict(starts=P + 1), dict(positions=P + 2), dict(words=0), dict(n=-1), dict(tokens=-1)], ids=str)
def test_bad_trees_are_refused(bad):
    assert tree(**bad) == b.LDA_EINVAL
    assert tree(words=b.LDA_MASK_MAX_WORDS + 1) == tree(n=1 << 31) == tree(tokens=1 << 31) == b.LDA_ERANGE


def test_the_workspace_is_enough_for_what_it_is_asked_for():
    need = b.lda_tree_attention_workspace(paged(), 3, 4)
    assert need > 0 and attend(size=need - 1) == b.LDA_EINVAL
    assert b.lda_tree_attention_workspace(paged(), 3, 3) == b.lda_tree_attention_workspace(paged(dim=60), 3, 4) == b.LDA_EINVAL


def test_nothing_to_do():
    none = dict(keys=None, values=None, pages=0, table=None, n_seqs=0, starts=None, offsets=None)
    assert append(of=paged(**none), k=None, v=None, q=None, out=None) == attend(of=paged(**none), q=None, out=None, space=None, size=0) == b.LDA_OK
    assert append(tokens=0, k=None, v=None, q=None, out=None) == attend(tokens=0, q=None, out=None, space=None, size=0) == b.LDA_OK
    assert tree(n=0, offsets=None, parents=None, mask=None) == tree(tokens=0, parents=None, mask=None) == b.LDA_OK
    assert b.lda_tree_attention_workspace(paged(), 0, 4) == 0
    assert b.lda_append_cache(None, 1, P, 8, 8, P, 8, 8, None, None, 0, 0) == b.LDA_EINVAL


# --- torch tensors -----------------------------------------------------------------------------------------------------------

def tensors(dtype=torch.bfloat16, tokens=3, pages=4, page=16, kv_heads=2, dim=64, heads=4):
    d = dict(k_cache=torch.zeros(pages, page, kv_heads, dim, dtype=dtype), v_cache=torch.zeros(pages, page, kv_heads, dim, dtype=dtype),
             table=torch.zeros(2, 2, dtype=torch.int32), starts=torch.zeros(2, dtype=torch.int32), offsets=torch.zeros(3, dtype=torch.int64))
    return d, torch.zeros(tokens, heads, dim, dtype=dtype), torch.zeros(tokens, kv_heads, dim, dtype=dtype)


def call_append(d, queries, kv, **other):
    return cache.append_cache(other.pop("k", kv), other.pop("v", kv), *d.values(), q=other.pop("q", queries), **other)


def call_attend(d, queries, kv, **other):
    return cache.tree_attention(other.pop("q", queries), *d.values(), **other)


def test_tensors_of_the_host_are_refused():
    for call in (call_append, call_attend):
        with pytest.raises(ValueError, match="CUDA"):
            call(*tensors())
    with pytest.raises(ValueError, match="CUDA"):
        cache.tree_mask(torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int64), None, 3)


@pytest.fixture
def no_gpu(monkeypatch):
    """The library's calls are left out; the checks and the tensors' bookkeeping are looked at."""
    calls = []
    monkeypatch.setattr(cache, "_cuda", lambda x, name: x.device)
    monkeypatch.setattr(cache, "_call", lambda name, device, *args: calls.append(name))
    return calls


CACHES = [(dict(k_cache=torch.zeros(4, 16, 2, 64)), TypeError, "k_cache"), (dict(v_cache=torch.zeros(4, 16, 2, 64, dtype=torch.float16)), TypeError, "v_cache"),
          (dict(v_cache=torch.zeros(4, 16, 2, 72, dtype=torch.bfloat16)), ValueError, "k_cache and v_cache"),
          (dict(table=torch.zeros(3, 2, dtype=torch.int32)), ValueError, "table"), (dict(table=torch.zeros(2, 2, dtype=torch.int64)), TypeError, "table"),
          (dict(table=torch.zeros(2, 4, dtype=torch.int32)[:, ::2]), ValueError, "table"), (dict(starts=torch.zeros(3, dtype=torch.int32)), ValueError, "starts"),
          (dict(starts=torch.zeros(2, dtype=torch.int64)), TypeError, "starts"), (dict(offsets=torch.zeros(3, dtype=torch.int32)), TypeError, "offsets"),
          (dict(offsets=torch.zeros(0, dtype=torch.int64)), ValueError, "offsets"),
          (dict(k_cache=torch.zeros(4, 16, 2, 65, dtype=torch.bfloat16)[..., :64]), ValueError, "k_cache"),
          (dict(k_cache=torch.zeros(4, 16, 2, 128, dtype=torch.bfloat16)[..., ::2]), ValueError, "k_cache"),
          (dict(k_cache=torch.zeros(8193, dtype=torch.bfloat16)[1:].view(4, 16, 2, 64)), ValueError, "k_cache")]


@pytest.mark.parametrize("call", [call_append, call_attend])
@pytest.mark.parametrize("other,error,name", CACHES, ids=[f"{c[2]}{i}" for i, c in enumerate(CACHES)])
def test_caches_of_another_kind_are_refused(no_gpu, call, other, error, name):
    d, q, kv = tensors()
    call(d, q, kv)
    assert no_gpu
    with pytest.raises(error, match=name):
        call(dict(d, **other), q, kv)
    for dim in (60, 264):
        d, q, kv = tensors(dim=dim)
        with pytest.raises(ValueError, match="k_cache"):
            call(d, q, kv)


def test_rows_of_another_kind_are_refused(no_gpu):
    d, q, kv = tensors()
    for other, error in ((dict(k=kv[:2]), ValueError), (dict(k=kv.float()), TypeError), (dict(v=q), ValueError), (dict(v=kv[..., :56]), ValueError),
                         (dict(q=q[:2]), ValueError), (dict(q=q.half()), TypeError), (dict(q=None, q_out=q), ValueError),
                         (dict(q_out=q[:2]), ValueError), (dict(q_out=q.float()), TypeError), (dict(q=q[:, :0]), ValueError),
                         (dict(positions=torch.zeros(2, dtype=torch.int32)), ValueError), (dict(positions=torch.zeros(3, dtype=torch.int64)), TypeError),
                         (dict(inv_freq=torch.zeros(33)), ValueError), (dict(inv_freq=torch.zeros(8).double()), TypeError)):
        with pytest.raises(error):
            call_append(d, q, kv, **other)
    for other, error in ((dict(q=q[:, :3]), ValueError), (dict(q=q.float()), TypeError), (dict(q=q[0]), ValueError), (dict(scale=0.0), ValueError),
                         (dict(scale=float("nan")), ValueError), (dict(mask=torch.zeros(3, 1)), TypeError), (dict(out=q[:2]), ValueError),
                         (dict(mask=torch.zeros(2, 1, dtype=torch.int64)), ValueError), (dict(mask=torch.zeros(3, 0, dtype=torch.int64)), ValueError),
                         (dict(mask=torch.zeros(3, 65, dtype=torch.int64)), ValueError), (dict(mask=torch.zeros(3, 4, dtype=torch.int64)[:, ::2]), ValueError)):
        with pytest.raises(error):
            call_attend(d, q, kv, **other)
    parents, offsets = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)
    for args, error in (((parents, offsets, None, 0), ValueError), ((parents, offsets, None, 4097), ValueError), ((parents.long(), offsets, None, 3), TypeError),
                        ((parents, offsets.int(), None, 3), TypeError), ((parents, offsets, parents, 3), ValueError), ((parents, offsets[:0], None, 3), ValueError)):
        with pytest.raises(error):
            cache.tree_mask(*args)


def test_what_autograd_follows_is_refused(no_gpu):
    d, q, kv = tensors()
    followed = q.clone().requires_grad_()
    with pytest.raises(ValueError, match="differentiable"):
        call_attend(d, followed, kv)
    with pytest.raises(ValueError, match="differentiable"):
        call_append(d, followed, kv)
    with pytest.raises(ValueError, match="written"):
        call_append(dict(d, k_cache=d["k_cache"].clone().requires_grad_()), q, kv)
    with pytest.raises(ValueError, match="out"):
        call_attend(d, q, kv, out=followed)
    with torch.no_grad():
        call_attend(d, followed, kv)
        call_append(d, followed, kv)
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(ValueError, match="differentiable"):
            call_attend(d, torch.autograd.forward_ad.make_dual(q, q), kv)


def test_tracing_is_refused():
    d, q, kv = tensors()
    with pytest.raises(RuntimeError, match="traced"):
        make_fx(lambda q: cache.tree_attention(q, *d.values()))(q)


def test_caches_that_are_written_go_up_in_version(no_gpu):
    d, q, kv = tensors()
    out = torch.zeros_like(q)
    before = [x._version for x in (d["k_cache"], d["v_cache"], out)]
    call_append(d, q, kv, q_out=out)
    assert all(x._version > n for x, n in zip((d["k_cache"], d["v_cache"], out), before))
    before = out._version
    call_attend(d, q, kv, out=out)
    assert out._version > before
