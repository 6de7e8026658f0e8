"""What the calls on lists of gradients refuse, before anything reaches a GPU: the C entries with addresses that are never
followed, and the binding's lists with tensors on the CPU."""
import ctypes as C
import weakref

import numpy as np
import pytest
import torch

from paper_2512_20017_amd import binding as B

K = 1 << 20      # addresses this far apart do not overlap


def grad(at=1, n=1000, planes=3, dtype=0, out=None, visible=None):
    return B.CGradTensor(at * K, out, visible, n, planes, dtype)


def call(entry, tensors, max_norm=1.0, result=100 * K, ws=101 * K, ws_bytes=1 << 16, count=None):
    arr = (B.CGradTensor * max(1, len(tensors)))(*tensors)
    return getattr(B.lib(), entry)(C.c_int32(len(tensors) if count is None else count), arr, C.c_float(max_norm), C.c_void_p(result), C.c_void_p(ws),
                                   C.c_size_t(ws_bytes), None)


BOTH = pytest.mark.parametrize("entry", ["pbdr_grad_norm", "pbdr_grad_clip"])


@BOTH
@pytest.mark.parametrize("bad", [dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(result=None), dict(result=100 * K + 4), dict(ws=None),
                                 dict(ws=101 * K + 16), dict(count=-1), dict(count=B.PBDR_MAX_GRAD_TENSORS + 1)])
def test_arguments(entry, bad):
    assert call(entry, [grad()], **bad) == B.PBDR_ERR_INVALID_ARG


@BOTH
@pytest.mark.parametrize("bad", [dict(n=-1), dict(planes=-1), dict(dtype=3), dict(dtype=-1), dict(n=1 << 41, planes=1), dict(n=1 << 40, planes=2),
                                 dict(visible=8 * K + 4), dict(n=1 << 62, planes=4)])
def test_tensors(entry, bad):
    assert call(entry, [grad(), grad(**{"at": 5, **bad})]) == B.PBDR_ERR_INVALID_ARG


@BOTH
def test_addresses(entry):
    for t in (B.CGradTensor(None, None, None, 5, 1, 0), B.CGradTensor(K + 8, None, None, 5, 1, 0)):
        assert call(entry, [t]) == B.PBDR_ERR_INVALID_ARG
    assert call(entry, [grad()], ws_bytes=64) == B.PBDR_ERR_WORKSPACE_TOO_SMALL
    arr = None
    assert getattr(B.lib(), entry)(C.c_int32(1), arr, C.c_float(1), C.c_void_p(K), C.c_void_p(2 * K), C.c_size_t(1 << 16), None) == B.PBDR_ERR_INVALID_ARG


@BOTH
def test_results_and_workspaces_that_lie_on_a_tensor(entry):
    t = grad()      # 12000 bytes from K on
    for bad in (dict(result=K), dict(result=K + 11984), dict(ws=K + 256), dict(result=101 * K)):
        assert call(entry, [t], **bad) == B.PBDR_ERR_INVALID_ARG
    assert call(entry, [grad(visible=7 * K)], result=7 * K + 512) == B.PBDR_ERR_INVALID_ARG


@pytest.mark.parametrize("tensors", [
    [grad(), grad()],                                     # twice in place
    [grad(), grad(2, out=K + 512)],                       # one's output on another
    [grad(out=3 * K), grad(2, out=3 * K)],                # two into one place
    [grad(out=K + 16)],                                   # shifted by part of itself
    [grad(out=K + 10)],                                   # misaligned
    [grad(visible=9 * K), grad(2, out=9 * K)],            # output on a mask
    [grad(dtype=1, out=K + 5984)],
])
def test_what_clipping_writes_overlaps_nothing(tensors):
    assert call("pbdr_grad_clip", tensors) == B.PBDR_ERR_INVALID_ARG


def test_workspace_bytes():
    for count in (0, 1, 64, 65, B.PBDR_MAX_GRAD_TENSORS):
        assert 0 < B.pbdr_grad_workspace_bytes(count) <= 1 << 16 and B.pbdr_grad_workspace_bytes(count) % 256 == 0
    for count in (-1, B.PBDR_MAX_GRAD_TENSORS + 1):
        with pytest.raises(B.PbdrError):
            B.pbdr_grad_workspace_bytes(count)
    assert B.lib().pbdr_grad_workspace_bytes(C.c_int32(1), None) == B.PBDR_ERR_INVALID_ARG


def adam(param=1, g=2, m=3, v=4, n=1000, planes=3, lr=1e-3, visible=None, off=0):
    return B.CAdamTensor(param * K + off, g * K, m * K, v * K, visible, n, planes, lr)


def call_adam(tensors, result=100 * K, count=None, beta1=0.9, beta2=0.999, eps=1e-8, step=1, zero=0):
    arr = (B.CAdamTensor * max(1, len(tensors)))(*tensors)
    cfg = B.CAdamConfig(0.0, beta1, beta2, eps, step, zero)
    return B.lib().pbdr_adam_selective_list(C.c_int32(len(tensors) if count is None else count), arr, C.c_void_p(result), C.byref(cfg), None)


@pytest.mark.parametrize("bad", [dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0), dict(step=0),
                                 dict(result=100 * K + 8), dict(result=K), dict(count=-1), dict(count=B.PBDR_MAX_GRAD_TENSORS + 1)])
def test_adam_arguments(bad):
    assert call_adam([adam()], **bad) == B.PBDR_ERR_INVALID_ARG


@pytest.mark.parametrize("tensors", [
    [adam(n=-1)], [adam(planes=-1)], [adam(lr=-1.0)], [adam(lr=float("nan"))], [adam(off=4)], [adam(n=1 << 41)], [adam(visible=9 * K + 1)],
    [adam(g=1)], [adam(m=4)], [adam(), adam()], [adam(), adam(5, 1, 6, 7)], [adam(visible=4 * K)], [adam(), adam(off=11984, g=5, m=6, v=7)],
])
def test_adam_tensors(tensors):
    assert call_adam(tensors) == B.PBDR_ERR_INVALID_ARG


def test_adam_shares_a_gradient_only_where_it_stays():
    assert call_adam([adam(), adam(5, 2, 6, 7)], zero=1) == B.PBDR_ERR_INVALID_ARG
    assert B.lib().pbdr_adam_selective_list(C.c_int32(1), None, None, C.byref(B.CAdamConfig(0, 0.9, 0.9, 1e-8, 1, 0)), None) == B.PBDR_ERR_INVALID_ARG
    assert B.lib().pbdr_adam_selective_list(C.c_int32(0), None, None, None, None) == B.PBDR_ERR_INVALID_ARG


def test_lists_of_the_binding_describe_and_refuse():
    t = torch.zeros(3, 8)
    mask = torch.ones(8, dtype=torch.uint8)
    a = B.GradList([t, torch.zeros(4, 3, 8, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.float16)], visible=[mask, mask.bool(), None])
    got = [(x.data, x.visible, x.n, x.planes, x.dtype) for x in a.array()]
    assert [g[2:] for g in got] == [(8, 3, 0), (8, 12, 2), (5, 1, 1)]
    assert got[0][:2] == (t.data_ptr(), mask.data_ptr()) and got[2][1] is None
    assert [(x.n, x.planes) for x in B.GradList([t, torch.zeros(()), torch.zeros(0, 4)]).array()] == [(24, 1), (1, 1), (0, 1)]
    assert [(x.n, x.planes) for x in B.GradList([torch.zeros(3, 0)], visible=mask[:0]).array()] == [(0, 0)]
    for bad in (lambda: B.GradList([t.t()]), lambda: B.GradList([t.double()]), lambda: B.GradList([t], visible=mask[:7]),
                lambda: B.GradList([t], visible=mask.float()), lambda: B.GradList([t], visible=[mask, mask]), lambda: B.GradList([t], out=[t.half()]),
                lambda: B.GradList([t], out=[]), lambda: B.GradList([t], out=[torch.zeros(8, 3)]), lambda: B.GradList([torch.zeros(())], visible=mask),
                lambda: B.GradList([t], visible=torch.ones(16, dtype=torch.uint8)[::2]),
                lambda: B.AdamList([t], [t], [t], [t], []), lambda: B.AdamList([t], [t, t], [t], [t], [1.0]),
                lambda: B.AdamList([t.half()], [t.half()], [t.half()], [t.half()], [1.0]), lambda: B.AdamList([t], [torch.zeros(24)], [t], [t], [1.0])):
        with pytest.raises(ValueError):
            bad()
    # a tensor that got other memory is described anew
    before = a.array()[0].data
    keep, t.data = t.data, torch.zeros(3, 8)
    assert a.array()[0].data == t.data_ptr() != before
    t.data = torch.zeros(2, 8)
    assert a.array()[0].planes == 2
    del keep
    # nothing runs on the CPU
    result, ws = torch.zeros(8), torch.zeros(1 << 16, dtype=torch.uint8)
    with pytest.raises(ValueError):
        B.pbdr_grad_norm(a, 1.0, result, ws)
    with pytest.raises(ValueError):
        B.pbdr_grad_norm(a, 1.0, result[:4], ws)
    with pytest.raises(ValueError):
        B.pbdr_adam_selective_list(B.AdamList([t], [t.clone()], [t.clone()], [t.clone()], [1.0]), 0.9, 0.999, 1e-8, 1)
    adam_list = B.AdamList([t], [t.clone()], [t.clone()], [t.clone()], [1.0])
    adam_list.set_lrs([0.5])
    assert adam_list.array()[0].lr == 0.5
    with pytest.raises(ValueError):
        adam_list.set_lrs([0.5, 0.5])


# ------------------------------------------------------- tensors that change where they lie: what a list says of them changes with them
def same_place(change, shape=(4, 6), dtype=torch.float32, mask=None):
    """A list over a tensor at the begin of a larger buffer, described, then `change`; the address stays."""
    t = torch.zeros(1000, dtype=dtype)[:24].view(shape)
    at = t.data_ptr()
    lists = [B.GradList([t], visible=mask), B.GradList([torch.zeros_like(t)], visible=mask, out=[t])]
    if dtype == torch.float32:
        lists.append(B.AdamList([torch.zeros_like(t)], [torch.zeros_like(t)], [t], [torch.zeros_like(t)], [1.0], visible=mask))
    for a in lists:
        a.array()
    change(t)
    assert t.data_ptr() == at
    return t, lists


def whole(t, shape):      # the buffer that t lies in, from its begin
    return torch.empty(0, dtype=t.dtype).set_(t.untyped_storage(), 0, shape)


@pytest.mark.parametrize("shape", [(4, 3), (2, 6), (4, 60), (9, 6), (24,), (1,)])
@pytest.mark.parametrize("how", ["data", "resize_"])
def test_a_tensor_that_grows_or_shrinks_in_place(shape, how):
    def change(t):
        if how == "data":
            t.data = whole(t, shape)
        else:
            t.resize_(shape)
    t = whole(torch.zeros(1000), (4, 6))
    a = B.GradList([t])
    change(t)
    assert (a.array()[0].n, a.array()[0].planes) == (t.numel(), 1)
    t = whole(torch.zeros(1000), (4, 6))
    m, v, g = (whole(torch.zeros(1000), (4, 6)) for _ in range(3))
    a = B.AdamList([t], [g], [m], [v], [1.0])
    change(t)
    with pytest.raises(ValueError):      # the others have not changed yet
        a.array()
    for x in (g, m, v):
        change(x)
    assert (a.array()[0].n, a.array()[0].planes) == (t.numel(), 1)


@pytest.mark.parametrize("n", [3, 5, 7, 40])
def test_a_mask_and_its_tensors_that_change_together(n):
    t, mask = whole(torch.zeros(1000), (4, 6)), whole(torch.ones(100, dtype=torch.uint8), (6,))
    a = B.GradList([t], visible=mask)
    t.resize_(4, n)
    with pytest.raises(ValueError):
        a.array()
    mask.resize_(n)
    assert (a.array()[0].n, a.array()[0].planes) == (n, 4)
    mask.resize_(n - 1)
    with pytest.raises(ValueError):
        a.array()


def test_changes_in_place_that_no_list_takes():
    mask = torch.ones(6, dtype=torch.uint8)
    def transposed(t): t.data = whole(t, (6, 6)).t()
    def strided(t): t.data = whole(t, (4, 12))[:, ::2]
    def doubled(t): t.data = t.data.view(torch.float64)
    def folded(t): t.data = t.data.view(2, 12)      # points other than the mask's
    for change, with_mask in ((transposed, False), (strided, False), (strided, True), (doubled, False), (folded, True)):
        _, lists = same_place(change, mask=mask if with_mask else None)
        for a in lists:
            with pytest.raises(ValueError):
                a.array()
    square = whole(torch.zeros(100), (6, 6))      # nothing but the order of its values changes
    a = B.GradList([square])
    square.t_()
    with pytest.raises(ValueError):
        a.array()
    bits = torch.ones(6, dtype=torch.uint8)
    a = B.GradList([torch.zeros(2, 6)], visible=bits)
    bits.data = bits.data.view(torch.int8)
    with pytest.raises(ValueError):
        a.array()


def test_a_type_that_changes_in_place():
    t = torch.zeros(24, dtype=torch.float16)
    a = B.GradList([t])
    t.data = t.data.view(torch.bfloat16)
    assert (a.array()[0].dtype, a.array()[0].n) == (2, 24)
    t.data = t.data.view(torch.float32)
    assert (a.array()[0].dtype, a.array()[0].n) == (0, 12)


def test_a_list_is_described_once_while_nothing_changes():
    t = torch.zeros(3, 8)
    a = B.GradList([t], visible=torch.ones(8, dtype=torch.bool))
    first = a.array()
    t.add_(1.0)
    assert a.array() is first


def test_a_list_does_not_keep_memory_that_its_tensors_have_left():
    array = np.zeros((3, 8), dtype=np.float32)
    left = weakref.ref(array)
    t = torch.from_numpy(array)
    lists = [B.GradList([t]), B.GradList([torch.zeros(3, 8)], out=[t]), B.AdamList([t], *[[torch.zeros(3, 8)] for _ in range(3)], [1.0])]
    del array
    assert left() is not None
    t.data = torch.zeros(3, 8)
    assert left() is None and len(lists) == 3


def test_what_is_looked_at():
    t = torch.zeros(1000)[:24].view(4, 6)
    look = lambda x: B._tensor_look([x])      # noqa: E731
    others = [t.view(6, 4), t.view(24), t.view(1, 4, 6), t[:2], t[:, :5], t.t(), t.view(-1)[1:].view(23), t.view(torch.int32), torch.zeros(4, 6)]
    seen = [look(x) for x in others]
    assert look(t) == look(t.view(4, 6)) and look(t) not in seen and len(set(seen)) == len(seen)
    assert look(t.view(-1)[:12].view(torch.float16)) != look(t.view(-1)[:12].view(torch.bfloat16))
    assert B._tensor_look([]) == b"" and B._tensor_look([t, others[0]]) != B._tensor_look([others[0], t])
    for bad in (t, (t,), [t, None], [np.zeros(3)]):
        with pytest.raises(TypeError):
            B._tensor_look(bad)


def test_memory_shared_until_it_is_written_is_not_written():
    t = torch.zeros(3, 8)
    a = B.GradList([t])
    a.array()
    other = torch._lazy_clone(t)
    at = a.array()[0].data
    assert at == t.data_ptr() != other.data_ptr()
