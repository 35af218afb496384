"""Argument checks of the calls for drafted tokens, without a GPU: every refused call
returns its status before anything is enqueued or any pointer is read; and their
structures against the header."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2608_15383_amd import _lib, api
from paper_2608_15383_amd._lib import EMOE_EINVAL, EMOE_ESHAPE, EMOE_F16, EMOE_F32, EMOE_OK
from tests.test_serving_refusals import P, append, status
from tests.test_serving_refusals import kv as cache

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                      "exactmoe_drafts.h")
SCALARS = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float}


@pytest.mark.parametrize("name,view", [
    ("emoe_paged_axes", _lib.PagedAxes), ("emoe_paged_tree_args", _lib.PagedTreeArgs),
    ("emoe_accept_args", _lib.AcceptArgs), ("emoe_compact_args", _lib.CompactArgs),
    ("emoe_fork_args", _lib.ForkArgs)])
def test_structures(name, view):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, re.S).group(1)
    want = []
    for line in filter(None, (d.strip() for d in body.split(";"))):
        kind, names = re.match(r"(?:const\s+)?(\w+)\s*(.*)", line, re.S).groups()
        for n in names.split(","):
            pointer, n = "*" in n, n.replace("*", "").strip()
            want.append((n, C.c_void_p if pointer else SCALARS[kind]))
    assert [tuple(f) for f in view._fields_] == want


def kv(layer=0, **kw):
    at = P + (2 * layer << 20)
    return cache(**{**dict(k_pages=at, v_pages=at + (1 << 20)), **kw})


def axes(**kw):
    return _lib.PagedAxes(**{**dict(angles=P, axes=P, angle_stride=3, n_axes=3), **kw})


def tree(**kw):
    f = dict(q=P, out=P, lengths=P, starts=P, page_table=P, q_stride=2048, out_stride=2048,
             table_stride=8, scale=0.1, dtype=_lib.EMOE_BF16, rows=9, trees=3, n_heads=16, n_seqs=3,
             table_width=8, max_keys=128, max_nodes=5)
    return _lib.PagedTreeArgs(**{**f, **kw})


def accept(**kw):
    f = dict(tokens=P, chosen=P, tree=P, starts=P, lengths=P, path=P, accepted=P, new_tokens=P,
             new_lengths=P, path_stride=5, new_tokens_stride=5, rows=9, trees=3, max_nodes=5)
    return _lib.AcceptArgs(**{**f, **kw})


def compact(**kw):
    f = dict(lengths=P, path=P, accepted=P, page_table=P, path_stride=5, table_stride=8, trees=3,
             max_nodes=5, n_seqs=3, table_width=8)
    return _lib.CompactArgs(**{**f, **kw})


def fork(**kw):
    f = dict(page_table=P, parents=P, lengths=P, fresh=P, new_table=P + 4096, table_stride=8,
             new_table_stride=8, forks=3, n_seqs=3, table_width=8)
    return _lib.ForkArgs(**{**f, **kw})


@pytest.mark.parametrize("change,want", [
    (dict(n_axes=0), EMOE_EINVAL),
    (dict(n_axes=-1), EMOE_EINVAL),
    (dict(angles=None), EMOE_EINVAL),
    (dict(angle_stride=2), EMOE_EINVAL),
])
def test_axes_checks(change, want):
    call = lambda a, x: status("emoe_paged_append_axes", C.byref(kv()), C.byref(a), x, None)
    assert call(append(), C.byref(axes(**change))) == want
    assert call(append(tokens=0), C.byref(axes())) == EMOE_OK
    assert call(append(tokens=0, rotary_dim=0), C.byref(axes(angles=None))) == EMOE_OK
    assert call(append(), None) == EMOE_EINVAL
    assert call(append(k=None), C.byref(axes())) == EMOE_EINVAL
    assert status("emoe_paged_append_axes", None, C.byref(append()), C.byref(axes()), None) == EMOE_EINVAL


@pytest.mark.parametrize("change,want", [
    (dict(rows=0, q=None), EMOE_OK),
    (dict(trees=0, q=None), EMOE_OK),
    (dict(rows=-1), EMOE_EINVAL),
    (dict(trees=-1), EMOE_EINVAL),
    (dict(max_keys=-1), EMOE_EINVAL),
    (dict(window=-1), EMOE_EINVAL),
    (dict(max_nodes=0), EMOE_ESHAPE),
    (dict(max_nodes=65), EMOE_ESHAPE),
    (dict(starts=None), EMOE_ESHAPE),                    # 9 rows are not 3 trees of 5
    (dict(starts=None, rows=15, trees=1 << 30, max_nodes=64), EMOE_ESHAPE),
    (dict(n_heads=0), EMOE_ESHAPE),
    (dict(n_heads=6), EMOE_ESHAPE),
    (dict(n_heads=1 << 21, q_stride=1 << 28, out_stride=1 << 28), EMOE_ESHAPE),
    (dict(n_heads=1 << 20, max_nodes=64, q_stride=1 << 28, out_stride=1 << 28), EMOE_ESHAPE),
    (dict(max_keys=(1 << 30) + 1), EMOE_ESHAPE),
    (dict(scale=float("nan")), EMOE_EINVAL),
    (dict(scale=float("inf")), EMOE_EINVAL),
    (dict(scale=-3e38), EMOE_EINVAL),
    (dict(cap=-1.0), EMOE_EINVAL),
    (dict(cap=float("nan")), EMOE_EINVAL),
    (dict(cap=float("inf")), EMOE_EINVAL),
    (dict(cap=2.0 ** -61), EMOE_EINVAL),
    (dict(dtype=EMOE_F16), EMOE_EINVAL),
    (dict(dtype=EMOE_F32), EMOE_EINVAL),
    (dict(q=None), EMOE_EINVAL),
    (dict(q=P + 8), EMOE_EINVAL),
    (dict(q_stride=2040), EMOE_EINVAL),
    (dict(out=None), EMOE_EINVAL),
    (dict(out_stride=2050), EMOE_EINVAL),
    (dict(lengths=None), EMOE_EINVAL),
    (dict(page_table=None), EMOE_EINVAL),
    (dict(table_stride=-8), EMOE_EINVAL),
])
def test_tree_checks(change, want):
    args = (C.byref(kv()), C.byref(tree(**change)))
    assert status("emoe_paged_tree_attention", *args, P, 1 << 40, None) == want


def test_tree_needs_its_workspace():
    size = _lib.lib().emoe_paged_tree_attention_workspace_bytes
    need = size(C.byref(kv()), 3, 16, 128, 5)
    assert need > 0
    args = (C.byref(kv()), C.byref(tree()))
    assert status("emoe_paged_tree_attention", *args, None, need, None) == EMOE_EINVAL
    assert status("emoe_paged_tree_attention", *args, P, need - 1, None) == EMOE_EINVAL
    assert status("emoe_paged_tree_attention", *args, P + 8, need, None) == EMOE_EINVAL
    assert status("emoe_paged_tree_attention", None, args[1], P, need, None) == EMOE_EINVAL
    assert status("emoe_paged_tree_attention", args[0], None, P, need, None) == EMOE_EINVAL
    for bad in ((-1, 16, 9, 5), (1, 0, 9, 5), (1, 6, 9, 5), (1, 16, -1, 5), (1, 16, 2 ** 31 - 1, 5),
                (1, 1 << 21, 9, 5), (1, 1 << 20, 9, 64), (1, 16, 9, 0), (1, 16, 9, 65)):
        assert size(C.byref(kv()), *bad) == 0
    # No window needs more than none does.
    assert size(C.byref(kv()), 1, 16, 1 << 30, 64) < 1 << 30


@pytest.mark.parametrize("change,want", [
    (dict(trees=0, path=None), EMOE_OK),
    (dict(trees=-1), EMOE_EINVAL),
    (dict(rows=-1), EMOE_EINVAL),
    (dict(max_nodes=0), EMOE_ESHAPE),
    (dict(max_nodes=65, path_stride=65, new_tokens_stride=65), EMOE_ESHAPE),
    (dict(starts=None), EMOE_ESHAPE),
    (dict(tokens=None), EMOE_EINVAL),
    (dict(chosen=None), EMOE_EINVAL),
    (dict(path=None), EMOE_EINVAL),
    (dict(accepted=None), EMOE_EINVAL),
    (dict(lengths=None), EMOE_EINVAL),                   # with new_lengths
    (dict(path_stride=4), EMOE_EINVAL),
    (dict(new_tokens_stride=4), EMOE_EINVAL),
])
def test_accept_checks(change, want):
    assert status("emoe_accept_drafts", C.byref(accept(**change)), None) == want
    assert status("emoe_accept_drafts", None, None) == EMOE_EINVAL


TABLES = [
    (dict(page_table=None), EMOE_EINVAL),
    (dict(n_seqs=-1), EMOE_EINVAL),
    (dict(table_width=-1), EMOE_EINVAL),
    (dict(table_stride=7), EMOE_EINVAL),
    (dict(lengths=None), EMOE_EINVAL),
]


@pytest.mark.parametrize("change,want", TABLES + [
    (dict(trees=0, path=None), EMOE_OK),
    (dict(trees=-1), EMOE_EINVAL),
    (dict(max_nodes=0), EMOE_ESHAPE),
    (dict(max_nodes=65, path_stride=65), EMOE_ESHAPE),
    (dict(path=None), EMOE_EINVAL),
    (dict(accepted=None), EMOE_EINVAL),
    (dict(path_stride=4), EMOE_EINVAL),
])
def test_compact_checks(change, want):
    assert status("emoe_paged_compact", C.byref(kv()), 1, C.byref(compact(**change)), None) == want
    check_layers("emoe_paged_compact", compact())


@pytest.mark.parametrize("change,want", TABLES + [
    (dict(forks=0, parents=None), EMOE_OK),
    (dict(table_width=0, table_stride=0, parents=None), EMOE_OK),
    (dict(forks=-1), EMOE_EINVAL),
    (dict(parents=None), EMOE_EINVAL),
    (dict(new_table=None), EMOE_EINVAL),
    (dict(new_table_stride=7), EMOE_EINVAL),
    (dict(new_table=P), EMOE_EINVAL),                    # the table itself
    (dict(new_table=P + 4 * 23), EMOE_EINVAL),           # its last entry
    (dict(new_table=P - 4 * 23), EMOE_EINVAL),
])
def test_fork_checks(change, want):
    assert status("emoe_paged_fork", C.byref(kv()), 1, C.byref(fork(**change)), None) == want
    check_layers("emoe_paged_fork", fork())


def check_layers(name, args):
    assert status(name, None, 1, C.byref(args), None) == EMOE_EINVAL
    assert status(name, C.byref(kv()), 1, None, None) == EMOE_EINVAL
    assert status(name, C.byref(kv()), 0, C.byref(args), None) == EMOE_EINVAL
    for other in (dict(n_pages=9), dict(dtype=EMOE_F16), dict(page_size=8),
                  dict(slot_stride=1024, page_stride=16 * 1024), dict(head_dim=64)):
        both = (_lib.PagedKVView * 2)(kv(), kv(1, **other))
        assert status(name, both, 2, C.byref(args), None) == EMOE_ESHAPE
    both = (_lib.PagedKVView * 2)(kv(), kv(1, k_pages=None))
    assert status(name, both, 2, C.byref(args), None) == EMOE_EINVAL
    # Keys or values of two layers, or the keys and values of one, in the same place.
    for same in ([kv(), kv()], [kv(), kv(1, v_pages=P)], [kv(v_pages=P), kv(1)], [kv(), kv(1), kv(2), kv(1)]):
        assert status(name, (_lib.PagedKVView * len(same))(*same), len(same), C.byref(args),
                      None) == EMOE_EINVAL


def test_binding_refuses_host_tensors():
    n = torch.zeros(1, dtype=torch.int32)
    for make in (lambda: api.accept_drafts(n, n, n, n[None], n),
                 lambda: api.accept_drafts([0], n, n, n[None], n), lambda: api.paged_compact([], n, n, n, n),
                 lambda: api.paged_fork([], n, n, n, n, n), lambda: api.paged_compact([None], n, n, n, n),
                 lambda: api.paged_compact(None, n, n, n, n), lambda: api.paged_fork(3, n, n, n, n, n),
                 lambda: api.paged_fork(n, n, n, n, n, n)):
        with pytest.raises(_lib.ExactMoEError) as e:
            make()
        assert e.value.status == EMOE_EINVAL


class Other:
    """Something else than a PagedKV, with the same numbers: of a cache that lives as long."""

    def __init__(self, view, index=0):
        self.view, self.address, self.index = view, C.addressof(view), index


class SpecialKV(api.PagedKV):
    pass


def handle(view, kind=api.PagedKV):
    """A PagedKV without tensors behind it, for calls that are refused."""
    made = kind.__new__(kind)
    made.view, made.address, made.index = view, C.addressof(view), 0
    return made


def refused_with(call):
    with pytest.raises(_lib.ExactMoEError) as e:
        call()
    assert e.value.status == EMOE_EINVAL
    return str(e.value)


@pytest.mark.parametrize("other", [Other(kv(1)), None, 3, object(), Other(kv(1), "x"), kv(1)])
def test_caches_are_paged_kvs(other):
    """Whatever stands in a cache's place is refused before an address is taken from it."""
    n, x = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 2, 128, dtype=torch.bfloat16)
    first, special = handle(kv(0)), handle(kv(2), SpecialKV)
    compact = lambda kvs: refused_with(lambda: api.paged_compact(kvs, n[None], n, n[None], n, stream=0))
    fork = lambda kvs: refused_with(lambda: api.paged_fork(kvs, n[None], n, n, None, n[None], stream=0))
    for call in (compact, fork):
        for kvs in ([other], [first, other], (first, special, other), [special, other, first]):
            assert "kvs: need a list of PagedKV" in call(kvs), kvs
        for kvs in ([first], [first, special], (special, first)):
            assert "kvs" not in call(kvs), kvs               # refused for its host tensors
    for call in (lambda c: api.paged_append_axes(c, None, x, x, n, n[None], None, n[None], None, stream=0),
                 lambda c: api.paged_tree_attention(c, x, n[None], n, x, None, 8, 1, stream=0)):
        assert "kv: need a PagedKV" in refused_with(lambda: call(other))
        assert "kv: need" not in refused_with(lambda: call(special))
    with pytest.raises(_lib.ExactMoEError):
        api.paged_tree_attention_workspace_bytes(other, 1, 1, 1, 1)


@pytest.mark.parametrize("trees,max_nodes", [(127, 16), (128, 16), (2000, 1), (40000, 64)])
def test_tree_cuts_long_keys_of_many_outputs(trees, max_nodes):
    """The workspace has room for parts wherever keys may be long, however many trees there are, and
    no more of it than the workers can fill."""
    size = _lib.lib().emoe_paged_tree_attention_workspace_bytes
    view = kv(n_kv_heads=8, slot_stride=1024, head_stride=128, page_stride=16 * 1024)
    short, long = size(C.byref(view), trees, 32, 600, max_nodes), size(C.byref(view), trees, 32, 131072, max_nodes)
    few = size(C.byref(view), 8, 32, 131072, max_nodes)
    if trees > 127:
        assert short == 16
    assert few <= long <= few + 12 * (1 << 14)
