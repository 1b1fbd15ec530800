"""Calls of the operators for drafted tokens, and of sampling, that the host refuses; nothing is launched, so no GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_2410_23668_b200 import binding as kl, build

OK, BAD, SHAPE = kl.KL_OK, kl.KL_ERR_INVALID_ARG, kl.KL_ERR_UNSUPPORTED_SHAPE
P = 4096   # stands for a device pointer; a refused call never follows it


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return kl.lib()


def cache(**over):
    d = dict(n_kv_heads=2, head_dim=128, page_size=16, n_pages=8, kv_type=kl.KL_KV_E4M3, page_stride=2 * 16 * 128, head_stride=16 * 128, row_stride=128,
             k_d=P, v_d=P, k_exp_d=P, v_exp_d=P, bounds_d=P)
    d.update(over)
    return kl.PagedCacheDesc(**d)


def seqs(**over):
    d = dict(positions_d=P, page_table_d=P, table_stride=4, table_pages=4, n_seqs=3)
    d.update(over)
    return kl.PagedSeqs(**d)


CACHES = [(dict(head_dim=96), SHAPE), (dict(head_dim=32), SHAPE), (dict(page_size=2), SHAPE), (dict(page_size=18), SHAPE), (dict(page_size=2048), SHAPE),
          (dict(n_kv_heads=0), SHAPE), (dict(kv_type=2), BAD), (dict(k_d=None), BAD), (dict(v_d=P + 8), BAD), (dict(k_exp_d=None), BAD), (dict(v_exp_d=P + 4), BAD),
          (dict(row_stride=120), BAD), (dict(head_stride=-128), BAD), (dict(page_stride=7), BAD)]
SEQS = [(dict(positions_d=None), BAD), (dict(page_table_d=None), BAD), (dict(table_pages=0), BAD), (dict(table_stride=3), BAD),
        (dict(table_pages=1 << 28, table_stride=1 << 28), SHAPE)]


def rotate_call(lib, c, s, starts=P, n=5, k=P, v=P, t=kl.KL_BF16, ks=256, vs=256, f=P, q=P, qo=P, qs=1024, qos=1024, nq=8):
    return lib.kl_paged_append_rotated(C.byref(c) if c else None, C.byref(s) if s else None, starts, n, k, v, t, ks, vs, f, None, q, qo, qs, qos, nq, None, None)


def tree_call(lib, c, s, starts=P, n=5, q=P, o=P, t=kl.KL_BF16, qs=1024, os=1024, nq=8, scale=0.0, window=0, sinks=0, mask=None, words=0, ws=P, wb=1 << 30):
    return lib.kl_paged_tree_attention(C.byref(c) if c else None, C.byref(s) if s else None, starts, n, q, o, t, qs, os, nq, scale, window, sinks, None, mask, words,
                                       None, ws, wb, None, None)


@pytest.mark.parametrize("call", [rotate_call, tree_call])
def test_descriptors(lib, call):
    for over, rc in CACHES:
        assert call(lib, cache(**over), seqs()) == rc, over
    for over, rc in SEQS:
        assert call(lib, cache(), seqs(**over)) == rc, over
    assert call(lib, None, seqs()) == BAD and call(lib, cache(), None) == BAD
    assert call(lib, cache(), seqs(n_seqs=0)) == OK and call(lib, cache(), seqs(), n=0) == OK
    assert call(lib, cache(), seqs(), starts=None) == BAD   # five rows, three sequences


def test_append_rotated(lib):
    for over in (dict(k=None), dict(v=None), dict(k=P + 2), dict(t=5), dict(ks=255), dict(ks=128), dict(vs=-256), dict(f=None), dict(f=P + 4), dict(q=None), dict(qo=None),
                 dict(q=P + 8), dict(qs=1020), dict(qos=512)):
        assert rotate_call(lib, cache(), seqs(), **over) == BAD, over
    for over in (dict(nq=7), dict(nq=0), dict(nq=65536)):
        assert rotate_call(lib, cache(), seqs(), **over) == SHAPE, over


def test_tree_attention(lib):
    for over in (dict(q=None), dict(o=None), dict(q=P + 8), dict(t=7), dict(qs=1020), dict(os=512), dict(scale=float("inf")), dict(scale=float("nan")), dict(mask=P),
                 dict(words=2), dict(mask=P, words=1 << 27), dict(ws=None), dict(ws=P + 16), dict(wb=1000)):
        assert tree_call(lib, cache(), seqs(), **over) == BAD, over
    for over in (dict(nq=7), dict(nq=0), dict(nq=65536), dict(t=kl.KL_F32), dict(n=1 << 29), dict(n=1 << 31)):
        assert tree_call(lib, cache(), seqs(), **over) == SHAPE, over
    b = C.c_size_t()
    assert lib.kl_paged_tree_workspace_bytes(C.byref(cache()), 7, C.byref(b)) == SHAPE and lib.kl_paged_tree_workspace_bytes(C.byref(cache()), 8, None) == BAD
    assert lib.kl_paged_tree_workspace_bytes(C.byref(cache()), 8, C.byref(b)) == OK and tree_call(lib, cache(), seqs(), wb=b.value - 1) == BAD


def sample_call(lib, x=P, stride=1000, n=3, vocab=1000, u=P, tokens=P):
    return lib.kl_sample(x, stride, n, vocab, u, None, None, None, None, tokens, None, None, None)


def test_sample(lib):
    for over in (dict(x=None), dict(u=None), dict(tokens=None), dict(vocab=0), dict(stride=999), dict(stride=-1000), dict(stride=1 << 40)):
        assert sample_call(lib, **over) == BAD, over
    for over in (dict(vocab=327681, stride=327681), dict(n=(1 << 24) + 1)):
        assert sample_call(lib, **over) == SHAPE, over
    assert sample_call(lib, n=0, x=None) == OK


def test_sample_binding():
    x, u, t = torch.zeros(2, 8), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(kl.KlError):   # not on a CUDA device
        kl.kl_sample(x, u, t)


def test_numbers_that_are_not_aligned(lib):
    c, s = C.byref(cache()), C.byref(seqs())
    for starts, at in ((P + 2, None), (P, P + 1)):
        assert lib.kl_paged_append_rotated(c, s, starts, 5, P, P, kl.KL_BF16, 256, 256, P, at, None, None, 0, 0, 0, None, None) == BAD
    for starts, at, mask, lse in ((P + 1, None, None, None), (P, P + 2, None, None), (P, None, P + 2, None), (P, None, None, P + 3)):
        assert lib.kl_paged_tree_attention(c, s, starts, 5, P, P, kl.KL_BF16, 1024, 1024, 8, 0.0, 0, 0, at, mask, 1 if mask else 0, lse, P, 1 << 30, None, None) == BAD
    assert sample_call(lib, x=P + 2) == BAD and sample_call(lib, u=P + 1) == BAD and sample_call(lib, tokens=P + 3) == BAD


def test_in_place_with_other_strides(lib):
    assert rotate_call(lib, cache(), seqs(), q=P, qo=P, qs=1024, qos=2048) == BAD
