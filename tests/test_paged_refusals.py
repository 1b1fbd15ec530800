"""Calls of the paged cache operators that the host refuses; nothing is launched, so no GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_2410_23668_b200 import binding as kl, build, inputs as gen

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
          (dict(n_kv_heads=0), SHAPE), (dict(kv_type=2), BAD)]
ROW_CACHES = [(dict(k_d=None), BAD), (dict(v_d=P + 8), BAD), (dict(k_exp_d=None), BAD), (dict(v_exp_d=P + 4), BAD), (dict(row_stride=120), BAD),
              (dict(head_stride=-128), BAD), (dict(page_stride=7), BAD)]
SEQS = [(dict(positions_d=None), BAD), (dict(page_table_d=None), BAD), (dict(table_pages=0), BAD), (dict(table_stride=3), BAD),
        (dict(table_pages=1 << 28, table_stride=1 << 28), SHAPE)]


def rows_call(lib, fn, c, s, starts=P, n=5, k=P, v=P, t=kl.KL_BF16, ks=256, vs=256):
    return getattr(lib, fn)(C.byref(c) if c else None, C.byref(s) if s else None, starts, n, k, v, t, ks, vs, None, None)


def select_call(lib, c, s, q=P, t=kl.KL_BF16, qs=1024, nq=8, first=1, last=1, k=4, sel=P, ws=P, wb=1 << 20):
    return lib.kl_paged_select(C.byref(c) if c else None, C.byref(s) if s else None, q, t, qs, nq, first, last, k, sel, ws, wb, None, None)


def attn_call(lib, c, s, q=P, o=P, t=kl.KL_BF16, qs=1024, os=1024, nq=8, scale=0.0, window=0, sel=None, k=0, ws=P, wb=1 << 30):
    return lib.kl_paged_attention(C.byref(c) if c else None, C.byref(s) if s else None, q, o, t, qs, os, nq, scale, window, sel, k, None, ws, wb, None, None)


@pytest.mark.parametrize("fn", ["kl_paged_append", "kl_paged_read"])
def test_rows_in_and_out(lib, fn):
    for over, rc in CACHES + ROW_CACHES:
        assert rows_call(lib, fn, cache(**over), seqs()) == rc, over
    for over, rc in SEQS:
        assert rows_call(lib, fn, cache(), seqs(**over)) == rc, over
    assert rows_call(lib, fn, None, seqs()) == BAD and rows_call(lib, fn, cache(), None) == BAD
    for over in (dict(k=None), dict(v=None), dict(k=P + 2), dict(t=5), dict(ks=255), dict(ks=128), dict(vs=-256), dict(starts=None)):
        assert rows_call(lib, fn, cache(), seqs(), **over) == BAD, over
    assert rows_call(lib, fn, cache(), seqs(), ks=260) == BAD            # rows would not start on 16 bytes
    assert rows_call(lib, fn, cache(), seqs(n_seqs=0), n=0) == OK        # nothing to do
    assert rows_call(lib, fn, cache(), seqs(), n=0) == OK


def test_select(lib):
    for over, rc in CACHES + [(dict(bounds_d=None), BAD), (dict(bounds_d=P + 2), BAD)]:
        assert select_call(lib, cache(**over), seqs()) == rc, over
    for over, rc in SEQS:
        assert select_call(lib, cache(), seqs(**over)) == rc, over
    for over in (dict(q=None), dict(q=P + 4), dict(t=2), dict(qs=1000), dict(k=0), dict(k=1), dict(first=3, last=2), dict(first=0xffffffff, last=1),
                 dict(sel=None), dict(ws=None), dict(ws=P + 16), dict(wb=16)):
        assert select_call(lib, cache(), seqs(), **over) == BAD, over
    for over in (dict(nq=0), dict(nq=7)):
        assert select_call(lib, cache(), seqs(), **over) == SHAPE, over
    assert select_call(lib, cache(), seqs(n_seqs=0)) == OK


def test_attention(lib):
    for over, rc in CACHES + ROW_CACHES:
        assert attn_call(lib, cache(**over), seqs()) == rc, over
    for over, rc in SEQS:
        assert attn_call(lib, cache(), seqs(**over)) == rc, over
    for over in (dict(q=None), dict(o=None), dict(o=P + 4), dict(t=-1), dict(qs=512), dict(os=1016), dict(sel=P), dict(k=3), dict(ws=None), dict(ws=P + 128),
                 dict(scale=float("inf")), dict(scale=float("nan"))):
        assert attn_call(lib, cache(), seqs(), **over) == BAD, over
    for over in (dict(nq=0), dict(nq=7)):
        assert attn_call(lib, cache(), seqs(), **over) == SHAPE, over
    assert attn_call(lib, cache(), seqs(n_seqs=0)) == OK


def test_workspace(lib):
    b = C.c_size_t()
    assert lib.kl_paged_workspace_bytes(C.byref(cache()), 8, 3, 4, None) == BAD
    assert lib.kl_paged_workspace_bytes(None, 8, 3, 4, C.byref(b)) == BAD
    assert lib.kl_paged_workspace_bytes(C.byref(cache()), 7, 3, 4, C.byref(b)) == SHAPE
    assert lib.kl_paged_workspace_bytes(C.byref(cache()), 8, 3, 4, C.byref(b)) == OK and b.value % 256 == 0 and b.value >= 3 * 2 * 4 * 4


def test_binding_checks():
    k = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    kl.PagedCache(k, k.clone())
    e = torch.zeros(4, 2, 16, dtype=torch.uint8)
    for args in ((k, k.transpose(1, 2)), (k.float(), k.float()), (k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn)),
                 (k.view(torch.uint8)[..., :128], k.view(torch.uint8)[..., :128], e, e[:, :1]), (None, None)):
        with pytest.raises(kl.KlError):
            kl.PagedCache(*args)
    c = kl.PagedCache(k, k.clone())
    q = torch.zeros(1, 8, 128)
    with pytest.raises(kl.KlError):   # tensors of the host: the library launches on the current device
        kl.kl_paged_attention(c, q, q, torch.zeros(1, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(9, dtype=torch.uint8))


def test_step_refuses_tensors_of_another_device(monkeypatch):
    """The step's buffers, the caches of its layers and the model lie on the current device, or the library is not called."""
    class Library:
        def kl_decode_step_paged(self, *args):
            raise AssertionError("the library was called")

        def kl_status_string(self, code):
            return b""

    shape = gen.TINY
    monkeypatch.setattr(kl, "lib", Library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    class Here:   # what the binding asks of a tensor of device 0
        def __init__(self, t):
            self.t = t

        def get_device(self):
            return 0

        def __getattr__(self, name):
            return getattr(self.t, name)

    k = torch.zeros(4, shape.n_kv_heads, 16, shape.head_dim, dtype=torch.bfloat16)
    host, there = kl.PagedCache(k, k.clone()), kl.PagedCache(k, k.clone())
    there._index = 0
    i32 = lambda *size: torch.zeros(size, dtype=torch.int32)
    args = dict(tok=i32(2), pos=i32(2), table=i32(2, 3), logits=torch.zeros(2, shape.vocab), ws=torch.zeros(256, dtype=torch.uint8))

    def step(arena=0, caches=None, **host_ones):
        dec = object.__new__(kl.Decoder)
        dec.shape, dec.handle, dec.weight_arena = shape, None, Here(k) if arena == 0 else k
        a = {n: host_ones.get(n, Here(t)) for n, t in args.items()}
        dec.kl_decode_step_paged(a["tok"], a["pos"], caches or [there] * shape.n_layers, a["table"], a["logits"], a["ws"])

    with pytest.raises(AssertionError):   # everything where it should be
        step()
    for over in ([dict(arena=-1), dict(caches=[there] * (shape.n_layers - 1) + [host])] + [{n: t} for n, t in args.items()]):
        with pytest.raises(kl.KlError) as e:
            step(**over)
        assert e.value.code == BAD, over


def test_sizes_beyond_any_workspace(lib):
    """Products of sizes that leave 64 bits are refused, not cut off to something small."""
    b = C.c_size_t()
    many = cache(n_kv_heads=65535, page_size=4)
    assert lib.kl_paged_workspace_bytes(C.byref(many), 65535, 65536, 1 << 29, C.byref(b)) == SHAPE
    assert lib.kl_paged_workspace_bytes(C.byref(cache()), 8, 1 << 31, 1 << 31, C.byref(b)) == SHAPE
    assert lib.kl_paged_workspace_bytes(C.byref(cache()), 8, 65535, 1 << 27, C.byref(b)) == OK and b.value == 65535 * 2 * (1 << 27) * 8
    s = seqs(n_seqs=65535, table_pages=(1 << 29) - 1, table_stride=(1 << 29) - 1)
    assert select_call(lib, many, s, nq=65535, qs=65535 * 128, wb=(1 << 64) - 1) == SHAPE
    assert select_call(lib, cache(page_size=4), s, wb=1 << 40) == BAD
