"""Refusals of the paged-cache operators: every argument that the header rules out is refused by a status and a message
before anything is launched (so these run without a GPU)."""
import ctypes as C
import os

import pytest
import torch

from paper_2502_08923_amd import binding as cs

A = 1 << 20                       # an address that is aligned and never touched


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cs.LIB_PATH):
        from paper_2502_08923_amd.build import build_lib
        build_lib()
    return cs.load_library()


def pages(**kw):
    d = dict(k=A, v=A, k_page=8 * 16 * 64, k_head=16 * 64, k_token=64, v_page=8 * 16 * 64, v_head=16 * 64, v_token=64, table=A,
             table_stride=10, len=A, batch=2, table_pages=10, n_pages=20, page_size=16, n_kv_heads=8, head_dim=64,
             dtype=cs.CS_BF16, reserved=0)
    d.update(kw)
    return cs.cs_pages(**d)


BAD_PAGES = [dict(dtype=2), dict(dtype=-1), dict(reserved=1), dict(batch=-1), dict(n_pages=0), dict(n_kv_heads=0), dict(table_pages=0),
             dict(table=None), dict(len=None), dict(table_stride=9), dict(head_dim=0), dict(head_dim=60), dict(head_dim=264),
             dict(page_size=8), dict(page_size=48), dict(page_size=0), dict(page_size=65536), dict(table_pages=1 << 27, table_stride=1 << 27),
             dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 2), dict(k_page=-8), dict(k_head=4), dict(v_head=-64), dict(v_page=1 << 41),
             dict(k_token=56), dict(v_token=68), dict(k_token=1 << 30), dict(batch=1 << 17), dict(n_kv_heads=4097)]


def norm_rope(lib, **kw):
    d = dict(ti=1, to=1, q=A, q_row=2048, q_head=64, k=A, k_row=2048, k_head=64, R=4, H=32, KVH=8, hd=64, qg=A, kg=A, eps=1e-6, pos=A,
             f=A, rot=64, qo=A, qo_row=2048, qo_head=64, ko=A, ko_row=2048, ko_head=64)
    d.update(kw)
    return lib.cs_op_qk_norm_rope(*d.values(), None)


def append(lib, p=None, **kw):
    d = dict(t=1, k=A, k_row=512, k_head=64, v=A, v_row=512, v_head=64, row0=A, R=4, f=A, rot=64)
    d.update(kw)
    return lib.cs_paged_append(C.byref(p if p is not None else pages()), *d.values(), None)


def attention(lib, p=None, **kw):
    d = dict(q=A, q_row=2048, q_head=64, H=32, row0=A, R=4, scale=0.125, window=0, max_rows=0, max_len=0, out=A, out_row=2048, out_head=64,
             ws=A, ws_bytes=1 << 40)
    d.update(kw)
    return lib.cs_paged_attention(C.byref(p if p is not None else pages()), *d.values(), None)


@pytest.mark.parametrize("bad", BAD_PAGES, ids=str)
def test_bad_pages(lib, bad):
    for rc in (append(lib, pages(**bad)), attention(lib, pages(**bad)),
               lib.cs_paged_attention_workspace(C.byref(pages(**bad)), 32, 1, 4, 0, 0)):
        assert rc in (-2, -6) and len(lib.cs_last_error()) > 10, (bad, rc)


def test_null_pages(lib):
    assert lib.cs_paged_append(None, 1, A, 512, 64, A, 512, 64, A, 4, A, 64, None) == -2
    assert lib.cs_paged_attention(None, A, 2048, 64, 32, A, 4, 0.1, 0, 0, 0, A, 2048, 64, A, 1 << 40, None) == -2
    assert lib.cs_paged_attention_workspace(None, 32, 1, 4, 0, 0) == -2


@pytest.mark.parametrize("bad", [dict(ti=1, to=0), dict(ti=2), dict(to=5), dict(R=-1), dict(H=0), dict(KVH=-1), dict(hd=60), dict(hd=512),
                                 dict(rot=128), dict(rot=-8), dict(rot=12), dict(f=None), dict(pos=None), dict(eps=-1.0),
                                 dict(eps=float("nan")), dict(eps=float("inf")), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None),
                                 dict(q=A + 4), dict(ko=A + 8), dict(q_row=2044), dict(k_head=-64), dict(qo_head=4), dict(qg=A + 4),
                                 dict(kg=A + 8), dict(R=1 << 27), dict(q_row=1 << 41)], ids=str)
def test_norm_rope_refuses(lib, bad):
    assert norm_rope(lib, **bad) in (-2, -6)


@pytest.mark.parametrize("bad", [dict(t=2), dict(t=-1), dict(R=-1), dict(k=None), dict(v=None), dict(k=A + 2), dict(v_row=4), dict(v_head=-8),
                                 dict(rot=72), dict(rot=4), dict(f=None), dict(row0=None, R=5), dict(R=1 << 27)], ids=str)
def test_append_refuses(lib, bad):
    assert append(lib, **bad) in (-2, -6)


def test_append_of_16_bit_rows_into_a_float32_cache(lib):
    assert append(lib, pages(dtype=0), t=1) == -2


@pytest.mark.parametrize("bad", [dict(q=None), dict(out=None), dict(q=A + 2), dict(out_row=2044), dict(out_head=-64), dict(H=0), dict(H=12),
                                 dict(H=8192), dict(R=-1), dict(row0=None, R=5), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(window=-1), dict(max_rows=-1), dict(max_len=-1), dict(R=1 << 27), dict(R=(1 << 25) + 1)], ids=str)
def test_attention_refuses(lib, bad):
    assert attention(lib, **bad) in (-2, -6)


def test_attention_refuses_a_small_workspace(lib):
    p = pages(table_pages=1 << 16, table_stride=1 << 16)
    need = lib.cs_paged_attention_workspace(C.byref(p), 32, 1, 4, 1, 1 << 20)
    assert need > 0                                        # two streams of a million tokens are split
    for ws, size in ((A, need - 1), (None, need), (A + 4, need), (A, 0)):
        assert attention(lib, p, max_rows=1, max_len=1 << 20, ws=ws, ws_bytes=size) in (-2, -3)


def test_nothing_to_do_is_no_error(lib):
    assert append(lib, R=0) == 0 and attention(lib, R=0) == 0 and norm_rope(lib, R=0) == 0
    assert append(lib, pages(batch=0)) == 0 and attention(lib, pages(batch=0)) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros((2, 4, 64))
    with pytest.raises(TypeError):
        cs.cs_op_qk_norm_rope(x)
    with pytest.raises(TypeError):
        cs.Pages(torch.zeros((4, 1, 16, 64)), torch.zeros((4, 1, 16, 64)), torch.zeros((1, 2), dtype=torch.int32),
                 torch.zeros(1, dtype=torch.int32))


def test_struct_layout_matches_the_header():
    assert C.sizeof(cs.cs_pages) == 2 * 8 + 6 * 8 + 3 * 8 + 8 * 4


@pytest.mark.parametrize("dtype", [cs.CS_BF16, cs.CS_F32])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("H,KVH", [(32, 8), (28, 4), (8, 1), (16, 16)])
def test_the_workspace_does_not_grow_with_the_table(lib, H, KVH, hd, dtype):
    """Without hints a call has room for token ranges of streams as long as the table.  A partial result of a workgroup is at most
    256 rows of 128 (or 128 of 256) float32 features with two statistics, 133120 bytes, and there are at most those of
    the tiles (less than two rounds of the chip, where ranges are cut at all) and of eight more rounds: 10 x 256 (bfloat16; 10 x 512 of half
    the rows in float32) and less than one for each KV head of a round; the kernel of few rows has at most 48 rows."""
    few, many = 48 * (min(hd, 128) * 4 + 8) * 2, 133120
    most = (10 * 256 + KVH) * (few + many) + (1 << 20)
    d = dict(k_page=KVH * 16 * hd, k_head=16 * hd, k_token=hd, v_page=KVH * 16 * hd, v_head=16 * hd, v_token=hd, n_kv_heads=KVH,
             head_dim=hd, dtype=dtype)
    for table in (1 << 10, 1 << 13, 1 << 16, 1 << 20):
        for batch in (1, 3, 16, 64, 65, 100, 300):
            p = pages(batch=batch, table_pages=table, table_stride=table, **d)
            for R in (1, 7, 64, 300, 520, 1040, 1488, 2048, 2976, 3968, 5000, 40000):
                for has_row0, rows in ((1, R), (0, R * batch)):
                    need = lib.cs_paged_attention_workspace(C.byref(p), H, has_row0, rows, 0, 0)
                    assert 0 <= need <= most, (table, batch, R, has_row0, need)


def test_binding_refuses_tensors_that_want_gradients():
    """Refused before the devices are looked at; without autograd the host tensors are what is refused."""
    x = torch.zeros((2, 4, 64), requires_grad=True)
    y, gain = torch.zeros((2, 4, 64)), torch.ones(64, requires_grad=True)
    pool = torch.zeros((4, 1, 16, 64))
    calls = [lambda: cs.cs_op_qk_norm_rope(x), lambda: cs.cs_op_qk_norm_rope(y, x), lambda: cs.cs_op_qk_norm_rope(y, q_gain=gain),
             lambda: cs.cs_op_qk_norm_rope(y, y, k_gain=gain), lambda: cs.cs_paged_append(None, x, y), lambda: cs.cs_paged_append(None, y, x),
             lambda: cs.cs_paged_attention(None, x),
             lambda: cs.Pages(pool.clone().requires_grad_(), pool, torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))]
    for call in calls:
        with pytest.raises(RuntimeError, match="no gradients"):
            call()
    with torch.no_grad(), pytest.raises(TypeError, match="CUDA"):
        cs.cs_op_qk_norm_rope(x)


def test_what_is_written_does_not_overlap_itself(lib):
    """Rows, heads and pages that a call writes lie apart; a stride that is never taken may be 0, and so may one of an input."""
    for bad in (dict(qo_row=0), dict(qo_head=0), dict(qo_row=56), dict(ko_row=0), dict(ko_head=32)):
        assert norm_rope(lib, **bad) == -2, bad
    for bad in (dict(out_row=0), dict(out_head=0), dict(out_head=56)):
        assert attention(lib, **bad) == -2, bad
    for bad in (dict(k_head=0), dict(v_head=0), dict(k_page=0), dict(v_page=56), dict(v_head=32)):
        assert append(lib, pages(**bad)) == -2, bad
        # such pools may be read: what is refused here is the missing workspace
        long = pages(table_pages=1 << 16, table_stride=1 << 16, **bad)
        assert attention(lib, long, max_rows=1, max_len=1 << 20, ws=None, ws_bytes=0) == -3, bad


@pytest.mark.parametrize("hd,short,long", [(64, 300, 600), (128, 180, 450), (256, 120, 400)])
def test_float32_contexts_are_cut_where_it_pays(lib, hd, short, long):
    """The merge of token ranges costs a time, not a number of tokens: the more features a token has, the shorter are the contexts that
    are cut.  A call that cannot have ranges asks for no workspace."""
    p = pages(dtype=cs.CS_F32, k_page=16 * hd, k_head=16 * hd, k_token=hd, v_page=16 * hd, v_head=16 * hd, v_token=hd, n_kv_heads=1,
              head_dim=hd, table_pages=1 << 10, table_stride=1 << 10)
    assert lib.cs_paged_attention_workspace(C.byref(p), 4, 0, 2, 1, short) == 0
    assert lib.cs_paged_attention_workspace(C.byref(p), 4, 0, 2, 1, long) > 0
