"""Refusals of the operators of a paged cache held in 4 bits: every argument that the header rules out is refused by a status
and a message before anything is launched (so these run without a GPU)."""
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
    """Head-major: 8 heads, pages of 32, 64 features."""
    d = dict(k=A, v=A, k_scale=A, v_scale=A, k_page=8 * 1024, k_head=1024, k_token=32, v_page=8 * 1024, v_head=1024, v_token=32,
             ks_page=512, ks_head=64, ks_group=32, vs_page=512, vs_head=64, vs_group=32, table=A, table_stride=10, len=A, batch=2,
             table_pages=10, n_pages=20, page_size=32, n_kv_heads=8, head_dim=64)
    d.update(kw)
    return cs.cs_pages_fp4(**d)


def append(lib, p=None, **kw):
    d = dict(t=1, k=A, k_row=512, k_head=64, v=A, v_row=512, v_head=64, row0=A, R=4)
    d.update(kw)
    return lib.cs_paged_fp4_append(C.byref(p if p is not None else pages()), *d.values(), None)


def read(lib, p=None, **kw):
    d = dict(t=1, k=A, k_row=512, k_head=64, v=A, v_row=512, v_head=64, row0=A, first=None, R=4)
    d.update(kw)
    return lib.cs_paged_fp4_read(C.byref(p if p is not None else pages()), *d.values(), None)


def attention(lib, p=None, **kw):
    d = dict(t=1, q=A, q_row=2048, q_head=64, H=32, row0=A, R=4, scale=0.125, window=0, max_rows=0, max_len=0, out=A, out_row=2048,
             out_head=64, ws=A, ws_bytes=1 << 40)
    d.update(kw)
    return lib.cs_paged_fp4_attention(C.byref(p if p is not None else pages()), *d.values(), None)


BAD_PAGES = [dict(reserved=(1, 0)), dict(reserved=(0, 1)), dict(batch=-1), dict(n_pages=0), dict(n_kv_heads=0), dict(table_pages=0),
             dict(table=None), dict(len=None), dict(table_stride=9), dict(head_dim=0), dict(head_dim=48), dict(head_dim=72),
             dict(head_dim=288), dict(page_size=16), dict(page_size=48), dict(page_size=0), dict(page_size=65536),
             dict(table_pages=1 << 26, table_stride=1 << 26), dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None),
             dict(k=A + 8), dict(v=A + 2), dict(k_scale=A + 4), dict(v_scale=A + 8), dict(k_page=-16), dict(k_head=8), dict(v_head=-64),
             dict(v_page=1 << 41), dict(k_token=16), dict(v_token=40), dict(k_token=1 << 27), dict(ks_group=16), dict(vs_group=40),
             dict(ks_group=1 << 31), dict(vs_page=-16), dict(ks_head=8), dict(vs_page=1 << 41), dict(batch=1 << 17), dict(n_kv_heads=4097)]


@pytest.mark.parametrize("bad", BAD_PAGES, ids=str)
def test_bad_pages(lib, bad):
    for rc in (append(lib, pages(**bad)), read(lib, pages(**bad)), attention(lib, pages(**bad)),
               lib.cs_paged_fp4_attention_workspace(C.byref(pages(**bad)), 1, 32, 1, 4, 0, 0)):
        assert rc in (-2, -6) and len(lib.cs_last_error()) > 10, (bad, rc)


def test_null_pages(lib):
    assert lib.cs_paged_fp4_append(None, 1, A, 512, 64, A, 512, 64, A, 4, None) == -2
    assert lib.cs_paged_fp4_read(None, 1, A, 512, 64, A, 512, 64, A, A, 4, None) == -2
    assert lib.cs_paged_fp4_attention(None, 1, A, 2048, 64, 32, A, 4, 0.1, 0, 0, 0, A, 2048, 64, A, 1 << 40, None) == -2
    assert lib.cs_paged_fp4_attention_workspace(None, 1, 32, 1, 4, 0, 0) == -2


ROWS = [dict(t=2), dict(t=-1), dict(R=-1), dict(k=None), dict(v=None), dict(k=A + 2), dict(v_row=4), dict(v_head=-8), dict(row0=None, R=5),
        dict(R=1 << 27), dict(k_row=1 << 41)]


@pytest.mark.parametrize("bad", ROWS, ids=str)
def test_append_and_read_refuse(lib, bad):
    assert append(lib, **bad) in (-2, -6) and read(lib, **bad) in (-2, -6)


@pytest.mark.parametrize("bad", [dict(t=2), dict(t=-1), dict(q=None), dict(out=None), dict(q=A + 2), dict(out_row=2044), dict(out_head=-64), dict(H=0),
                                 dict(H=12), dict(H=8192), dict(R=-1), dict(row0=None, R=5), dict(scale=0.0), dict(scale=-1.0),
                                 dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1), dict(max_rows=-1), dict(max_len=-1),
                                 dict(R=1 << 27), dict(R=(1 << 25) + 1)], ids=str)
def test_attention_refuses(lib, bad):
    assert attention(lib, **bad) in (-2, -6)


@pytest.mark.parametrize("t", [0, 1])
def test_attention_refuses_a_small_workspace(lib, t):
    p = pages(table_pages=1 << 16, table_stride=1 << 16)
    need = lib.cs_paged_fp4_attention_workspace(C.byref(p), t, 32, 1, 4, 1, 1 << 20)
    assert need > 0                                        # two streams of a million tokens are split
    for ws, size in ((A, need - 1), (None, need), (A + 4, need), (A, 0)):
        assert attention(lib, p, t=t, max_rows=1, max_len=1 << 20, ws=ws, ws_bytes=size) in (-2, -3)


def test_nothing_to_do_is_no_error(lib):
    assert append(lib, R=0) == 0 and read(lib, R=0) == 0 and attention(lib, R=0) == 0
    assert append(lib, pages(batch=0)) == 0 and read(lib, pages(batch=0)) == 0 and attention(lib, pages(batch=0)) == 0


def test_what_is_written_does_not_overlap_itself(lib):
    """Pages, heads, rows and groups that a call writes lie apart; pools that are only read may be broadcast."""
    for bad in (dict(k_head=0), dict(v_head=0), dict(k_page=0), dict(v_page=16), dict(v_head=16), dict(ks_page=0), dict(vs_head=16)):
        assert append(lib, pages(**bad)) == -2, bad
        # such pools may be read: what is refused here is the missing workspace
        long = pages(table_pages=1 << 16, table_stride=1 << 16, **bad)
        assert attention(lib, long, max_rows=1, max_len=1 << 20, ws=None, ws_bytes=0) == -3, bad
    for bad in (dict(k_row=0), dict(k_head=0), dict(v_row=56), dict(v_head=32)):
        assert read(lib, **bad) == -2, bad
    for bad in (dict(out_row=0), dict(out_head=0), dict(out_head=56)):
        assert attention(lib, **bad) == -2, bad


def test_struct_layout_matches_the_header():
    assert C.sizeof(cs.cs_pages_fp4) == 4 * 8 + 12 * 8 + 3 * 8 + 8 * 4


@pytest.mark.parametrize("t", [0, 1])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("H,KVH", [(32, 8), (28, 4), (8, 1), (16, 16)])
def test_the_workspace_does_not_grow_with_the_table(lib, H, KVH, hd, t):
    """Without hints a call has room for token ranges of streams as long as the table: never half a gigabyte."""
    d = dict(k_page=KVH * 16 * hd, k_head=16 * hd, k_token=hd // 2, v_page=KVH * 16 * hd, v_head=16 * hd, v_token=hd // 2, n_kv_heads=KVH,
             head_dim=hd, ks_page=KVH * hd, ks_head=hd, vs_page=KVH * hd, vs_head=hd)
    for table in (1 << 10, 1 << 13, 1 << 16, 1 << 20):
        for batch in (1, 3, 16, 64, 65, 100, 300):
            p = pages(batch=batch, table_pages=table, table_stride=table, **d)
            for R in (1, 7, 64, 300, 520, 1040, 1488, 2048, 2976, 3968, 5000, 40000):
                for has_row0, rows in ((1, R), (0, R * batch)):
                    need = lib.cs_paged_fp4_attention_workspace(C.byref(p), t, H, has_row0, rows, 0, 0)
                    assert 0 <= need <= 1 << 29, (table, batch, R, has_row0, need)


@pytest.mark.parametrize("t", [0, 1])
@pytest.mark.parametrize("H,KVH,singles,block,longest", [(32, 2, 15, 8192, 8192), (32, 2, 23, 8192, 8192), (64, 8, 31, 4096, 4096), (32, 8, 15, 2048, 2048),
                                                         (16, 1, 400, 0, 1), (32, 2, 100, 0, 2), (32, 8, 15, 8192, 0)])
def test_a_wide_table_does_not_take_the_cut_of_tokens_away(lib, H, KVH, singles, block, longest, t):
    """Streams that bring few rows are cut over their tokens whatever the width of the table and however long the blocks beside them: the
    partial results that there is room for are those over a table just as wide as the contexts."""
    hd, P, R = 128, 64, singles + block
    d = dict(k_page=KVH * P * 64, k_head=P * 64, k_token=64, v_page=KVH * P * 64, v_head=P * 64, v_token=64, n_kv_heads=KVH, head_dim=hd, page_size=P,
             ks_page=KVH * P * 4, ks_head=P * 4, ks_group=P, vs_page=KVH * P * 4, vs_head=P * 4, vs_group=P, batch=singles + (block > 0))
    need = []
    for table in (1 << 15, 1 << 18, 1 << 19, 1 << 20, 1 << 21, 1 << 24):
        p = pages(table_pages=table // P, table_stride=table // P, **d)
        need.append(lib.cs_paged_fp4_attention_workspace(C.byref(p), t, H, 1, R, longest, 20000))
    assert need[0] > 0 and need == need[:1] * len(need), need


def _handle(**kw):
    d = dict(k=torch.zeros((4, 1, 32, 32), dtype=torch.uint8), k_scale=torch.zeros((4, 1, 2, 32), dtype=torch.uint8),
             table=torch.zeros((1, 2), dtype=torch.int32), length=torch.zeros(1, dtype=torch.int32))
    d.update(v=d["k"], v_scale=d["k_scale"])
    d.update(kw)
    return cs.PagesFP4(**{n: d[n] for n in ("k", "v", "k_scale", "v_scale", "table", "length")})


def test_binding_refuses_host_tensors():
    with pytest.raises(TypeError, match="CUDA"):
        _handle()


def test_binding_refuses_pools_of_other_shapes_and_types(monkeypatch):
    monkeypatch.setattr(cs, "_device_of", lambda tensors: 0)          # what is checked behind the devices
    _handle()
    u8 = dict(dtype=torch.uint8)
    for bad in (dict(k=torch.zeros((4, 1, 32, 32))), dict(k=torch.zeros((4, 1, 32, 33), **u8)), dict(v=torch.zeros((4, 1, 32, 64), **u8)),
                dict(k_scale=torch.zeros((4, 1, 2, 16), **u8)), dict(k_scale=torch.zeros((4, 1, 32, 2), **u8)),
                dict(v_scale=torch.zeros((4, 1, 2, 32), dtype=torch.int8)), dict(k=torch.zeros((4, 1, 32, 64), **u8)[..., ::2]),
                dict(k_scale=torch.zeros((4, 1, 32, 2), **u8).transpose(2, 3), v_scale=torch.zeros((4, 1, 32, 2), **u8).transpose(2, 3)),
                dict(table=torch.zeros((1, 2), dtype=torch.int64)), dict(length=torch.zeros(2, dtype=torch.int32)),
                dict(k=torch.zeros((4, 32, 32), **u8))):
        with pytest.raises(TypeError):
            _handle(**bad)


def test_binding_refuses_tensors_that_want_gradients():
    x, y = torch.zeros((2, 4, 64), requires_grad=True), torch.zeros((2, 4, 64))
    for call in (lambda: cs.cs_paged_fp4_append(None, x, y), lambda: cs.cs_paged_fp4_append(None, y, x), lambda: cs.cs_paged_fp4_attention(None, x),
                 lambda: cs.cs_paged_fp4_attention(None, y, out=x), lambda: cs.cs_paged_fp4_read(None, out=(x, y)), lambda: cs.cs_paged_fp4_read(None, out=(y, x))):
        with pytest.raises(RuntimeError, match="no gradients"):
            call()


def test_binding_refuses_a_read_of_unknown_size():
    class P:
        device, k, c = 0, torch.zeros(1), cs.cs_pages_fp4()
    with pytest.raises(TypeError):
        cs.cs_paged_fp4_read(P, out=(torch.zeros((2, 4, 64)), torch.zeros((2, 4, 64), dtype=torch.bfloat16)))
