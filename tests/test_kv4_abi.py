"""Refusals of the 4-bit cache's and the beam selection's entry points, and their sizes (no GPU needed): nothing is
launched and no pointer below is followed."""
import ctypes

import pytest

from paper_2607_20357_gb300 import svl

INVALID, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 7
P = 1 << 20  # an aligned address that nothing reads


def code(fn, *args):
    with pytest.raises(svl.SvlError) as e:
        fn(*args, stream=0)
    return e.value.code


def D(slots=2, kv=4, dh=128, length=100):
    return svl.Kv4Desc(slots, kv, dh, length)


BAD_DESC = [(D(0), INVALID), (D(kv=0), INVALID), (D(length=0), INVALID), (D(dh=-64), INVALID), (D(dh=96), UNSUPPORTED),
            (D(dh=256), UNSUPPORTED), (D(slots=65536), UNSUPPORTED)]


def test_cache_size(svl_lib):
    assert svl.svl_kv4_cache_size(D()) == 2 * 4 * 4 * 4608
    assert svl.svl_kv4_cache_size(D(1, 1, 64, 32)) == 2304
    assert svl.svl_kv4_cache_size(D(1, 1, 64, 33)) == 4608
    assert svl.svl_kv4_cache_size(D(1, 32, 128, 2 ** 31 - 1)) == 32 * 2 ** 26 * 4608
    for d, _ in BAD_DESC:
        assert svl.svl_kv4_cache_size(d) == 0
    assert svl.svl_kv4_cache_size(None) == 0


@pytest.mark.parametrize("desc,want", BAD_DESC + [(None, INVALID)])
def test_bad_descriptions(svl_lib, desc, want):
    assert code(svl.svl_kv4_write, desc, P, P, 512, P, 512, 2, None, P, None) == want
    assert code(svl.svl_kv4_read, desc, P, 2, None, P, P, 512, P, 512) == want
    assert code(svl.svl_kv4_attention, desc, P, 28, 1, P, 3584, P, 0, 0, 1.0, P, 3584, P, 1 << 30) == want
    assert code(svl.svl_kv4_reorder, desc, P, 1, 2, P, None, P, None) == want


def test_rows(svl_lib):
    w = svl.svl_kv4_write
    assert code(w, D(), None, P, 512, P, 512, 2, None, P, None) == INVALID
    assert code(w, D(), P + 8, P, 512, P, 512, 2, None, P, None) == INVALID
    assert code(w, D(), P, None, 512, P, 512, 2, None, P, None) == INVALID
    assert code(w, D(), P, P + 2, 512, P, 512, 2, None, P, None) == INVALID
    assert code(w, D(), P, P, 511, P, 512, 2, None, P, None) == INVALID
    assert code(w, D(), P, P, 512, P, 504, 2, None, P, None) == INVALID
    assert code(w, D(), P, P, 516, P, 512, 2, None, P, None) == INVALID
    assert code(w, D(), P, P, 512, P, 512, -1, P, P, None) == INVALID
    assert code(w, D(), P, P, 512, P, 512, 2 ** 31, P, P, None) == INVALID
    assert code(w, D(), P, P, 512, P, 512, 3, None, P, None) == SHAPE     # one row per slot
    r = svl.svl_kv4_read
    assert code(r, D(), P, 2, None, P, None, 512, P, 512) == INVALID
    assert code(r, D(), P, 2, None, P, P, 512, P, 8) == INVALID
    assert code(r, D(), P, 1, None, P, P, 512, P, 512) == SHAPE
    # no rows: nothing to do, and nothing is launched
    before = svl.svl_launch_count()
    w(D(), P, P, 512, P, 512, 0, P, P, None, stream=0)
    r(D(), P, 0, P, P, P, 512, P, 512, stream=0)
    assert svl.svl_launch_count() == before


def test_attention(svl_lib):
    def call(desc=None, cache=P, heads=28, rows=1, q=P, ld_q=3584, start=P, window=0, sinks=0, out=P, ld_out=3584, ws=P,
             size=1 << 30):
        return code(svl.svl_kv4_attention, desc or D(), cache, heads, rows, q, ld_q, start, window, sinks, 1.0, out,
                    ld_out, ws, size)
    assert call(cache=None) == INVALID
    assert call(cache=P + 8) == INVALID
    assert call(heads=0) == INVALID
    assert call(heads=27) == INVALID
    assert call(rows=0) == INVALID
    assert call(rows=17) == UNSUPPORTED
    assert call(q=None) == INVALID
    assert call(q=P + 2) == INVALID
    assert call(ld_q=3583) == INVALID
    assert call(ld_q=3588) == INVALID
    assert call(start=None) == INVALID
    assert call(window=-1) == INVALID
    assert call(sinks=-1) == INVALID
    assert call(out=None) == INVALID
    assert call(out=P + 8) == INVALID
    assert call(ld_out=3576) == INVALID
    assert call(ws=None) == WORKSPACE
    assert call(ws=P + 16) == WORKSPACE
    size = svl.svl_kv4_attention_workspace_size
    assert size(D(), 28, 1) >= 256
    for bad in ((D(dh=32), 28, 1), (D(), 27, 1), (D(), 0, 1), (D(), 28, 0), (D(), 28, 17)):
        assert size(*bad) == 0


def test_beam(svl_lib):
    def call(S=2, W=4, V=100, K=8, x=P, ld=100, c=P, fin=None, eos=2, outs=(P, P, P, P), ws=P, size=1 << 30):
        return code(svl.svl_beam_select, S, W, V, K, x, ld, c, fin, eos, *outs, ws, size)
    assert call(S=0) == INVALID
    assert call(W=0) == INVALID
    assert call(W=17) == UNSUPPORTED
    assert call(V=0) == INVALID
    assert call(K=0) == INVALID
    assert call(K=33) == UNSUPPORTED
    assert call(V=7, ld=7) == SHAPE           # more than there are ids
    assert call(x=None) == INVALID
    assert call(ld=99) == INVALID
    assert call(c=None) == INVALID
    assert call(eos=100) == INVALID
    for i in range(3):
        outs = [P, P, P, P]
        outs[i] = None
        assert call(outs=outs) == INVALID
    assert call(ws=None) == WORKSPACE
    assert call(ws=P + 8) == WORKSPACE
    assert call(size=16) == WORKSPACE
    size = svl.svl_beam_select_workspace_size
    assert size(2, 4, 100, 8) > 0
    for bad in ((0, 4, 100, 8), (2, 17, 100, 8), (2, 4, 7, 8), (2, 4, 100, 33), (2, 4, 100, 0)):
        assert size(*bad) == 0


def test_reorder(svl_lib):
    r = svl.svl_kv4_reorder
    assert code(r, D(), None, 1, 2, P, None, P, None) == INVALID
    assert code(r, D(), P, 0, 2, P, None, P, None) == INVALID
    assert code(r, D(), P, 1, 0, P, None, P, None) == INVALID
    assert code(r, D(), P, 1, 2, None, None, P, None) == INVALID
    assert code(r, D(), P, 1, 2, P, None, None, None) == INVALID
    assert code(r, D(slots=3), P, 1, 2, P, None, P, None) == SHAPE
    assert code(r, D(slots=34), P, 1, 17, P, None, P, None) == UNSUPPORTED


def test_description_is_four_integers():
    assert ctypes.sizeof(svl.Kv4Desc) == 16
