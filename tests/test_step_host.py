"""The argument checks of a step's calls and of the 8-bit cache's, on the host alone, and
the mirrors of their C structures."""
import ctypes
import subprocess

import pytest

from conftest import ROOT
from paper_2607_13500_amd import _lib

G = 1 << 20          # an address that is never followed


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def pool(**bad):
    p = dict(pages=9, ring=G, state=G, state_out=G)
    p.update(bad)
    return _lib.Pool(**p)


def pages(lib, pool_=None, **bad):
    a = dict(seqs=3, change=G, kv_len=G, kv_out=G, table=G, table_width=4, table_stride=4, page_size=16, pool=ctypes.byref(pool_ or pool()), q_start=G,
             rows=5, slots=G, pos=G, short_of=G, stream=None)
    a.update(bad)
    return lib.tr_update_pages(*a.values())


def test_update_pages_refusals(lib):
    for bad in (dict(seqs=-1), dict(rows=-1), dict(rows=1 << 31), dict(page_size=0), dict(table_width=-1), dict(table_stride=3), dict(table_stride=0),
                dict(q_start=None), dict(short_of=None), dict(change=None), dict(kv_len=None), dict(kv_out=None), dict(table=None), dict(kv_out=G + 4),
                dict(kv_out=G - 8), dict(change=G + 1024, kv_out=G + 1024), dict(change=G + 1024, kv_out=G + 1028), dict(pool=None)):
        assert pages(lib, **bad) == _lib.TR_EINVAL, bad
        assert lib.tr_last_error()
    for bad in (dict(pages=0), dict(ring=None), dict(state=None), dict(state_out=None), dict(state_out=G + 4)):
        assert pages(lib, pool(**bad)) == _lib.TR_EINVAL, bad
    for bad in (dict(change=G + 2), dict(pos=G + 1), dict(slots=G + 4), dict(table=G + 2)):
        assert pages(lib, **bad) == _lib.TR_EUNSUPPORTED, bad


def verify(lib, **bad):
    a = dict(T=8, vocab=100, dtype=_lib.TR_FP32, target=G, ld_target=100, draft=G, ld_draft=100, ids=G, seqs=2, q_start=G, accept=G, draw=G, width=4,
             tokens=G, accepted=G, change=G, scratch=G, stream=None)
    a.update(bad)
    return lib.tr_verify_drafts(*a.values())


def test_verify_drafts_refusals(lib):
    for bad in (dict(T=-1), dict(T=1 << 31), dict(seqs=-1), dict(seqs=1 << 20), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(width=0), dict(dtype=7),
                dict(q_start=None), dict(draw=None), dict(tokens=None), dict(accepted=None), dict(change=None), dict(scratch=None), dict(target=None),
                dict(ids=None), dict(accept=None), dict(ld_target=99), dict(ld_draft=99)):
        assert verify(lib, **bad) == _lib.TR_EINVAL, bad
        assert lib.tr_last_error()
    for bad in (dict(target=G + 2), dict(draft=G + 1), dict(ids=G + 2), dict(scratch=G + 8), dict(dtype=_lib.TR_BF16, target=G + 1)):
        assert verify(lib, **bad) == _lib.TR_EUNSUPPORTED, bad
    assert verify(lib, seqs=0) == _lib.TR_OK                     # nothing to do
    assert lib.tr_verify_scratch(0) == 0 and lib.tr_verify_scratch(3) == 3 * lib.tr_verify_scratch(1) > 0


def test_calls_on_the_8_bit_cache_need_a_context(lib):
    h = _lib.Heads(G, 64, 64)
    c, s = _lib.Cache8(), _lib.StepArgs()
    assert lib.tr_append8(None, 1, h, h, h, None, None, None, 0, h, ctypes.byref(c), ctypes.byref(s), None) == _lib.TR_EINVAL
    assert lib.tr_attend8(None, 1, h, ctypes.byref(c), ctypes.byref(s), 1.0, 1, 0, h, None, None) == _lib.TR_EINVAL


def test_structures_are_those_of_the_header(tmp_path):
    """Sizes and offsets of the mirrors, as a C compiler sees the header."""
    lines, want = [], []
    for name, mirror in (("tr_cache8", _lib.Cache8), ("tr_pool", _lib.Pool), ("tr_cache", _lib.Cache), ("tr_step", _lib.StepArgs)):
        lines.append('printf("%%zu ", sizeof(%s));' % name)
        want.append(ctypes.sizeof(mirror))
        for field, _ in mirror._fields_:
            lines.append('printf("%%zu ", offsetof(%s, %s));' % (name, field))
            want.append(getattr(mirror, field).offset)
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "tr.h"\nint main(void) { %s return 0; }\n' % " ".join(lines))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", ROOT + "/include", str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    assert [int(x) for x in out.split()] == want
