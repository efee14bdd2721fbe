"""switchsd_kv_map_granted refuses what switchsd_kv_map does, without a GPU."""
import ctypes

import pytest

FAKE = 0x10000  # never dereferenced by host validation


@pytest.mark.parametrize("code,kw", [(-1, dict(lens=None)), (-1, dict(new_lens=None)), (-1, dict(held=None)), (-1, dict(free_count=None)),
                                     (-2, dict(B=0)), (-2, dict(B=8193)), (-2, dict(T=0)), (-2, dict(page=24)), (-2, dict(pages=1 << 28)),
                                     (-2, dict(T=1 << 30, B=4))])
@pytest.mark.parametrize("granted", [None, FAKE])
def test_granted_refuses(code, kw, granted):
    from paper_2609_20186_gb300 import binding as bd
    from paper_2609_20186_gb300 import build
    build.build()
    p = bd.switchsd_kv_map_params()
    for key, v in {**dict(B=2, T=3, page=16, blocks=4, pages=9, lens=FAKE, new_lens=FAKE, block_table=FAKE, held=FAKE, free_list=FAKE, free_count=FAKE,
                          slots=FAKE), **kw}.items():
        setattr(p, key, v)
    lib = bd.load()
    assert lib.switchsd_kv_map_granted(ctypes.byref(p), granted) == code
    assert lib.switchsd_kv_map(ctypes.byref(p)) == code
    assert lib.switchsd_kv_map_granted(None, granted) == -1
