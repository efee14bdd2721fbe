"""Host-side validation of the entry points of include/switchsd_target.h, without a GPU: the documented codes come back
before any CUDA call is made."""
import ctypes

import pytest

FAKE = 0x10000  # a 16-byte-aligned non-NULL address; never dereferenced by host validation
ARG, SHAPE = -1, -2


@pytest.fixture(scope="module")
def bd():
    from paper_2609_20186_gb300 import build, binding
    build.build()
    binding.load()
    return binding


def _call(bd, name, struct, base, **kw):
    p = getattr(bd, struct)()
    for key, v in {**base, **kw}.items():
        if isinstance(v, tuple):
            v = (ctypes.c_int64 * 3)(*v)
        setattr(p, key, v)
    return getattr(bd.load(), name)(ctypes.byref(p))


MAP = dict(B=2, T=3, page=16, blocks=4, pages=9, lens=FAKE, new_lens=FAKE, block_table=FAKE, held=FAKE, free_list=FAKE, free_count=FAKE, slots=FAKE)
APPEND = dict(B=2, T=3, Hkv=2, D=64, page=16, pages=9, dtype=0, k=FAKE, v=FAKE, k_stride=(384, 128, 64), v_stride=(384, 128, 64), slots=FAKE, cache=FAKE)
READ = dict(B=2, T=3, Hkv=2, D=64, page=16, pages=9, cache=FAKE, slots=FAKE, out_k=FAKE, out_v=FAKE)
ATTN = dict(B=2, T=3, Hq=4, Hkv=2, D=64, page=16, pages=9, blocks=4, dtype=0, q=FAKE, q_stride=(768, 256, 64), cache=FAKE, block_table=FAKE, lens=FAKE,
            new_lens=FAKE, scale=0.1, out=FAKE, workspace=FAKE, workspace_bytes=1 << 40)
LOGITS = dict(B=2, T=3, V=100, cap=8, dtype=0, logits=FAKE, stride_b=300, stride_t=100, ctx_tokens=FAKE, ctx_lens=FAKE, draft=FAKE, draft_stride=2, argmax=FAKE,
              workspace=FAKE, workspace_bytes=1 << 40)


@pytest.mark.parametrize("code,kw", [(ARG, dict(lens=None)), (ARG, dict(new_lens=None)), (ARG, dict(block_table=None)), (ARG, dict(held=None)),
                                     (ARG, dict(free_list=None)), (ARG, dict(free_count=None)), (SHAPE, dict(B=0)), (SHAPE, dict(B=8193)), (SHAPE, dict(T=0)),
                                     (SHAPE, dict(page=8)), (SHAPE, dict(page=24)), (SHAPE, dict(page=512)), (SHAPE, dict(blocks=0)), (SHAPE, dict(pages=0)),
                                     (SHAPE, dict(pages=1 << 27)), (SHAPE, dict(B=8192, T=1 << 19))])
def test_map_refuses(bd, code, kw):
    assert _call(bd, "switchsd_kv_map", "switchsd_kv_map_params", MAP, **kw) == code


@pytest.mark.parametrize("code,kw", [(ARG, dict(k=None)), (ARG, dict(v=None)), (ARG, dict(slots=None)), (ARG, dict(cache=None)), (ARG, dict(dtype=2)),
                                     (ARG, dict(dtype=-1)), (ARG, dict(k=FAKE + 8)), (ARG, dict(cache=FAKE + 4)), (ARG, dict(k_stride=(384, 128, 68))),
                                     (ARG, dict(v_stride=(-384, 128, 64))), (SHAPE, dict(D=96)), (SHAPE, dict(D=256)), (SHAPE, dict(Hkv=0)), (SHAPE, dict(page=20)),
                                     (SHAPE, dict(B=0)), (SHAPE, dict(T=0)), (SHAPE, dict(pages=1 << 28)), (SHAPE, dict(B=1 << 20, T=1 << 12))])
def test_append_refuses(bd, code, kw):
    assert _call(bd, "switchsd_kv4_append", "switchsd_kv4_append_params", APPEND, **kw) == code


@pytest.mark.parametrize("code,kw", [(ARG, dict(cache=None)), (ARG, dict(slots=None)), (ARG, dict(out_k=None)), (ARG, dict(out_v=FAKE + 2)), (SHAPE, dict(D=32)),
                                     (SHAPE, dict(page=0)), (SHAPE, dict(pages=0))])
def test_read_refuses(bd, code, kw):
    assert _call(bd, "switchsd_kv4_read", "switchsd_kv4_read_params", READ, **kw) == code


@pytest.mark.parametrize("code,kw", [(ARG, dict(q=None)), (ARG, dict(cache=None)), (ARG, dict(block_table=None)), (ARG, dict(lens=None)), (ARG, dict(new_lens=None)),
                                     (ARG, dict(out=None)), (ARG, dict(workspace=None)), (ARG, dict(workspace_bytes=0)), (ARG, dict(dtype=2)), (ARG, dict(q=FAKE + 2)),
                                     (ARG, dict(workspace=FAKE + 8)), (ARG, dict(q_stride=(768, 252, 64))), (SHAPE, dict(Hq=3)), (SHAPE, dict(Hq=130)),
                                     (SHAPE, dict(Hq=0)), (SHAPE, dict(Hkv=0)), (SHAPE, dict(D=80)), (SHAPE, dict(page=1)), (SHAPE, dict(blocks=0)),
                                     (SHAPE, dict(B=0)), (SHAPE, dict(T=0)), (SHAPE, dict(blocks=1 << 28)), (SHAPE, dict(pages=1 << 28))])
def test_attention_refuses(bd, code, kw):
    assert _call(bd, "switchsd_kv4_attention", "switchsd_kv4_attention_params", ATTN, **kw) == code


@pytest.mark.parametrize("code,kw", [(ARG, dict(logits=None)), (ARG, dict(argmax=None)), (ARG, dict(dtype=3)), (ARG, dict(logits=FAKE + 1)), (ARG, dict(ctx_lens=None)),
                                     (ARG, dict(ctx_tokens=FAKE + 4)), (ARG, dict(nbias=3)), (ARG, dict(workspace=None)), (ARG, dict(workspace=FAKE + 4)), (ARG, dict(workspace_bytes=8)), (ARG, dict(nbias=-1)), (ARG, dict(stride_t=-100)), (SHAPE, dict(B=0)),
                                     (SHAPE, dict(B=65536)), (SHAPE, dict(T=0)), (SHAPE, dict(V=0)), (SHAPE, dict(V=262145)), (SHAPE, dict(cap=6)),
                                     (SHAPE, dict(draft_stride=1)), (SHAPE, dict(mask=FAKE, mask_words=3)), (SHAPE, dict(nbias=4097, bias_ids=FAKE, bias=FAKE))])
def test_logits_refuses(bd, code, kw):
    assert _call(bd, "switchsd_logits", "switchsd_logits_params", LOGITS, **kw) == code


def test_null_parameters(bd):
    for name in ("switchsd_kv_map", "switchsd_kv4_append", "switchsd_kv4_read", "switchsd_kv4_attention", "switchsd_logits"):
        assert getattr(bd.load(), name)(None) == ARG
    assert bd.load().switchsd_kv4_attention_workspace_bytes(None) == 0


def test_bytes_of_a_page_and_head(bd):
    assert bd.switchsd_kv4_bytes(16, 128) == 16 * 136 and bd.switchsd_kv4_bytes(64, 64) == 64 * 68
    for page, D in ((8, 64), (48, 64), (512, 64), (16, 32), (16, 96), (16, 256), (0, 64), (-16, 64)):
        assert bd.switchsd_kv4_bytes(page, D) == 0
