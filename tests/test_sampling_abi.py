"""Host-side validation of the 16-bit cache's and the sampling's entry points, without a GPU: the documented codes come back
before any CUDA call is made."""
import ctypes

import pytest
import torch

FAKE = 0x10000  # a 16-byte-aligned non-NULL address; never dereferenced by host validation
ARG, SHAPE = -1, -2


@pytest.fixture(scope="module")
def bd():
    from paper_2609_20186_gb300 import build, binding
    build.build()
    binding.load()
    return binding


def _call(bd, name, base, **kw):
    p = getattr(bd, name + "_params")()
    for key, v in {**base, **kw}.items():
        setattr(p, key, (ctypes.c_int64 * 3)(*v) if isinstance(v, tuple) else v)
    return getattr(bd.load(), name)(ctypes.byref(p))


APPEND = dict(B=2, T=3, Hkv=2, D=64, page=16, pages=9, dtype=0, k=FAKE, v=FAKE, k_stride=(384, 128, 64), v_stride=(384, 128, 64), slots=FAKE, cache=FAKE)
READ = dict(B=2, T=3, Hkv=2, D=64, page=16, pages=9, cache=FAKE, slots=FAKE, out_k=FAKE, out_v=FAKE)
ATTN = dict(B=2, T=3, Hq=4, Hkv=2, D=64, page=16, pages=9, blocks=4, dtype=0, q=FAKE, q_stride=(768, 256, 64), cache=FAKE, block_table=FAKE, lens=FAKE,
            new_lens=FAKE, scale=0.1, out=FAKE, workspace=FAKE, workspace_bytes=1 << 40)
PROBS = dict(B=2, T=3, V=100, K=3, top=5, dtype=0, logits=FAKE, stride_b=300, stride_t=100, tokens=FAKE, tokens_stride=3, logprob=FAKE, prob=FAKE, entropy=FAKE,
             lse=FAKE, top_ids=FAKE, top_logprobs=FAKE)
TOKEN = dict(B=2, T=3, V=100, dtype=0, logits=FAKE, stride_b=300, stride_t=100, lse=FAKE, draft=FAKE, draft_len=FAKE, p_draft=FAKE, u=FAKE, q_logits=FAKE,
             q_stride_b=200, q_stride_t=100, q_lse=FAKE, seeds=FAKE, ctx_lens=FAKE, out=FAKE)


@pytest.mark.parametrize("code,kw", [(ARG, dict(k=None)), (ARG, dict(v=None)), (ARG, dict(slots=None)), (ARG, dict(cache=None)), (ARG, dict(dtype=2)),
                                     (ARG, dict(dtype=-1)), (ARG, dict(k=FAKE + 8)), (ARG, dict(cache=FAKE + 4)), (ARG, dict(k_stride=(384, 128, 68))),
                                     (ARG, dict(v_stride=(-384, 128, 64))), (SHAPE, dict(D=96)), (SHAPE, dict(D=256)), (SHAPE, dict(Hkv=0)), (SHAPE, dict(page=20)),
                                     (SHAPE, dict(B=0)), (SHAPE, dict(T=0)), (SHAPE, dict(pages=0)), (SHAPE, dict(pages=1 << 28)), (SHAPE, dict(B=1 << 20, T=1 << 10)),
                                     (SHAPE, dict(B=1 << 15, T=1 << 10, Hkv=32))])
def test_append_refuses(bd, code, kw):
    assert _call(bd, "switchsd_kv16_append", APPEND, **kw) == code


@pytest.mark.parametrize("code,kw", [(ARG, dict(cache=None)), (ARG, dict(slots=None)), (ARG, dict(out_k=None)), (ARG, dict(out_v=FAKE + 2)), (SHAPE, dict(D=32)),
                                     (SHAPE, dict(page=0)), (SHAPE, dict(pages=0)), (SHAPE, dict(B=1 << 15, T=1 << 15))])
def test_read_refuses(bd, code, kw):
    assert _call(bd, "switchsd_kv16_read", READ, **kw) == code


@pytest.mark.parametrize("code,kw", [(ARG, dict(q=None)), (ARG, dict(cache=None)), (ARG, dict(block_table=None)), (ARG, dict(lens=None)), (ARG, dict(new_lens=None)),
                                     (ARG, dict(out=None)), (ARG, dict(workspace=None)), (ARG, dict(workspace_bytes=0)), (ARG, dict(dtype=2)), (ARG, dict(q=FAKE + 2)),
                                     (ARG, dict(workspace=FAKE + 8)), (ARG, dict(q_stride=(768, 252, 64))), (SHAPE, dict(Hq=3)), (SHAPE, dict(Hq=130)),
                                     (SHAPE, dict(Hq=0)), (SHAPE, dict(Hkv=0)), (SHAPE, dict(D=80)), (SHAPE, dict(page=1)), (SHAPE, dict(blocks=0)),
                                     (SHAPE, dict(B=0)), (SHAPE, dict(T=0)), (SHAPE, dict(blocks=1 << 28)), (SHAPE, dict(pages=1 << 28))])
def test_attention_refuses(bd, code, kw):
    assert _call(bd, "switchsd_kv16_attention", ATTN, **kw) == code


@pytest.mark.parametrize("code,kw", [(ARG, dict(logits=None)), (ARG, dict(dtype=3)), (ARG, dict(logits=FAKE + 1)), (ARG, dict(dtype=2, logits=FAKE + 2)), (ARG, dict(tokens=None)),
                                     (ARG, dict(K=0)), (ARG, dict(top=0)), (ARG, dict(top=-1)), (ARG, dict(stride_t=-100)), (ARG, dict(stride_b=-1)),
                                     (ARG, dict(logprob=None, prob=None, entropy=None, lse=None, top_ids=None, top_logprobs=None)),
                                     (SHAPE, dict(B=0)), (SHAPE, dict(B=65536)), (SHAPE, dict(T=0)), (SHAPE, dict(T=262141)), (SHAPE, dict(V=0)), (SHAPE, dict(V=262145)),
                                     (SHAPE, dict(K=4)), (SHAPE, dict(top=33)), (SHAPE, dict(tokens_stride=2))])
def test_logprobs_refuses(bd, code, kw):
    assert _call(bd, "switchsd_logprobs", PROBS, **kw) == code


@pytest.mark.parametrize("code,kw", [(ARG, dict(logits=None)), (ARG, dict(draft=None)), (ARG, dict(draft_len=None)), (ARG, dict(p_draft=None)), (ARG, dict(u=None)),
                                     (ARG, dict(seeds=None)), (ARG, dict(ctx_lens=None)), (ARG, dict(out=None)), (ARG, dict(lse=None)), (ARG, dict(q_lse=None)),
                                     (ARG, dict(dtype=3)), (ARG, dict(logits=FAKE + 1)), (ARG, dict(q_logits=FAKE + 1)), (ARG, dict(stride_t=-100)),
                                     (ARG, dict(q_stride_b=-200)), (SHAPE, dict(B=0)), (SHAPE, dict(B=65536)), (SHAPE, dict(T=0)), (SHAPE, dict(T=262141)),
                                     (SHAPE, dict(V=0)), (SHAPE, dict(V=262145))])
def test_resample_refuses(bd, code, kw):
    assert _call(bd, "switchsd_resample", TOKEN, **kw) == code


def test_null_parameters(bd):
    for name in ("switchsd_kv16_append", "switchsd_kv16_read", "switchsd_kv16_attention", "switchsd_logprobs", "switchsd_resample"):
        assert getattr(bd.load(), name)(None) == ARG
    assert bd.load().switchsd_kv16_attention_workspace_bytes(None) == 0
    assert bd.switchsd_kv16_attention_workspace(96) == 0 < bd.switchsd_kv16_attention_workspace(64) < bd.switchsd_kv16_attention_workspace(128)


def test_the_binding_refuses(bd):
    """Tensors of the wrong kind, named in the message."""
    x = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16)
    cache, ids = torch.zeros(9, 2, 4, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(TypeError, match="k must be a CUDA tensor"):
        bd.switchsd_kv16_append(x, x, ids, cache)
    with pytest.raises(ValueError, match="the cache has shape"):
        bd.switchsd_kv16_append(x, x, ids, cache[:, 0])
    with pytest.raises(ValueError, match="the cache has shape"):
        bd.switchsd_kv16_read(cache, ids, x[:, :, :3], x[:, :, :3])
    with pytest.raises(TypeError, match="the cache must be bfloat16 or float16"):
        bd.switchsd_kv16_attention(x, cache.float(), ids, ids[:, 0], ids[:, 0], x)
    with pytest.raises(TypeError, match="q must be a CUDA tensor"):
        bd.switchsd_kv16_attention(x, cache, ids, ids[:, 0], ids[:, 0], x)
    with pytest.raises(TypeError, match="logits must be a CUDA tensor"):
        bd.switchsd_logprobs(torch.zeros(2, 3, 100), lse=torch.zeros(2, 3))
    with pytest.raises(TypeError, match="logits must be a CUDA tensor"):
        bd.switchsd_resample(torch.zeros(2, 3, 100), ids, ids[:, 0], ids, ids, ids, seeds=ids, ctx_lens=ids)


def test_a_cache_of_another_type_is_refused(bd):
    from paper_2609_20186_gb300 import KVCache
    with pytest.raises(ValueError, match="no cache holds"):
        KVCache(1, 1, layers=1, heads=1, dim=64, pages=1, max_len=16, page=16, dtype=torch.float32, device="cpu")


def test_parameter_blocks_as_bytes(bd):
    """Every field of the blocks that the binding packs lies where the structure has it."""
    import re
    import struct
    for params, fmt in bd._BLOCKS.items():
        fields = [(name, i) for name, t in params._fields_ for i in (range(3) if t is bd._c_i64x3 else (None,))]
        codes = [c for n, c in re.findall(r"(\d*)([a-zA-Z])", fmt[1:]) for _ in range(int(n or 1))]
        assert len(fields) == len(codes)
        p = params.from_buffer_copy(struct.pack(fmt, *(i + 1 for i in range(len(codes)))))
        for i, (name, k) in enumerate(fields):
            got = getattr(p, name)
            assert (got if k is None else got[k]) == i + 1, (params, name)
