"""The controller, the 16-bit cache and the sampling's operators together: what a step at temperature > 0 runs."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _decode(steps, **kw):
    import torch
    from paper_2609_20186_gb300 import target_demo as demo
    target = demo.SmallTarget()
    prompts, lens = demo.prompts_of(6, target)
    d = demo.Decoder(target, prompts, lens, room=640, **kw)
    for _ in range(steps):
        before = d.sess.lens.clone()
        d.step()
        assert not d.sess.vstatus.any() and not d.cache.status.any() and not d.cache.attend_status.any()
        assert int(d.cache.held.sum()) + int(d.cache.free_count) == d.cache.pages
        assert torch.equal(d.sess.lens - before, d.sess.accept + 1)
    ctx, now = d.sess.ctx.cpu().numpy(), d.sess.lens.cpu().numpy()
    return [ctx[b, lens[b]:now[b]] for b in range(6)], target


@pytest.mark.parametrize("cache16", [False, True])
def test_a_temperature_of_0_is_the_greedy_verification(cache16):
    import torch
    dtype = torch.bfloat16 if cache16 else None
    # (40 steps: a text repeats, and so has drafts, once its cycle of 24 tokens is over)
    greedy, _ = _decode(40, dtype=dtype)
    sampled, _ = _decode(40, dtype=dtype, temperature=0.0)
    for g, s in zip(greedy, sampled):
        assert np.array_equal(g, s)
    assert sum(map(len, sampled)) > 2 * 40 * 6  # drafts are accepted


def test_drafts_leave_the_text_as_it_is_with_a_cache_of_16_bits():
    import torch
    plain, target = _decode(30, dtype=torch.bfloat16, drafts=False)
    drafted, _ = _decode(30, dtype=torch.bfloat16)
    follows = target.follows.cpu().numpy()
    for p, d in zip(plain, drafted):
        assert np.array_equal(d[:30], p) and np.array_equal(d[1:], follows[d[:-1]])  # the head's margin is far above every rounding


@pytest.mark.parametrize("temperature", [0.7, 40.0])
def test_texts_at_a_temperature(temperature):
    """The same seed gives the same text, another one another where the temperature leaves more than one token; the banned
    token never comes."""
    import torch
    a, target = _decode(25, dtype=torch.bfloat16, temperature=temperature, seed=3)
    b, _ = _decode(25, dtype=torch.bfloat16, temperature=temperature, seed=3)
    c, _ = _decode(25, dtype=torch.bfloat16, temperature=temperature, seed=4)
    assert all(np.array_equal(x, y) for x, y in zip(a, b))
    assert all((x >= 0).all() and (x < target.vocab - 1).all() for x in a + c)
    if temperature > 1:
        assert any(not np.array_equal(x[:20], y[:20]) for x, y in zip(a, c))


def test_the_command_runs(capsys):
    from paper_2609_20186_gb300 import target_demo as demo
    demo.main(["--rows", "2", "--steps", "4", "--temperature", "0.8", "--cache16"])
    assert "4 steps of 2 rows" in capsys.readouterr().out
