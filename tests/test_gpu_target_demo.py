"""The target's operators and the controller together: drafts change how fast a text comes, not the text."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _decode(drafts, steps):
    from paper_2609_20186_gb300 import target_demo as demo
    target = demo.SmallTarget()
    prompts, lens = demo.prompts_of(6, target)
    d = demo.Decoder(target, prompts, lens, room=640, drafts=drafts)
    for _ in range(steps):
        before = d.sess.lens.clone()
        cached = before - 1 + d.sess.vlen + 1
        d.step()
        assert not d.sess.vstatus.any() and not d.cache.status.any()
        # the step's tokens have pages, and no page is lost
        assert np.array_equal(d.cache.held.cpu().numpy(), -(-cached.cpu().numpy() // d.cache.page))
        assert int(d.cache.held.sum()) + int(d.cache.free_count) == d.cache.pages
        assert np.array_equal((d.sess.lens - before).cpu().numpy(), d.sess.accept.cpu().numpy() + 1)
    ctx, now = d.sess.ctx.cpu().numpy(), d.sess.lens.cpu().numpy()
    return [ctx[b, lens[b]:now[b]] for b in range(6)], target


def test_drafts_leave_the_text_as_it_is():
    plain, target = _decode(False, 40)
    drafted, _ = _decode(True, 40)
    follows = target.follows.cpu().numpy()
    for p, d in zip(plain, drafted):
        assert len(p) == 40 and np.array_equal(d[:40], p)
        assert np.array_equal(d[1:], follows[d[:-1]])  # the head's margin is far above every rounding
    assert sum(map(len, drafted)) > 2 * sum(map(len, plain))


def test_the_command_runs(capsys):
    from paper_2609_20186_gb300 import target_demo as demo
    demo.main(["--rows", "2", "--steps", "4"])
    assert "4 steps of 2 rows" in capsys.readouterr().out
