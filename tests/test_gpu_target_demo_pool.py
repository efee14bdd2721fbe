"""The small target on a pool that is too short: rows sit steps out and lose nothing."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("drafts", [False, True])
def test_rows_that_sit_steps_out_keep_their_text(drafts):
    from paper_2609_20186_gb300 import target_demo as demo
    target = demo.SmallTarget()
    prompts, lens = demo.prompts_of(6, target)

    def decode(pages, steps):
        d = demo.Decoder(target, prompts, lens, room=640, drafts=drafts, pages=pages)
        out = 0
        for _ in range(steps):
            before = d.sess.lens.clone()
            d.step()
            held_back = d.cache.status.cpu().numpy() == 1
            out += int(held_back.sum())
            grew = (d.sess.lens - before).cpu().numpy()
            assert (grew[held_back] == 0).all() and (grew[~held_back] > 0).all()
            assert int(d.cache.held.sum()) + int(d.cache.free_count) == d.cache.pages
        ctx, now = d.sess.ctx.cpu().numpy(), d.sess.lens.cpu().numpy()
        return [ctx[b, lens[b]:now[b]] for b in range(6)], out
    full, out = decode(None, 30)
    assert out == 0
    some, out = decode(int((-(-lens // 16)).sum()) + 5, 30)
    assert out > 10
    for a, b in zip(full, some):
        assert len(b) <= len(a) and np.array_equal(a[:len(b)], b)
    assert sum(map(len, some)) > 6


def test_prompts_that_do_not_fit_are_refused():
    from paper_2609_20186_gb300 import target_demo as demo
    target = demo.SmallTarget()
    prompts, lens = demo.prompts_of(6, target)
    with pytest.raises(RuntimeError):
        demo.Decoder(target, prompts, lens, pages=2)
