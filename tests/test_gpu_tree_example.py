"""Trees of drafts over bounded caches together, as examples/tree_chat.py runs them (GPU)."""
import pytest

from tests.gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(chats=3, length=320, steps=4, budget=256, slack=8),
                                dict(chats=2, length=128, steps=3, budget=1000, heads=4, kv_heads=4, d=64, tau=0.7)])
def test_chats(kw):
    require_gpu()
    from examples.tree_chat import run

    said, lengths, worst = run(check=True, **kw)
    # Final hidden states are rms-normed to 1; the two attentions differ by bf16
    # roundings of their outputs (2^-8 of about 0.2) in two layers, and the residual
    # stream, the projections and the norm round to bf16 likewise: a few 2^-8.
    assert worst <= 16 * 2.0 ** -8
    for b, tokens in enumerate(said):
        assert kw["steps"] <= len(tokens) <= 14 * kw["steps"] and all(0 <= t < 500 for t in tokens)
        if kw["budget"] > kw["length"]:  # nothing is evicted: every emitted token has joined the context
            assert lengths[-1][b] == kw["length"] + len(tokens)
        else:
            assert all(step[b] <= kw["budget"] + 8 for step in lengths) and lengths[0][b] == kw["budget"]
    assert run(**kw)[:2] == (said, lengths)  # deterministic
