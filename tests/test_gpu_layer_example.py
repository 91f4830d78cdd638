"""The decoder-layer operators together, as examples/shared_video.py runs them (GPU)."""
import pytest

from tests.gpu_helpers import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(questions=5, frames=3, steps=3, drafts=4, heads=14, kv_heads=2, d=128),
                                dict(questions=2, frames=1, steps=2, drafts=1, heads=4, kv_heads=4, d=64)])
def test_questions_about_one_video(kw):
    require_gpu()
    from examples.shared_video import run

    said, worst = run(check=True, vocab=500, **kw)
    # Final hidden states are rms-normed to 1; the two attentions differ by bf16
    # roundings of their outputs (2^-8 of about 0.2) in two layers, and the residual
    # stream, the projections and the norm round to bf16 likewise: a few 2^-8.
    assert worst <= 16 * 2.0 ** -8
    for tokens in said:
        assert kw["steps"] <= len(tokens) <= kw["steps"] * (kw["drafts"] + 1)
        assert all(0 <= t < 500 for t in tokens)
    again, _ = run(vocab=500, **kw)
    assert again == said  # deterministic
