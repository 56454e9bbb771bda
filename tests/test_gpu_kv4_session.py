"""The example session over 4-bit caches runs, and 4 bits stay near bf16."""
import pytest

pytestmark = pytest.mark.gpu


def test_session():
    from examples import kv4_session
    r = kv4_session.main(["--layers", "2", "--hidden", "512", "--heads", "8", "--kv-heads", "2", "--prompt", "300",
                          "--chunk", "128", "--steps", "6"])
    # 4.5 of 16 bits and slots rounded up to 64
    assert r["bytes"] < 0.30 * r["bytes_bf16"]
    # a value of a normal group is off by at most half a step, (hi - lo) / 30 of about 4.2 deviations: 0.14 / sqrt 3 rms,
    # a few percent more for the rounded-up scale; measured against deviation 1
    assert 0.03 < r["k"] < 0.11 and 0.03 < r["v"] < 0.11
    # attention averages such errors and the residual stream carries most of the state
    assert r["prompt"] < 0.05


def test_decoded_and_drafted_tokens_stay_near_bf16():
    """What the graph and the verification compute, and the slot that the first decoded token fills."""
    from examples import kv4_session
    r = kv4_session.main(["--layers", "2", "--hidden", "512", "--heads", "8", "--kv-heads", "2", "--prompt", "300",
                          "--chunk", "128", "--steps", "1"])
    # the same reasons and bar as for the prompt's states; the drafts are the same tokens in both sessions
    assert r["token"] < 0.05 and r["drafts"] < 0.05
    # quantised as the prompt's (0.11), of a state that is itself off by up to 0.05: 0.121 together
    assert 0.03 < r["token_k"] < 0.125 and 0.03 < r["token_v"] < 0.125
