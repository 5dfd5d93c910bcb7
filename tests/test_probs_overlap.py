"""Probabilities written over the temperatures that other rows are still to read are refused (CPU: before any GPU work)."""

FAKE = 1 << 20  # an address that no call below gets to use


def test_results_over_the_temperatures_are_refused():
    from paper_2405_03594_gb300 import sp

    def call(temperature, out=2 * FAKE, tokens=3, vocab=100, out_stride=110):
        return sp._lib.sp_token_probs(FAKE, 0, 100, tokens, vocab, temperature, 1.0, 0.0, out, out_stride, None)

    last = 2 * FAKE + 4 * (2 * 110 + 100)  # behind the last entry
    for at in (2 * FAKE, 2 * FAKE - 8, 2 * FAKE + 4, last - 4):
        assert call(at) == 1, at
