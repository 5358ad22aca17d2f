"""More pins of the oracle of the calls around attention."""
import math

import numpy as np

from oracle import answer


def test_top_p_is_a_share_of_what_top_k_left():
    """Of 0.4 and 0.3 the first is four sevenths, 0.571: below that it is enough, above it is not.  Of all four words neither 0.56 nor 0.58 is reached by one, and 0.72 not by two."""
    x = np.log([0.1, 0.4, 0.3, 0.2])
    assert answer.kept_tokens(x, top_k=2, top_p=0.56)[0] == [1]
    assert answer.kept_tokens(x, top_k=2, top_p=0.58)[0] == [1, 2]
    assert answer.kept_tokens(x, top_p=0.56)[0] == [1, 2] and answer.kept_tokens(x, top_p=0.72)[0] == [1, 2, 3]
    # and min-p of the largest, whatever the others left
    assert answer.kept_tokens(x, top_k=3, top_p=0.99, min_p=0.74)[0] == [1, 2] and answer.kept_tokens(x, top_k=3, min_p=0.49)[0] == [1, 2, 3]
    token, kept, logprob = answer.sample(x, 0.999, top_k=2, top_p=0.56)
    assert (token, kept, logprob) == (1, 1, 0.0)
    token, kept, logprob = answer.sample(x, 0.999, top_k=2, top_p=0.58)
    assert (token, kept) == (2, 2) and math.isclose(logprob, math.log(3 / 7))


def test_words_ruled_out_by_finite_numbers_count():
    """They may be drawn, so the first top_k in order may hold some; they weigh nothing."""
    x = [-1e9, 1.0, -1e9, 0.0, -1e9]
    assert answer.kept_tokens(x, top_k=3)[0] == [1, 3, 0] and answer.kept_tokens(x, top_k=3, top_p=0.9)[0] == [1, 3]
    token, kept, logprob = answer.sample(x, 0.9, top_k=4)
    assert (token, kept) == (3, 4) and math.isclose(logprob, -1 - math.log(1 + math.exp(-1)))


def test_relu_keeps_what_is_no_number():
    assert np.isnan(answer.activate("relu", np.array([np.nan, -1.0]))[0]) and answer.activate("relu", np.array([np.nan, -1.0]))[1] == 0
