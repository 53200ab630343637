"""The oracle of the token losses where a factor of zero meets what is infinite.  Needs no GPU."""
import math

from oracle import learning as le


def test_pairs_with_an_answer_of_probability_zero():
    inf = math.inf
    for beta in (0.1, 2.0):
        assert le.pair(-3.0, -inf, beta, 0.0, 1) == (0.0, 0.0)
        assert le.pair(-inf, -3.0, beta, 0.0, 1) == (inf, -beta)
        assert le.pair(-inf, -3.0, beta, 1.0, 1) == (0.0, 0.0)
        assert le.pair(-3.0, -inf, beta, 1.0, 1) == (inf, beta)
        assert le.pair(-3.0, -inf, beta, 0.5, 1)[0] == inf
