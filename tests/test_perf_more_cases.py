"""The cases of perf/more_operators.py within every limit of the calls, one by one."""
import random

from test_perf_more_operators import operators  # noqa: F401


def test_every_case_is_within_the_limits(operators):  # noqa: F811
    from paper_2311_09445_b200 import layers, routing
    rng = random.Random(11)
    for c in operators.listed() + [operators.draw(rng) for _ in range(500)]:
        assert 1 <= c["rows"] < 1 << 31 and c["width"] >= 1, c
        if c["op"] in ("norm", "norm_grad"):
            assert c["width"] <= layers.MAX_WIDTH, c
            assert c["ld"] == 0 or c["ld"] >= c["width"], c
        elif c["op"] == "dropout":
            assert c["width"] * operators.BYTES[c["dtype"]] <= 1 << 23 and 0 <= c["p"] <= 1, c
        else:
            assert c["rows"] <= layers.MAX_FEW and 1 <= c["k"] <= min(c["experts"], routing.MAX_CHOICES), c
            assert c["width"] <= layers.MAX_INNER and 1 <= c["hidden"] <= layers.MAX_INNER and c["experts"] <= routing.MAX_EXPERTS, c
            assert 0 <= c["barred"] < 1, c
