"""What the operators on rows ask for as scratch stays within a card's memory for any number of queries."""
import pytest

pytest.importorskip("torch")
avq = pytest.importorskip("paper_1908_10396_amd")


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("n,d", [(1_183_514, 100), (670_091, 1024), (10_000, 32)])
def test_log_probabilities_of_many_queries_with_alternatives(kind, n, d):
    L = avq.lib()
    sizes = [L.avq_log_probs_scratch(kind, n, d, nq, 1, 10) for nq in (1, 64, 65, 2048, 8192, 65_536, 1 << 19)]
    assert all(s > 0 for s in sizes)
    # operands of the rows and maxima of the groups, 1 GiB each, and what every query takes: its operands, statistics and id
    per_query = 4 * (d + 64) + 20 * 16 * 2 + 64
    for nq, s in zip((1, 64, 65, 2048, 8192, 65_536, 1 << 19), sizes):
        assert s <= (2 << 30) + 16 * n + nq * per_query + (64 << 20)
