"""A layer that runs in parts, in its place: what stands around it is timed at its whole size."""
import pytest

from paper_2609_39350_amd import workloads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


def test_norm_embedding_and_dropout_are_timed_at_their_whole_size(torch, monkeypatch):
    """Where a part of the experts runs with a part of the tokens, a part's time of these is more than a part of the
    whole's: launches count in each."""
    from paper_2609_39350_amd import measure
    problem = workloads.config(1)
    m = problem["model"]
    whole, hidden = int(m["seq_len"]) * int(m["micro_batch_size"]), int(m["hidden"])
    names = ("embed", "embed_backward", "layer_norm", "layer_norm_backward", "dropout")
    seen = {name: [] for name in names}
    for name in names:
        real = getattr(measure.operators, name)

        def call(*a, real=real, name=name, **k):
            rows = a[0].shape[0]   # tokens, or rows of the matrix
            seen[name].append(rows)
            return real(*a, **k)

        monkeypatch.setattr(measure.operators, name, call)
    steps, warmup = 3, 1
    got = measure.measure(problem, steps=steps, warmup=warmup, limit_bytes=10**8, state_bits=8, vocab=300,
                          balance={"scores": "sigmoid"})
    assert got["part"] > 1
    for name, rows in seen.items():
        # dropout_backward is a call of dropout
        assert rows.count(whole) == (steps + warmup) * (2 if name == "dropout" else 1), (name, rows)
    assert all(got[n] > 0 for n in ("embed_ns", "norm_ns", "dropout_ns"))
