"""The measuring command takes no option that it would leave out (no GPU needed: it ends before any is used)."""
import pytest

from paper_2609_39350_amd import measure


@pytest.fixture
def taken(monkeypatch):
    """What the command measures with."""
    got = {}

    class Done(Exception):
        pass

    def stop(problem, **how):
        got.update(how)
        raise Done

    monkeypatch.setattr(measure, "measure", stop)

    def run(*argv):
        got.clear()
        with pytest.raises(Done):
            measure.main(list(argv))
        return dict(got)
    return run


@pytest.mark.parametrize("argv", [["--groups", "8"], ["--groups", "1"], ["--top-groups", "2"], ["--groups", "8", "--block"],
                                  ["--vocab", "100"], ["--vocab", "100", "--scores", "sigmoid"], ["--block", "--vocab", "0"],
                                  ["--scores", "tanh"]])
def test_refused(argv, taken, capsys):
    with pytest.raises(SystemExit) as e:
        measure.main(["--config", "1"] + argv)
    assert e.value.code == 2 and "--" in capsys.readouterr().err


def test_taken(taken):
    none = taken("--config", "1")
    assert none["balance"] is None and none["vocab"] == 0
    assert taken("--config", "1", "--block")["vocab"] == 32768
    assert taken("--config", "1", "--block", "--vocab", "100")["vocab"] == 100
    balance = taken("--config", "1", "--scores", "sigmoid")["balance"]
    assert balance == {"scores": "sigmoid", "groups": 1, "top_groups": None}
    balance = taken("--config", "1", "--scores", "softmax", "--groups", "4", "--top-groups", "2")["balance"]
    assert balance == {"scores": "softmax", "groups": 4, "top_groups": 2}
