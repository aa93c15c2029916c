"""What measured times become in a planner problem (no GPU needed: the measurement is made up)."""
import numpy as np
import pytest

from paper_2609_39350_amd import binding, measure, workloads


def made_up(problem, experts_ns=9_000_017.0):
    m = problem["model"]
    layer = int(np.flatnonzero(m["is_moe"])[0])
    return {"layer": layer, "tokens": int(m["seq_len"]) * int(m["micro_batch_size"]), "hidden": int(m["hidden"]),
            "width": 512, "experts": int(m["n_experts"]), "part": 1, "route_ns": 2e5, "combine_ns": 1e5,
            "experts_ns": experts_ns, "opt_ns_per_param": 0.005,
            "expert_tokens": np.full(int(m["n_experts"]), 3, dtype=np.int64)}


def expert_term(problem, h):
    """Eq. 2's expert time at EP = TPE = TP = CP = 1 without imbalance, for every MoE layer."""
    m, c = problem["model"], problem["cluster"]
    moe = np.asarray(m["is_moe"]) == 1
    return m["moe_ffn_mult"] * c["t_ffn"][h][0, 0, moe] / c["eff"][h]


@pytest.mark.parametrize("n,shared", [(1, 0), (2, 0), (3, 1), (4, 0), (5, 1)])
def test_expert_term_is_the_routed_and_the_shared_experts_time(n, shared):
    problem = workloads.config(n)
    m, h = problem["model"], problem["cluster"]["n_types"] - 1
    k = int(m["top_k"])
    assert m["moe_ffn_mult"] == k + shared
    got = made_up(problem)
    q = measure.apply(problem, h, got)
    binding.validate(q)
    want = got["experts_ns"] * (k + shared) / k
    moe = np.asarray(m["is_moe"]) == 1
    assert np.all(q["cluster"]["t_ffn"][h][0, 0, moe] == np.ceil(got["experts_ns"] / k))   # one expert's
    assert np.all(np.abs(expert_term(q, h) - want) <= m["moe_ffn_mult"])   # t_ffn is rounded up to whole ns
    # the share over TP and CP, the dense layers, the other parts of a layer and the other types stay
    was, now = problem["cluster"], q["cluster"]
    share = was["t_ffn"][h][:, :, moe] / was["t_ffn"][h][0, 0, moe]
    assert np.all(np.abs(now["t_ffn"][h][:, :, moe] - share * got["experts_ns"] / k) <= 1)
    assert np.array_equal(now["t_ffn"][h][:, :, ~moe], was["t_ffn"][h][:, :, ~moe])
    assert np.array_equal(now["t_dense"][h] - now["t_ffn"][h], was["t_dense"][h] - was["t_ffn"][h])
    assert all(np.array_equal(now[f][o], was[f][o]) for f in ("t_ffn", "t_dense") for o in range(h))


@pytest.mark.parametrize("mult,shared,of_routed", [
    (1.0, None, 1.0),        # experts of half the dense FFN: all of the factor is routed
    (4.0, 0, 1.0),           # experts of twice the dense FFN, none shared
    (4.0, None, 2.0),        # two shared beside two routed
    (3.0, 1, 1.5), (6.0, 1, 1.5)])
def test_expert_term_by_factor_and_shared_experts(mult, shared, of_routed):
    problem = workloads.config(1)   # top 2
    problem["model"]["moe_ffn_mult"] = mult
    got = made_up(problem)
    q = measure.apply(problem, 0, got, shared=shared)
    binding.validate(q)
    assert np.all(np.abs(expert_term(q, 0) - of_routed * got["experts_ns"]) <= mult)


def test_a_factor_of_zero():
    problem = workloads.config(1)
    problem["model"]["moe_ffn_mult"] = 0.0
    q = measure.apply(problem, 0, made_up(problem))
    binding.validate(q)
    assert np.all(expert_term(q, 0) == 0)


def test_counts_of_a_profile_stay():
    """The measured layer's router is random: its counts replace those of a problem only where they are asked for."""
    problem = workloads.config(2)
    got = made_up(problem)
    tokens = problem["model"]["expert_tokens"].copy()
    kept = measure.apply(problem, 1, got, counts=False)
    assert np.array_equal(kept["model"]["expert_tokens"], tokens)
    taken = measure.apply(problem, 1, got, counts=True)
    assert np.array_equal(taken["model"]["expert_tokens"][got["layer"]], got["expert_tokens"])
    for q in (kept, taken):
        assert np.array_equal(problem["model"]["expert_tokens"], tokens)
        assert np.array_equal(np.delete(q["model"]["expert_tokens"], got["layer"], 0), np.delete(tokens, got["layer"], 0))


def test_command_plans_with_the_workloads_counts(monkeypatch, capsys):
    planned = []

    class Planner:
        def __init__(self, problem, device):
            planned.append(problem)

        def run(self):
            return {"config": (1,) * 6, "n_micro": 1, "objective": 1, "layers": [1]}

    problem = workloads.config(3)
    monkeypatch.setattr(measure, "measure", lambda p, **kw: made_up(p))
    monkeypatch.setattr(measure.binding, "Planner", Planner)
    measure.main(["--config", "3", "--type", "1"])
    assert len(planned) == 2 and len(capsys.readouterr().out.splitlines()) == 4
    for q in planned:
        assert np.array_equal(q["model"]["expert_tokens"], problem["model"]["expert_tokens"])
    assert not np.array_equal(planned[0]["cluster"]["t_ffn"][1], planned[1]["cluster"]["t_ffn"][1])
