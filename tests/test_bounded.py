"""The bounded request: the replay, chunked attention, the account, eviction and a drafted tree together."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_a_bounded_request_is_served_where_the_whole_one_is_refused():
    from paper_2605_24259_amd import bounded
    assert bounded.asked(60, 70, 80) == (2, 0, 60, 70)  # refused, claim 0, 60 + 70 > 80
    r = bounded.run(evict=False)
    assert r["served"] == 2 and r["outcomes"][-1] == (2, 0, 60, 30)
    r = bounded.run()
    assert r["served"] == 7 and all(o[0] == 0 for o in r["outcomes"]) and not r["cache"].status.any().item()
    assert r["length"] == 161 and r["tokens"] == 70 * 16 + 1


def test_what_it_keeps_and_computes():
    import torch

    from paper_2605_24259_amd import bounded
    first, second = bounded.run(seed=3), bounded.run(seed=3)
    for k in ("out", "lse", "weight"):
        assert torch.equal(first[k][..., :161] if k == "weight" else first[k], second[k][..., :161] if k == "weight" else second[k])
    r, c, n = first, first["cache"], first["length"]
    # the first block and the last 32 tokens of the prompt are kept by every head
    pos = r["pos"][1, :, :n - 1].cpu().numpy()
    for p in pos:
        assert len(set(p)) == n - 1 and set(range(16)) <= set(p) and set(range(1120 - 32, 1120)) <= set(p)
        assert p[:16].tolist() == list(range(16))
    assert len({tuple(sorted(p)) for p in pos}) > 1  # heads choose for themselves
    # the resident claim's account was never touched by rows of its own, its slots neither moved
    assert r["weight"][0, :, : r["held"]].eq(0).all()

    # the decoded token and the drafted tree against 64 bits over the slots as they lie in the cache
    def slots(pool, head, m):
        t = c.block_table[1].cpu().long()
        j = np.arange(m)
        return pool.cpu()[t[j // 16], j % 16, head].double().numpy()

    def softmax(x):
        e = np.exp(x - x.max())
        return e / e.sum()
    # drafted slots behind the decoded one hold what the tree put there
    d = r["drafted"]
    base, parent = n - 1, d["parent"].tolist()
    lines = []
    for i, p in enumerate(parent):
        lines.append((lines[p] if p >= 0 else []) + [i])
    vmax = float(c.v.abs().max())
    for head in range(d["q"].shape[1]):
        k, v = slots(c.k, head // 4, d["length"]), slots(c.v, head // 4, d["length"])
        for i, line in enumerate(lines):
            at = list(range(base)) + [base + a for a in line]
            x = d["q"][i, head].double().cpu().numpy() @ k[at].T * r["scale"]
            want = softmax(r["softcap"] * np.tanh(x / r["softcap"])) @ v[at]
            # weights and outputs are rounded to bfloat16: 2^-8 of the largest value, twice, and 32-bit scores
            assert np.abs(d["out"][i, head].double().cpu().numpy() - want).max() <= 2.0 ** -7 * vmax
            if i == 0:
                assert np.abs(r["out"][0, head].double().cpu().numpy() - want).max() <= 2.0 ** -7 * vmax


def test_command(capsys):
    from paper_2605_24259_amd import bounded
    bounded.main()
    text = capsys.readouterr().out
    assert "whole: outcome 2 (claim 0: protected 60, required 70, usable 80)" in text and "7 chunks served" in text
