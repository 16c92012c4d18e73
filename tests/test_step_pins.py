"""Pins of the oracle of the operators around the expert layer: worked cases,
identities, and gradients against differences."""
import numpy as np
import pytest

import oracle.foremoe_step as S

INF = np.inf


def test_router_worked_case():
    # exp of the logits: 1, 2, 4, 1 -> probabilities 1/8, 1/4, 1/2, 1/8
    l = np.log(np.array([[1.0, 2.0, 4.0, 1.0], [4.0, 4.0, 1.0, 1.0]]))
    r = S.router_forward(l, 2, renorm=False)
    assert r["ids"].tolist() == [[2, 1], [0, 1]]
    assert np.allclose(r["gates"], [[0.5, 0.25], [0.4, 0.4]])
    assert np.allclose(S.router_forward(l, 2, scale=3.0)["gates"], [[2.0, 1.0], [1.5, 1.5]])
    assert r["counts"].tolist() == [1, 2, 1, 0] and r["n_tokens"] == 2
    assert np.allclose(r["prob_mean"], [0.2625, 0.325, 0.3, 0.1125])
    assert np.isclose(r["balance_loss"], 4 * (0.25 * 0.2625 + 0.5 * 0.325 + 0.25 * 0.3))


def test_router_even_load_has_loss_one():
    l = np.zeros((4, 4))
    r = S.router_forward(l, 2, ids=np.array([[0, 1], [2, 3], [0, 2], [1, 3]]))
    assert np.isclose(r["balance_loss"], 1.0)


def test_router_empty_places():
    l = np.array([[0.0, -INF, 1.0], [-INF, -INF, -INF], [2.0, 1.0, 0.0]])
    r = S.router_forward(l, 3, mask=np.array([1, 1, 0]))
    assert r["ids"].tolist() == [[2, 0, -1], [-1, -1, -1], [-1, -1, -1]]
    assert r["n_tokens"] == 1 and np.all(r["gates"][1:] == 0)
    r = S.router_forward(l, 3, ids=np.array([[1, 2, 7], [0, 1, 2], [-1, 0, 0]]))
    assert r["ids"].tolist() == [[-1, 2, -1], [-1, -1, -1], [-1, 0, 0]]
    assert np.allclose(r["gates"], [[0, 1, 0], [0, 0, 0], [0, 0.5, 0.5]])


def test_router_bias_picks_but_does_not_weigh():
    l = np.array([[0.0, 0.1, 0.2]])
    bias = np.array([1.0, 0.0, 0.0])
    r = S.router_forward(l, 2, score="sigmoid", bias=bias, renorm=False)
    assert r["ids"].tolist() == [[0, 2]]
    assert np.allclose(r["gates"], 1 / (1 + np.exp(-np.array([[0.0, 0.2]]))))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_router_gradient_against_differences(score, renorm):
    rng = np.random.default_rng(5)
    T, E, K = 4, 6, 3
    l = rng.standard_normal((T, E))
    l[1, 2] = -INF
    mask = np.array([1, 1, 1, 0])
    dg = rng.standard_normal((T, K))
    coef = 0.7
    kw = dict(score=score, renorm=renorm, scale=1.3, mask=mask)
    r = S.router_forward(l, K, **kw)
    ids = r["ids"].copy()
    ids[2, 1] = ids[2, 0]  # an id twice in a row, as a record may have it
    r = S.router_forward(l, K, ids=ids, **kw)

    def f(x):
        q = S.router_forward(x, K, ids=ids, **kw)
        fr = r["counts"] / r["counts"].sum()  # the counts do not follow the logits
        return np.sum(q["gates"] * dg) + coef * E * np.sum(fr * q["prob_mean"])

    got = S.router_backward(l, ids, dg, counts=r["counts"], n_tokens=r["n_tokens"], balance_coef=coef, **kw)
    h = 1e-6
    for t in range(T):
        for e in range(E):
            if l[t, e] == -INF:
                assert got[t, e] == 0
                continue
            a, b = l.copy(), l.copy()
            a[t, e] += h
            b[t, e] -= h
            assert abs((f(a) - f(b)) / (2 * h) - got[t, e]) < 1e-7


def test_logprobs_worked_case():
    l = np.log(np.array([[1.0, 2.0, 1.0], [1.0, 1.0, 1.0], [3.0, 2.0, 1.0]]))
    l = np.concatenate([l, [[-INF] * 3]])
    r = S.token_logprobs(l, np.array([1, 0, -1, 2]), n_top=2)
    assert np.allclose(r["logp"][:3], [np.log(0.5), -np.log(3), 0]) and r["logp"][3] == -INF
    assert np.allclose(r["entropy"], [1.5 * np.log(2), np.log(3), 0, 0])
    assert r["top_ids"].tolist() == [[1, 0], [0, 1], [-1, -1], [-1, -1]]
    # temperature 0.5 squares the odds
    r = S.token_logprobs(l[:1], np.array([1]), temperature=0.5)
    assert np.isclose(r["logp"][0], np.log(4 / 6))


@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_logprobs_gradient_against_differences(temperature):
    rng = np.random.default_rng(6)
    N, V = 3, 7
    l = rng.standard_normal((N, V)) * 2
    l[0, 3] = -INF
    t = np.array([2, 5, -1])
    a, b = rng.standard_normal(N), rng.standard_normal(N)
    got = S.token_logprobs_backward(l, t, a, b, temperature=temperature)

    def f(x):
        r = S.token_logprobs(x, t, temperature=temperature)
        return np.sum(r["logp"] * a) + np.sum(r["entropy"] * b)

    h = 1e-6
    for i in range(N):
        for j in range(V):
            if l[i, j] == -INF:
                assert got[i, j] == 0
                continue
            p, q = l.copy(), l.copy()
            p[i, j] += h
            q[i, j] -= h
            assert abs((f(p) - f(q)) / (2 * h) - got[i, j]) < 1e-7


def test_adamw_first_step_moves_by_lr():
    # at step 1 the corrected moments are g and g^2: the move is lr g / (|g| + eps)
    g = np.array([2.0, -3.0, 0.0])
    p, m, v = S.adamw_step(np.ones(3), g, np.zeros(3), np.zeros(3), lr=0.1, beta1=0.9, beta2=0.95, eps=0.0 + 1e-12,
                           weight_decay=0.5, step=1)
    assert np.allclose(p, 0.95 - 0.1 * np.sign(g))
    assert np.allclose(m, 0.1 * g) and np.allclose(v, 0.05 * g * g)


def test_state_codes_are_float_patterns():
    # the same codes from the bits of the fp32 pattern, rounded to even
    for bits, codes, table, one in ((3, 128, S.TABLE_M, 127), (4, 256, S.TABLE_V, 255)):
        shift = 23 - bits
        assert table[one] == 1.0 and table[0] == 0.0 and np.all(np.diff(table) > 0)
        for c in (1, 2, one // 2, one - 1, one):
            pattern = np.array([(c + (0x3F800000 >> shift) - one) << shift], dtype=np.int32).view(np.float32)
            assert pattern[0] == table[c]
        # halfway between two codes, and one step beside it
        lo, hi = table[one // 2].astype(np.float32), table[one // 2 + 1].astype(np.float32)
        mid = np.float32((float(lo) + float(hi)) / 2)
        for x in (mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(1))):
            b = int(np.array([x]).view(np.int32)[0])
            want = ((b + (1 << (shift - 1)) - 1 + ((b >> shift) & 1)) >> shift) - ((0x3F800000 >> shift) - one)
            assert S._nearest(np.array([float(x)]), table)[0] == want


def test_state_round_trip_is_within_half_a_step():
    rng = np.random.default_rng(7)
    m = (rng.standard_normal(700) * np.exp(rng.uniform(-8, 0, 700))).astype(np.float32)
    v = (m * m).astype(np.float32)
    c, s = S.encode_m(m)
    assert s.shape == (3,) and np.all(np.abs(S.decode_m(c, s) - m) <= np.abs(m) / 16 + 2e-5 * np.repeat(s, 256)[:700])
    c, s = S.encode_v(v)
    assert np.all(np.abs(np.sqrt(S.decode_v(c, s)) - np.abs(m)) <= np.abs(m) / 32 * 1.001 + 2e-5 * np.repeat(s, 256)[:700])
    # a v above zero never becomes zero, zero stays zero
    v = np.zeros(256, dtype=np.float32)
    v[0], v[1] = 1.0, 1e-30
    c, s = S.encode_v(v)
    assert c[0] == 255 and c[1] == 1 and np.all(c[2:] == 0)
