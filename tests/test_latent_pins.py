"""The oracle of the latent calls, pinned on the CPU; geometry checks that need no device."""
import numpy as np
import pytest

from oracle import latent as ol

P = 16


def bf16(x):
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7fff + ((u >> 16) & 1)) & np.uint32(0xffff0000)).view(np.float32).astype(np.float64)


def cache(lens, seed):
    rng = np.random.default_rng(seed)
    need = [-(-n // P) for n in lens]
    perm = rng.permutation(sum(need) + 2)
    table, at = np.full((len(lens), max(need + [1])), -1), 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return bf16(rng.standard_normal((sum(need) + 2, P, ol.ROW))), table


def test_decode_by_hand():
    """Two tokens whose logits differ by ln 3: weights 1/4 and 3/4."""
    pages, table = cache([2], 1)
    pages[table[0, 0], :2, 512:] = 0
    pages[table[0, 0], 1, 512] = 1
    q = np.zeros((1, 1, 576))
    q[0, 0, 512] = 1
    c = pages[table[0, 0], :2, :512]
    out, lse, _, _ = ol.decode(q, pages, table, [2], np.log(3.0))
    assert np.allclose(out[0, 0], c[0] / 4 + 3 * c[1] / 4, atol=1e-13) and np.isclose(lse[0, 0], np.log(4.0))
    out, lse, _, _ = ol.decode(q, pages, table, [0], 1.0)
    assert not out.any() and np.isneginf(lse).all()


def test_decode_by_loops():
    lens = [1, 16, 19]
    pages, table = cache(lens, 2)
    q = np.random.default_rng(3).standard_normal((3, 2, 576))
    out, lse, _, _ = ol.decode(q, pages, table, lens, 0.1)
    for b, n in enumerate(lens):
        for h in range(2):
            s = [0.1 * sum(float(q[b, h, i]) * float(pages[table[b, t // P], t % P, i]) for i in range(576)) for t in range(n)]
            e = [np.exp(x) for x in s]
            want = sum(w * pages[table[b, t // P], t % P, :512] for t, w in enumerate(e)) / sum(e)
            assert np.allclose(out[b, h], want, atol=1e-12) and np.isclose(lse[b, h], np.log(sum(e)))


def test_absorbed_and_expanded_forms_agree():
    """q_nope . (W_k c) = (W_k^T q_nope) . c and sum p (W_v c) = W_v sum p c."""
    n, h = 21, 3
    pages, table = cache([n], 4)
    rng = np.random.default_rng(5)
    w = rng.standard_normal((h, 256, 512)) / 512 ** 0.5
    q = rng.standard_normal((1, h, 192))
    lo, k, v, _, _ = ol.expand(w, pages, table, [n])[0]
    assert lo == 0
    k_pages, v_pages = np.zeros((2, h, P, 128)), np.zeros((2, h, P, 128))
    for t in range(n):
        k_pages[t // P, :, t % P], v_pages[t // P, :, t % P] = k[t], v[t]
    out, lse, _, _ = ol.prefill(q, [0, 1], k_pages, v_pages, [[0, 1]], pages, table, [n], 0.07)
    absorbed = np.concatenate([np.einsum("hdl,bhd->bhl", w[:, :128], q[..., :128]), q[..., 128:]], -1)
    lat, lse2, _, _ = ol.decode(absorbed, pages, table, [n], 0.07)
    assert np.allclose(np.einsum("hdl,bhl->bhd", w[:, 128:], lat), out, atol=1e-12) and np.allclose(lse, lse2)


def test_prefill_is_causal():
    """Query i of the new tokens sees positions up to its own: the same as attending alone over the shorter context."""
    n, m, h = 40, 7, 2
    pages, table = cache([n], 6)
    rng = np.random.default_rng(7)
    k_pages, v_pages = rng.standard_normal((3, h, P, 128)), rng.standard_normal((3, h, P, 128))
    q = rng.standard_normal((m, h, 192))
    out, lse, _, _ = ol.prefill(q, [0, m], k_pages, v_pages, [[2, 0, 1]], pages, table, [n], 0.1)
    for i in range(m):
        a, b, _, _ = ol.prefill(q[i:i + 1], [0, 1], k_pages, v_pages, [[2, 0, 1]], pages, table, [n - m + 1 + i], 0.1)
        assert np.allclose(out[i], a[0], atol=1e-13) and np.allclose(lse[i], b[0])


def test_append_rows():
    rng = np.random.default_rng(8)
    x, weight = rng.standard_normal((3, 576)), rng.standard_normal(512)
    freq = 10000.0 ** (-np.arange(32) / 32.0)
    rows, _ = ol.append_rows(x, weight, 0.0, np.array([[0, 1, 5]]), freq, [0] * 32, 64, False)
    assert np.allclose((rows[:, :512] / weight) ** 2 @ np.ones(512), 512)          # unit root mean square
    assert np.allclose(rows[0, 512:], x[0, 512:])                                  # position 0 turns nothing
    assert np.allclose(np.hypot(rows[:, 512:544], rows[:, 544:]), np.hypot(x[:, 512:544], x[:, 544:]))
    assert np.allclose(rows[1, 512], x[1, 512] * np.cos(1) - x[1, 544] * np.sin(1))
    plain, _ = ol.append_rows(x, None, 0.0, np.array([[0, 1, 5]]), freq, [0] * 32, 64, False)
    assert np.array_equal(plain[:, :512], x[:, :512])


def test_rounded_weights_stay_inside_the_bound():
    """The bound against a computation with bf16 weights normalised by their own sum."""
    lens = [1, 5, 400]
    pages, table = cache(lens, 9)
    q = bf16(np.random.default_rng(10).standard_normal((3, 4, 576)))
    out, _, bound, _ = ol.decode(q, pages, table, lens, 0.07)
    for b, n in enumerate(lens):
        x = ol.rows_of(pages, table[b], n)
        z = 0.07 * (q[b] @ x.T)
        p = bf16(np.exp(z - z.max(-1, keepdims=True) + 1.7))
        got = bf16((p @ x[:, :512]) / p.sum(-1, keepdims=True))
        assert np.all(np.abs(got - out[b]) <= bound[b])


def test_geometry_of_a_latent_context():
    import paper_2609_35158_b200 as pd

    for args, code in (((129, 1, 512, 16, 4, 4, 16), pd.PD_ERR_UNSUPPORTED), ((64, 2, 512, 16, 4, 4, 16), pd.PD_ERR_UNSUPPORTED),
                       ((64, 1, 256, 16, 4, 4, 16), pd.PD_ERR_UNSUPPORTED), ((64, 1, 512, 32, 4, 4, 16), pd.PD_ERR_UNSUPPORTED),
                       ((0, 1, 512, 16, 4, 4, 16), pd.PD_ERR_INVALID_ARG), ((64, 1, 512, 16, 4, 4, 1 << 28), pd.PD_ERR_UNSUPPORTED),
                       ((64, 1, 512, 16, 5000, 4, 16), pd.PD_ERR_INVALID_ARG)):
        with pytest.raises(pd.PdError) as e:
            pd.pd_create(*args, 0, pd.PD_FLAG_LATENT)
        assert e.value.code == code
    with pytest.raises(pd.PdError) as e:                                           # without the flag the geometry stays unknown
        pd.pd_create(8, 1, 512, 16, 4, 4, 16)
    assert e.value.code == pd.PD_ERR_UNSUPPORTED
