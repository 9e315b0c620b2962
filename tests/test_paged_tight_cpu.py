"""The bounds of paged_tight.py hold what they are for: results with a token lost, a
page in another's place, or operands of fewer bits fall outside them."""
import numpy as np
import pytest

import paged_ref as ref
import paged_tight as tight


def cut(x, bits):
    """x rounded to so many bits of mantissa."""
    m, e = np.frexp(x.astype(np.float64))
    return np.ldexp(np.round(m * 2.0 ** bits), e - bits)


def as_type(x, kind):
    return cut(x, 8 if kind == "bf16" else 24)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("n,d,page", [(300, 32, 16), (41595, 128, 16), (90000, 64, 64),
                                      (128000, 128, 64)])
def test_marked_tokens_show_every_mistake(n, d, page, kind):
    rng = np.random.default_rng(n)
    N = 60
    K, V = tight.marked_inputs(rng, N, 1, page, d)
    table = rng.integers(0, N, ref.pages(n, page))
    j = np.arange(n)
    for trial in range(6):
        channel = rng.integers(0, d, 1)

        def result(tokens, table=table):
            O, LSE = tight.marked(K, V, table[tokens // page], tokens % page, 0, channel)
            return as_type(O, kind), as_type(LSE, "f32")

        want = tight.marked(K, V, table[j // page], j % page, 0, channel)
        assert not tight.marked_off(*result(j), *want, kind).any()
        first = int(rng.integers(0, n - 64))
        seen = K[table[first // page], 0, first % page, channel[0]] == 0
        for lost in (1, page, 32, 64):
            gone = np.delete(j, slice(first, first + lost))
            assert lost == 1 and not seen or tight.marked_off(*result(gone), *want, kind).all()
        twice = np.insert(j, first, j[first:first + 32])
        assert tight.marked_off(*result(twice), *want, kind).all()
        wrong = table.copy()
        at = int(rng.integers(0, len(table) - 1))
        wrong[at] = (wrong[at] + 1) % N
        assert tight.marked_off(*result(j, wrong), *want, kind).all()


@pytest.mark.parametrize("n,d,bits", [(40, 32, 13), (256, 64, 13), (700, 128, 13), (2000, 128, 12)])
def test_weighted_tokens_show_lost_bits(n, d, bits):
    """f32 operands of fewer bits, bf16 probabilities of 8, in most of single rows."""
    rng = np.random.default_rng(n + d)
    scale = d ** -0.5
    caught = {"q": 0, "k": 0, "v": 0, "p": 0}
    for trial in range(8):
        k, v = (cut(rng.standard_normal((n, d)) * np.exp(0.5 * rng.standard_normal(d)) +
                    0.5 * rng.standard_normal(d), 8) for _ in range(2))
        q = cut(rng.standard_normal(d), 8)
        want = tight.weighted(q, k, v, scale, "bf16")
        assert not tight.weighted_off(as_type(want[0], "bf16"), as_type(want[1], "f32"), want, "bf16")
        s = scale * (k @ q)
        p = np.exp(s - s.max())
        O = as_type(cut(p, 8) @ v / p.sum(), "bf16")
        caught["p"] += tight.weighted_off(O, want[1], want, "bf16")
        k, v, q = (x + 0.01 * rng.standard_normal(x.shape) for x in (k, v, q))
        want = tight.weighted(q, k, v, scale, "f32")
        assert not tight.weighted_off(as_type(want[0], "f32"), as_type(want[1], "f32"), want, "f32")
        for what in "qkv":
            low = {"q": q, "k": k, "v": v, what: cut({"q": q, "k": k, "v": v}[what], bits)}
            O, LSE, *_ = tight.weighted(low["q"], low["k"], low["v"], scale, "f32")
            caught[what] += tight.weighted_off(O, LSE, want, "f32")
    assert min(caught.values()) > 4, caught
