"""Products with 8-bit weights, rules on the logits and the draw, without a GPU: the oracle against independent
statements, and what the binding and the library refuse before a device is touched."""
import ctypes

import numpy as np
import pytest

F = np.float32


def test_oracle_codes_are_half_a_step_off_at_most():
    from oracle import next_token_ref as ref
    rng = np.random.default_rng(0)
    for scale in (1e-20, 1.0, 3e30):
        x = (rng.standard_normal(640) * scale).astype(F)
        q, d = ref.quantise(x, 1e-30)
        assert np.abs(q).max() == 127
        # half a step, and the roundings of 1 / a, s, x s and a / 127 on |q| <= 127 (1 / a may be denormal, off by 2^-20)
        assert np.abs(q * np.float64(d) - x).max() <= d * (0.5 + 127 * (4 * 2.0 ** -24 + (2.0 ** -20 if scale > 1 else 0)))
    assert not ref.quantise(np.zeros(16, F), 1e-5)[0].any()
    assert np.isnan(ref.quantise(np.array([1, np.inf], F), 1e-5)[1])


def test_oracle_products_of_python_integers():
    from oracle import next_token_ref as ref
    rng = np.random.default_rng(2)
    x = (rng.standard_normal((3, 48)) * 10.0 ** rng.integers(-3, 4, (3, 1))).astype(F)
    x[1] = 0.0
    codes = rng.integers(-128, 128, (5, 48)).astype(np.int8)
    steps = rng.random(5).astype(F)
    got = ref.linear(x, codes, steps)
    for m in range(3):
        q, d = ref.quantise(x[m], 1e-5)
        for n in range(5):
            total = sum(int(a) * int(b) for a, b in zip(q, codes[n]))
            assert got[m, n] == total * float(d) * float(steps[n])


def test_oracle_rules_token_by_token():
    """Against a statement in Python numbers, a token at a time (fp32 values whose results are exact)."""
    from oracle import next_token_ref as ref
    x = np.array([2.0, -2.0, 0.0, 8.0, -8.0, 1.0, 4.0, np.nan], F)
    h = [0, 1, 3, 3, 9, -1, 4, 3]
    got = ref.adjust(x, h, start=3, repetition=2.0, presence=0.5, frequency=0.25,
                     bias=np.array([0, 0, 0, 1, 0, 0, -4, 0], F), allowed=np.array([1, 1, 1, 1, 1, 0, 1, 0], bool))
    want = [1.0, -4.0, 0.0, 4.0 - 2 * 0.25 - 0.5 + 1, -16.0 - 0.25 - 0.5, -np.inf, 0.0, -np.inf]
    assert got.tolist() == want


def test_oracle_draw_against_enumeration():
    """Shares of an enumeration over a fine grid of u equal the kept weights' shares; kept tokens equal those of a
    statement that walks the sorted tokens."""
    from oracle import next_token_ref as ref
    rng = np.random.default_rng(1)
    for k, p, mp, T in ((0, 1.0, 0.0, 1.0), (3, 1.0, 0.0, 0.7), (0, 0.6, 0.0, 1.3), (5, 0.8, 0.1, 1.0), (0, 0.0, 0.0, 1.0)):
        x = rng.integers(-4, 5, 12).astype(F) / 2                     # with ties
        w = [float(np.exp((float(v) - float(x.max())) / T)) for v in x]
        mine = []
        order = sorted(range(12), key=lambda t: (-x[t], t))
        first = [t for i, t in enumerate(order) if (k == 0 or i < k) and (w[t] >= mp or i == 0)]
        total, s = sum(w[t] for t in first), 0.0
        for t in first:
            if mine and s >= p * total:
                break
            mine.append(t)
            s += w[t]
        got, gw, _ = ref.kept(x, T, k, p, mp)
        assert got.tolist() == mine and np.allclose(gw, w, rtol=1e-15)
        n = 20000
        drawn = np.bincount([ref.sample(x, (i + 0.5) / n, temperature=T, top_k=k, top_p=p, min_p=mp)[0] for i in range(n)],
                            minlength=12) / n
        share = np.zeros(12)
        share[mine] = np.array([w[t] for t in mine]) / s
        assert np.abs(drawn - share).max() <= 1.0 / n
    assert ref.sample(np.full(4, -np.inf, F), 0.3)[0] == -1
    assert ref.sample(np.array([1, 5, 5, 2], F), 0.9, temperature=0)[:2] == (1, 0.0)


def test_null_handles_are_rejected():
    from paper_2609_33548_amd import termezo as T
    L, bad = T.lib, T.ERR_INVALID_ARG
    rules = T.LogitRules()
    assert L.termezo_quantize_rows(None, None, 0, 1, 16, None, None) == bad
    assert L.termezo_linear_i8(None, None, 0, 1, 16, None, None, 1, None, 0) == bad
    assert L.termezo_adjust_logits(None, None, 1, 1, ctypes.byref(rules), None) == bad
    assert L.termezo_sample(None, None, None, 1, 1, None, None, None, None, None, None) == bad
    assert L.termezo_model_set_head(None, None, None) == bad


def test_binding_refuses_wrong_tensors_and_incomplete_rules():
    import torch
    from paper_2609_33548_amd import termezo as T

    class Ctx:
        device, handle = torch.device("cpu"), None

        def _check(self, st, what):
            if st != T.OK:
                raise T.TermezoError(st, what)

    c, z = Ctx(), torch.zeros
    i32, i8 = torch.int32, torch.int8
    x, o, h = z(2, 40), z(2, 40), z(2, 5, dtype=i32)
    for kw in (dict(lengths=z(2, dtype=i32)), dict(repetition=z(2)), dict(starts=z(2, dtype=i32)),
               dict(mask_index=z(2, dtype=i32)), dict(bias_index=z(2, dtype=i32)), dict(history=h, lengths=z(2)),
               dict(history=h, presence=z(3)), dict(history=z(3, 5, dtype=i32)), dict(bias=z(1, 39)),
               dict(mask=z(1, 1, dtype=i32)), dict(mask=z(1, 2)), dict(history=h.long())):
        with pytest.raises(ValueError):
            T.Context.adjust_logits(c, x, o, **kw)
    with pytest.raises(ValueError):
        T.Context.adjust_logits(c, x, o.double())
    with pytest.raises(ValueError):
        T.Context.adjust_logits(c, x[:, :30], o[:, :30])
    u, t = z(2), z(2, dtype=i32)
    for args, kw in (((x, z(3), t), {}), ((x, u, t.long()), {}), ((x.double(), u, t), {}), ((x, u, t), dict(top_k=z(2))),
                     ((x, u, t), dict(top_p=z(1))), ((x, u, t), dict(logprobs=z(2, 1))),
                     ((x, u, t), dict(temperature=z(2).double()))):
        with pytest.raises(ValueError):
            T.Context.sample(c, *args, **kw)
    codes, steps = z(3, 32, dtype=i8), z(3)
    for args in ((z(2, 16), codes, steps, z(2, 3)), (z(2, 32), codes.int(), steps, z(2, 3)),
                 (z(2, 32), codes, z(4), z(2, 3)), (z(2, 32), codes, steps, z(3, 2)),
                 (z(64, 2).t(), codes, steps, z(2, 3)), (z(2, 32), codes, steps.double(), z(2, 3))):
        with pytest.raises(ValueError):
            T.Context.linear_i8(c, *args)
    with pytest.raises(TypeError):
        T.Context.linear_i8(c, z(2, 32).half(), codes, steps, z(2, 3))
    with pytest.raises(ValueError):
        T.Context.quantize_rows(c, z(3, 32), z(3, 16, dtype=i8), steps)
    # what fits goes on to the library
    for f in (lambda: T.Context.adjust_logits(c, x, o, history=h), lambda: T.Context.sample(c, x, u, t),
              lambda: T.Context.linear_i8(c, z(2, 32), codes, steps, z(2, 3)),
              lambda: T.Context.quantize_rows(c, z(3, 32), codes, steps)):
        with pytest.raises(T.TermezoError):
            f()


def test_sizes_beyond_the_c_types_are_refused():
    """Sizes that ctypes would wrap around: 2^32 + 9 logits are not 9."""
    import torch
    from paper_2609_33548_amd import termezo as T

    class Ctx:
        device, handle = torch.device("meta"), None

        def _check(self, st, what):
            raise AssertionError("reached the library")

    c, far = Ctx(), (1 << 32) + 9
    z = lambda *s, dt=torch.float32: torch.empty(s, dtype=dt, device="meta")
    i32 = torch.int32
    for R, V in ((1, far), (far, 1), (1, (1 << 31) + 1), ((1 << 31) + 1, 1)):
        with pytest.raises(ValueError):
            T.Context.sample(c, z(R, V), z(R), z(R, dt=i32))
        with pytest.raises(ValueError):
            T.Context.adjust_logits(c, z(R, V), z(R, V))
    for kw in (dict(bias=z(far, 2), bias_index=z(3, dt=i32)), dict(mask=z(far, 1, dt=i32), mask_index=z(3, dt=i32))):
        with pytest.raises(ValueError):
            T.Context.adjust_logits(c, z(3, 2), z(3, 2), **kw)
    for B, W, V, n in ((1, 1, far, 1), (far, 1, 1, 1), (1, far, 1, 1), (1, 1, 2, far)):
        with pytest.raises(ValueError):
            T.Context.beam_select(c, z(B, W, V), z(B, W), z(B, n), z(B, n, dt=i32), z(B, n, dt=i32))
