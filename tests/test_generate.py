"""Generation operators without a GPU: the oracle against independent statements, the pages' byte
order, and what the binding refuses."""
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "tmz_pages.h"
// every byte of a page is one (token, dim), and lane l's e-th byte of a 16-byte piece is the value
// that the matrix instruction takes from it
template <int HD> int check() {
  int bad = 0;
  bool k[64 * HD] = {}, v[64 * HD] = {};
  for (int t = 0; t < 64; ++t)
    for (int d = 0; d < HD; ++d) {
      const int a = tmz::key_at<HD>(t, d), b = tmz::value_at(t, d);
      if (a < 0 || a >= 64 * HD || k[a]) { ++bad; continue; }
      if (b < 0 || b >= 64 * HD || v[b]) { ++bad; continue; }
      k[a] = v[b] = true;
      int piece = a / 1024, lane = a / 16 % 64, e = a % 16;
      bad += t != 32 * (piece / (HD / 32)) + 16 * (e / 8) + lane % 16;
      bad += d != 32 * (piece % (HD / 32)) + 8 * (lane / 16) + e % 8;
      piece = b / 1024; lane = b / 16 % 64; e = b % 16;
      bad += d != 16 * piece + lane % 16;
      bad += t != 32 * (e / 8) + 16 * (e % 8 / 4) + 4 * (lane / 16) + e % 4;
    }
  return bad;
}
int main() { std::printf("%d\n", check<64>() + check<96>() + check<128>()); return 0; }
"""


def test_page_byte_order(tmp_path):
    src = tmp_path / "pages.cpp"
    src.write_text(PROGRAM)
    exe = tmp_path / "pages"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2609_33548_amd", "csrc"),
                    str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.strip() == "0"


def test_oracle_quantiser_is_half_a_step_off_at_most(orc):
    from oracle import generate_ref as ref
    rng = np.random.default_rng(0)
    for scale in (1e-8, 1.0, 3e4):
        x = (rng.standard_normal((64, 96)) * scale).astype(np.float32)
        q, d = ref.quantise_block(x)
        assert np.abs(q).max() == 127
        # half a step, and the roundings of 1 / a, s, x s, 1 / 127 and d (5 of 2^-24 on |q| <= 127)
        assert np.abs(q * np.float64(d) - x).max() <= d * (0.5 + 127 * 5 * 2.0 ** -24)
    q, d = ref.quantise_block(np.zeros((64, 64), np.float32))
    assert not q.any() and d > 0
    x[5, 5] = np.inf
    assert np.isnan(ref.quantise_block(x)[1])


def test_oracle_cache_does_not_depend_on_the_split(orc):
    from oracle import generate_ref as ref
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((2, 150, 2, 64)).astype(np.float32)
    whole, parts = ref.Sequence(True, 10000.0), ref.Sequence(True, 10000.0)
    whole.append(k, v)
    for a, b in ((0, 1), (1, 64), (64, 65), (65, 150)):
        parts.append(k[a:b], v[a:b])
    for a, b in zip(whole.values(), parts.values()):
        assert np.array_equal(a, b)


def test_oracle_attention_against_torch(orc):
    """Against torch's own attention in fp64 on the cached values (tolerance: fp64 sums of 100 terms)."""
    import torch
    from oracle import generate_ref as ref
    rng = np.random.default_rng(2)
    s = ref.Sequence(False, 10000.0)
    s.append(*rng.standard_normal((2, 100, 2, 64)).astype(np.float32))
    q = rng.standard_normal((30, 6, 64)).astype(np.float32)
    out, mag, _ = ref.attend(s, q)
    k, v = (torch.from_numpy(x).double().repeat_interleave(3, 1).transpose(0, 1) for x in s.values())
    qr = torch.from_numpy(ref.rotate(q, np.arange(70, 100), 10000.0)).double().transpose(0, 1)
    mask = torch.ones(30, 100, dtype=torch.bool).tril(70)
    want = torch.nn.functional.scaled_dot_product_attention(qr[None], k[None], v[None], attn_mask=mask)[0]
    assert np.abs(out - want.transpose(0, 1).numpy()).max() < 1e-12
    assert (np.abs(out) <= mag * (1 + 1e-12)).all()


def test_oracle_beam_selection_against_a_full_sort(orc):
    from oracle import generate_ref as ref
    rng = np.random.default_rng(3)
    for W, V, n in ((1, 7, 7), (3, 50, 6), (4, 20, 64)):
        logits = rng.integers(-3, 4, (W, V)).astype(np.float32)       # many ties
        scores = rng.integers(-2, 1, W).astype(np.float32)
        got = ref.beam_select(logits, scores, n)
        every = []
        for b in range(W):
            lse = np.log(sum(np.exp(float(x)) for x in logits[b]))
            every += [(-(float(scores[b]) + float(logits[b, t]) - lse), b * V + t) for t in range(V)]
        every.sort()
        # equal scores of a beam are equal in both statements; across beams they differ in the last bits
        assert np.allclose(got[0], [-e[0] for e in every[:n]], rtol=0, atol=1e-12)
        for b in range(W):
            mine = [t for t, p in zip(got[1], got[2]) if p == b]
            order = sorted(range(V), key=lambda t: (-logits[b, t], t))
            assert mine == order[:len(mine)]


def test_oracle_beam_selection_of_empty_and_finished_beams(orc):
    from oracle import generate_ref as ref
    logits = np.zeros((3, 5), np.float32)
    logits[1] = -np.inf
    logits[2, 1:] = np.nan
    s, tok, par, done, hist = ref.beam_select(logits, np.float32([-1.0, 0.0, -9.0]), 8, eos=2,
                                              finished=[1, 0, 0], history=np.arange(6).reshape(3, 2))
    assert (par[0], tok[0], s[0], done[0]) == (0, 2, -1.0, True)      # finished: its score, unchanged
    assert (par[1], tok[1], s[1], done[1]) == (2, 0, -9.0, False)     # the only finite logit
    assert np.isneginf(s[2:]).all() and list(par[2:] * 5 + tok[2:]) == [0, 1, 3, 4, 5, 6]
    assert hist[1].tolist() == [4, 5, 0]


def test_binding_refuses_wrong_tensors():
    import torch
    from paper_2609_33548_amd import termezo as T
    dev = torch.device("cpu")
    x = torch.zeros(2, 3, 4)
    assert T._tensor(x, "x", (2, 3, 4), torch.float32, dev) == x.data_ptr()
    for bad in (x.double(), x[0], x.transpose(0, 1), x[:, :, :2], torch.zeros(2, 3, 5)):
        with pytest.raises(ValueError, match="x must be"):
            T._tensor(bad, "x", (2, 3, 4), torch.float32, dev)
    with pytest.raises(ValueError, match="cuda:0"):
        T._tensor(x, "x", (2, 3, 4), torch.float32, torch.device("cuda", 0))


def test_binding_refuses_integers_that_would_wrap():
    """A layer, group, size or token id beyond the C types must not arrive as another one."""
    import torch
    from paper_2609_33548_amd import termezo as T

    class Ctx:
        device, handle = torch.device("cpu"), None

        def _check(self, st, what):
            if st != T.OK:
                raise T.TermezoError(st, what)

    c = T.KVCache.__new__(T.KVCache)
    c.ctx, c.handle, c.dtype, c.groups, c.beams, c._width = Ctx(), None, torch.float32, 1, 1, 1
    c.n_heads, c.n_kv_heads, c.head_dim, c.max_len = 2, 2, 64, 8
    x = torch.zeros(1, 3, 2, 64)
    for big in (1 << 32, -(1 << 32), (1 << 31), (1 << 64) + 1):
        for f in (lambda: c.append(big, x, x), lambda: c.attention(big, x, x.clone()), lambda: c.read(big, 0, x),
                  lambda: c.reset(big), lambda: T.KVCache(Ctx(), big, 2, 2, 64, 8, 1),
                  lambda: T.KVCache(Ctx(), 1, 2, 2, 64, 8, big), lambda: T.KVCache(Ctx(), 1, 2, 2, 64, 8, 1, big),
                  lambda: T.KVCache(Ctx(), 1, big, 2, 64, 8, 1), lambda: T.KVCache(Ctx(), 1, 2, 2, big, 8, 1),
                  lambda: T.Context.beam_select(Ctx(), x, x[..., 0].contiguous(), x[:, :1, 0].contiguous(), None, None,
                                                eos=big)):
            with pytest.raises(ValueError, match="32 bits"):
                f()
    for big in (1 << 63, (1 << 64) + 5):
        for f in (lambda: c.read(0, big, x), lambda: T.KVCache(Ctx(), 1, 2, 2, 64, big, 1)):
            with pytest.raises(ValueError, match="64 bits"):
                f()
    with pytest.raises(T.TermezoError):                      # what fits goes on to the library
        c.append(-1, x, x)


def test_null_handles_are_rejected():
    from paper_2609_33548_amd import termezo as T
    import ctypes
    L, bad, out = T.lib, T.ERR_INVALID_ARG, ctypes.c_void_p(7)
    cfg = T.KVCacheConfig(1, 4, 4, 64, 1, 1, 64, 0.0, T.BF16)
    assert L.termezo_kvcache_create(None, ctypes.byref(cfg), ctypes.byref(out)) == bad
    assert out.value is None
    assert L.termezo_kvcache_create(None, None, None) == bad
    assert L.termezo_kvcache_reset(None, -1) == bad
    assert L.termezo_kvcache_fork(None) == bad
    assert L.termezo_kvcache_append(None, 0, None, None, 1, None) == bad
    assert L.termezo_kvcache_attention(None, 0, None, None, None, 1, None, None) == bad
    assert L.termezo_kvcache_advance(None) == bad
    assert L.termezo_kvcache_reorder(None, None) == bad
    assert L.termezo_kvcache_read(None, 0, 0, 1, None, None, 0) == bad
    assert L.termezo_kvcache_lengths(None, None) == bad
    assert L.termezo_logits(None, None, None, 0, 1, 16, 1, None) == bad
    assert L.termezo_beam_select(None, None, None, None, 1, 1, 1, 1, -1, None, None, None, None, None,
                                 None, 0) == bad
    assert L.termezo_model_decode(None, None, None, 1, None, None) == bad
    L.termezo_kvcache_destroy(None)
