"""The example decoder (examples/serve_decoder.py), which runs all operators between the layer products as a server does: prompts at once or in pieces and single tokens
give the same log probabilities, and these are those of a decoder in 64 bits.

Tolerance: every activation is rounded to fp16 (2^-11) some ten times a block, and a key or value near a boundary between two codes of 4 bits may fall to either side, a
step of a third of the values' size in one of 64 terms of a score or one of many of an output: a few hundredths of the logits' unit size at two blocks.  0.15 for the largest of
some hundred tokens, 0.03 for their mean size."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import gpu_util as G
from oracle import dbf_oracle as O
from oracle import serve_oracle as S

pytestmark = pytest.mark.gpu
LARGEST, MEAN = 0.15, 0.03

_path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_decoder.py")
_spec = importlib.util.spec_from_file_location("serve_decoder", _path)
E = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(E)


def near(got, want, what):
    d = np.abs(got - want)
    G.say("%s: %d log probabilities, largest difference %.3g, mean %.3g" % (what, d.size, d.max(), d.mean()))
    assert d.max() <= LARGEST and d.mean() <= MEAN


def dense(L):
    return O.dense_weight(O.f16_bits_to_f64(L.a), O.unpack_signs(L.A_bits, L.n_out, L.k).astype(np.float64), O.f16_bits_to_f64(L.m),
                          O.unpack_signs(L.B_bits, L.k, L.n_in).astype(np.float64), O.f16_bits_to_f64(L.b))


def in_64_bits(d, text):
    """Log probabilities of a text's tokens but the first."""
    c = d.cfg
    f = lambda t: t.detach().cpu().double().numpy()   # noqa: E731
    x = f(d.embedding)[text]
    cos, sin = f(d.rope)[: len(text), : c.head_dim // 2], f(d.rope)[: len(text), c.head_dim // 2:]
    norm = lambda x, w: x / np.sqrt((x * x).mean(-1, keepdims=True) + c.eps) * f(w)   # noqa: E731
    for block, w in zip(d.inputs, d.norms):
        h = norm(x, w["in"])
        q, k, v = ((h @ dense(block[n]).T).reshape(len(text), -1, c.head_dim) for n in "qkv")
        q, k = (S.norm_rope(t, f(w[n]), c.eps, cos, sin, False) for t, n in ((q, "q"), (k, "k")))
        out, _, _ = S.attend(q, S.held(k), S.held(v), 1 / math.sqrt(c.head_dim), True)
        x = x + out.reshape(len(text), -1) @ dense(block["o"]).T
        h = norm(x, w["mlp"])
        g = h @ dense(block["gate"]).T
        x = x + (g / (1 + np.exp(-g)) * (h @ dense(block["up"]).T)) @ dense(block["down"]).T
    logits = norm(x, d.last_norm) @ dense(d.head_inputs).T
    return S.token_logprobs(logits[:-1], text[1:], 0)[0]


@pytest.fixture(scope="module")
def decoder():
    d = E.Decoder(E.Config(), seed=3)
    yield d
    d.close()


def test_texts_against_64_bits(decoder):
    rng = np.random.default_rng(5)
    texts = [[int(t) for t in rng.integers(0, decoder.cfg.vocab, n)] for n in (90, 2, 41)]
    decoder.free = list(range(decoder.cfg.pages))
    decoder.start(3)
    lp = decoder.forward(texts, [t[1:] + [-1] for t in texts])[0]
    for text, part in zip(texts, lp.split([len(t) for t in texts])):
        assert float(part[-1]) == 0.0
        near(part[:-1].cpu().double().numpy(), in_64_bits(decoder, text), "a text of %d tokens" % len(text))


def test_in_pieces_and_token_by_token(decoder):
    """The same texts at once, in two pieces that end anywhere in a page, and token by token from some place on; pages in another order."""
    rng = np.random.default_rng(6)
    texts = [[int(t) for t in rng.integers(0, decoder.cfg.vocab, n)] for n in (100, 77, 64, 33)]
    targets = [t[1:] + [-1] for t in texts]

    def run(cuts):
        decoder.free = [int(p) for p in rng.permutation(decoder.cfg.pages)]
        decoder.start(len(texts))
        out = [[] for _ in texts]
        for a, b in zip(cuts[:-1], cuts[1:]):
            new = [t[a:b] for t in texts]
            if not any(new):
                continue
            lp = decoder.forward(new, [t[a:b] for t in targets])[0].cpu().double().numpy()
            at = 0
            for i, piece in enumerate(new):
                out[i] += list(lp[at: at + len(piece)])
                at += len(piece)
        return np.concatenate([o[:-1] for o in out])

    whole = run([0, 100])
    near(run([0, 45, 100]), whole, "two pieces")
    near(run([0, 60] + list(range(61, 101))), whole, "token by token")


def test_a_full_cache_is_said_so(decoder):
    decoder.free = [0]
    decoder.start(1)
    with pytest.raises(RuntimeError):
        decoder.forward([[1] * 40], [[-1] * 40])
    decoder.free = list(range(decoder.cfg.pages))


def test_the_example_runs():
    E.main()
