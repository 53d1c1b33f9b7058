"""The decoder in small numbers (cmt_quant_beam_decode) against a search in 64 bits with the same numbers: the weights that the 4-bit codes
stand for, keys and source states rounded to the 8-bit codes' values.

What the two may differ by: sums in fp32 (1e-5 of a score here), and a code of a key or state whose quotient lies within fp32's
rounding of the border between two falls either way.  With weights of +-0.1 and 64 units one such code moves the attentional
layer's sums by at most 0.1 / 127 and a score by some 0.1 * 8 * 0.1 / 127 = 6e-4; 16-bit operands round every state by 2^-9 of it
(8 roundings of 64 terms of 0.1: 0.1 * 8 * 2^-9 = 2e-3 a layer and position).  Scores are held to LOOSE, ten times that; tokens where no decision was
closer than twice LOOSE."""
import numpy as np
import pytest

from oracle import nmt_oracle as O
from paper_1802_07170_amd import binding, inputs as I
from tests.test_decoding_ops import MAGNITUDES, plain_cache, plain_pack

pytestmark = pytest.mark.gpu

LOOSE = {0: 6e-3, 1: 6e-2}


def in_four_bits(w, group):
    code, scale = plain_pack(np.asarray(w, np.float32), group)
    return MAGNITUDES[code] * np.repeat(scale.astype(np.float64), group, 1)[:, :w.shape[1]]


class Sentence:
    """One sentence's encoder, and the decoder's log-probabilities position by position, for any number of hypotheses."""

    def __init__(self, cfg, params, src):
        self.p = p = {k: np.asarray(v, np.float64) for k, v in params.items()}
        H, self.L, Hd, n = cfg["hidden"], cfg["layers"], cfg["hidden"] // 2, len(src)
        x, one, zd, zh = p["E_src"][src][:, None], np.ones((n, 1)), np.zeros((1, Hd)), np.zeros((1, H))
        f, hf, cf, _ = O.lstm_forward(x, one, p["enc.l0.fwd.W"], p["enc.l0.fwd.b"], zd, zd)
        g, hg, cg, _ = O.lstm_forward(x, one, p["enc.l0.bwd.W"], p["enc.l0.bwd.b"], zd, zd, reverse=True)
        y, self.h, self.c = np.concatenate([f, g], 2), [np.concatenate([hf, hg], 1)], [np.concatenate([cf, cg], 1)]
        for l in range(1, self.L):
            y, hl, cl, _ = O.lstm_forward(y, one, p[f"enc.l{l}.W"], p[f"enc.l{l}.b"], zh, zh)
            self.h.append(hl)
            self.c.append(cl)
        states = y[:, 0]
        held = lambda rows: plain_cache(rows.astype(np.float32)[None, :, None], [n])[0, :, 0].astype(np.float64)
        self.keys, self.values, self.ho = held(states @ p["W_a"]), held(states), zh

    def advance(self, prev):
        p = self.p
        x = np.concatenate([p["E_tgt"][prev], self.ho], 1)
        for l in range(self.L):
            _, self.h[l], self.c[l], _ = O.masked_step_forward(x, self.h[l], self.c[l], np.ones((len(prev), 1)), p[f"dec.l{l}.W"], p[f"dec.l{l}.b"])
            x = self.h[l]
        s = x @ self.keys.T
        a = np.exp(s - s.max(1, keepdims=True))
        self.ho = np.tanh(np.concatenate([a / a.sum(1, keepdims=True) @ self.values, x], 1) @ p["W_c"].T)
        z = self.ho @ p["W_o"].T + p["B_o"]
        z = z - z.max(1, keepdims=True)
        return z - np.log(np.exp(z).sum(1, keepdims=True))

    def keep(self, rows):
        self.h, self.c, self.ho = [v[rows] for v in self.h], [v[rows] for v in self.c], self.ho[rows]


def score_of(cfg, params, src, tokens, alpha, bos=2):
    sentence, total = Sentence(cfg, params, src), 0.0
    for prev, tok in zip([bos, *tokens], tokens):
        total += sentence.advance(np.array([prev]))[0, tok]
    return total / O.length_penalty(len(tokens), alpha)


def search(cfg, params, src, max_len, beam, alpha, bos=2, eos=3):
    """Tokens, normalised score and the smallest gap at a decision."""
    sentence, live, score, prev, done, gap = Sentence(cfg, params, src), [[]], np.zeros(1), np.array([bos]), [], np.inf
    for j in range(max_len):
        logp = sentence.advance(prev)
        total, V, keep = (score[:, None] + logp).ravel(), logp.shape[1], []
        order = np.argsort(-total, kind="stable")
        if len(order) > beam:                                # (the order of those that are kept decides nothing)
            gap = min(gap, total[order[beam - 1]] - total[order[beam]])
        for i in order[:beam]:
            row, tok = divmod(int(i), V)
            if tok == eos or j == max_len - 1:
                done.append((total[i] / O.length_penalty(j + 1, alpha), live[row] + [tok]))
            else:
                keep.append((row, tok, total[i]))
        if not keep:
            break
        live = [live[r] + [t] for r, t, _ in keep]
        score, prev = np.array([v for _, _, v in keep]), np.array([t for _, t, _ in keep])
        sentence.keep([r for r, _, _ in keep])
    ends = sorted((v for v, _ in done), reverse=True)
    if len(ends) > 1:
        gap = min(gap, ends[0] - ends[1])
    best = max(range(len(done)), key=lambda i: (done[i][0], -i))
    return done[best][1], done[best][0], gap


def network(cfg, seed):
    params = I.make_params(cfg, seed)
    rng = np.random.default_rng(seed)
    for k in ("E_src", "E_tgt"):
        params[k] = params[k] * 10
    params["B_o"] = rng.normal(0, 1.0, params["B_o"].shape).astype(np.float32)
    return params


@pytest.mark.parametrize("H,E,L,V,lens,beam,alpha,group", [
    (64, 32, 1, 104, [1, 7, 12], 1, 0.0, 32), (64, 64, 2, 200, [5, 33, 18, 9], 4, 0.6, 64), (48, 40, 3, 304, [20, 1, 65], 10, 0.6, 128),
    (80, 24, 2, 104, [130, 3], 16, 1.0, 64), (112, 64, 4, 504, [9, 11, 30, 2, 17], 3, 0.6, 32)])
@pytest.mark.parametrize("prec", [0, 1])
def test_search_in_small_numbers(H, E, L, V, lens, beam, alpha, group, prec):
    from paper_1802_07170_amd.decoding import QuantDecoder
    cfg = dict(src_vocab=V, tgt_vocab=V, emb=E, hidden=H, layers=L)
    params = network(cfg, H + L)
    rng = np.random.default_rng(H)
    B, S, T = len(lens), max(lens), 9
    src = rng.integers(4, V, (B, S)).astype(np.int32)
    src_len = np.array(lens, np.int32)
    rounded = dict(params, **{k: in_four_bits(params[k], group) for k in params if k.startswith("dec.") and k.endswith(".W") or k in ("W_c", "W_o")})
    want = [search(cfg, rounded, src[b, :n], T, beam, alpha) for b, n in enumerate(lens)]
    tr = binding.Trainer(cfg, max(16, B * beam), S + 3, T + 2, precision=prec)
    try:
        tr.set_params(I.flatten(params, cfg))
        qd = QuantDecoder(tr, group)
        ids, length, score = qd.beam_decode(src, src_len, T, beam=beam, length_penalty=alpha)
        again = qd.beam_decode(src, src_len, T, beam=beam, length_penalty=alpha)
        assert all(np.array_equal(a, b) for a, b in zip((ids, length, score), again))
        for b, (tokens, value, gap) in enumerate(want):
            got = ids[b, :length[b]].tolist()
            assert (ids[b, length[b]:] == 0).all() and 1 <= length[b] <= T and (3 in got[-1:] or length[b] == T) and 3 not in got[:-1]
            assert abs(score[b] - score_of(cfg, rounded, src[b, :lens[b]], got, alpha)) <= LOOSE[prec], b     # of what came out, whatever it is
            if gap > 2 * LOOSE[prec]:
                assert got == tokens and abs(score[b] - value) <= LOOSE[prec], b
        # the ordinary decoders are as before, and the packed weights follow the parameters when asked to
        if beam == 1:
            assert np.array_equal(qd.greedy_decode(src, src_len, T)[0], ids)
        before = tr.beam_decode(src, src_len, T, beam=beam, length_penalty=alpha)
        qd.beam_decode(src, src_len, T, beam=beam, length_penalty=alpha)
        assert all(np.array_equal(a, b) for a, b in zip(before, tr.beam_decode(src, src_len, T, beam=beam, length_penalty=alpha)))
        tr.init_params(3, 0.1)
        assert np.array_equal(qd.beam_decode(src, src_len, T, beam=beam, length_penalty=alpha)[0].shape, ids.shape)
        tr.set_params(I.flatten(params, cfg))
        qd.pack()
        assert np.array_equal(qd.beam_decode(src, src_len, T, beam=beam, length_penalty=alpha)[2], score)
    finally:
        tr.close()


def test_training_goes_on_beside_it():
    """A step, a search in small numbers, the same step: the same gradients; and sentences by themselves score as they do in a batch."""
    from paper_1802_07170_amd.decoding import QuantDecoder
    c = I.CONFIGS["tiny"]
    cfg = I.model_cfg(c)
    batch = I.make_batch(c)
    tr = binding.Trainer(cfg, 40, 12, 12, precision=1)
    try:
        tr.set_params(I.flatten(network(cfg, 5), cfg))
        dev = tr.upload_batch(*batch)
        loss = tr.train_step(dev)
        grads = tr.get_grads()
        qd = QuantDecoder(tr)
        ids, length, score = qd.beam_decode(batch[0], batch[1], 10, beam=5)
        assert tr.train_step(dev) == loss and np.array_equal(tr.get_grads(), grads)
        one = [qd.beam_decode(batch[0][b:b + 1], batch[1][b:b + 1], 10, beam=5) for b in range(8)]
        assert np.allclose([o[2][0] for o in one], score, atol=LOOSE[1])
    finally:
        tr.close()


def test_refusals():
    from paper_1802_07170_amd.decoding import QuantDecoder
    cfg = dict(src_vocab=104, tgt_vocab=104, emb=16, hidden=32, layers=1)
    tr = binding.Trainer(cfg, 8, 6, 6, precision=0)
    try:
        tr.init_params(1, 0.1)
        with pytest.raises(binding.CmtError):
            QuantDecoder(tr, 48)
        qd = QuantDecoder(tr, 32)
        src, n = np.full((2, 6), 5, np.int32), np.array([6, 3], np.int32)
        for kw in (dict(beam=17), dict(beam=5), dict(beam=0), dict(length_penalty=-1.0), dict(eos_id=104)):
            with pytest.raises(binding.CmtError):
                qd.beam_decode(src, n, 6, **{**dict(beam=2), **kw})
        for bad in ((src[:, :0], n, 6), (src, n, 0), (src, n, 7)):
            with pytest.raises(binding.CmtError):
                qd.beam_decode(*bad, beam=2)
        with pytest.raises(binding.CmtError, match="vocabulary"):
            qd.beam_decode(np.full((2, 6), 104, np.int32), n, 6, beam=2)
        with pytest.raises(binding.CmtError, match="length"):
            qd.beam_decode(src, np.array([7, 3], np.int32), 6, beam=2)
        assert qd.beam_decode(src, n, 6, beam=4)[0].shape == (2, 6)
    finally:
        tr.close()


@pytest.mark.parametrize("precision", [0, 1])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_many_rows_score_as_few(precision, group):
    """1664 rows take another kernel for the layers' products than 128 do: a sentence scores the same."""
    from paper_1802_07170_amd.decoding import QuantDecoder
    c = I.CONFIGS["tiny"]
    cfg = dict(I.model_cfg(c), hidden=512, layers=2)
    src, n = I.make_batch(c)[:2]
    tr = binding.Trainer(cfg, 1664, src.shape[1], 8, precision=precision)
    try:
        tr.init_params(3, 0.1)
        qd = QuantDecoder(tr, group)
        few = qd.beam_decode(src[:8], n[:8], 6, beam=16)[2]
        many = qd.beam_decode(np.tile(src[:8], (13, 1)), np.tile(n[:8], 13), 6, beam=16)[2]
        assert np.allclose(many, np.tile(few, 13), atol=LOOSE[precision])
    finally:
        tr.close()


def test_lengths_of_another_batch_are_refused():
    from paper_1802_07170_amd.decoding import QuantDecoder
    cfg = dict(src_vocab=104, tgt_vocab=104, emb=16, hidden=32, layers=1)
    tr = binding.Trainer(cfg, 8, 6, 6, precision=0)
    try:
        tr.init_params(1, 0.1)
        qd = QuantDecoder(tr, 32)
        for src, n in ((np.full((2, 6), 5), [6]), (np.full((2, 6), 5), [6, 6, 6]), (np.full(6, 5), [6])):
            with pytest.raises(ValueError):
                qd.beam_decode(np.array(src, np.int32), np.array(n, np.int32), 6, beam=2)
    finally:
        tr.close()
