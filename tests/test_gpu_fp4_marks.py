"""Where the keys of a long prefix go when several waves and blocks share them:
attention over a 4-bit store whose answer is known exactly and hangs on single
slots.  No rotation (all frequencies zero) and a softmax scale of ln 2, so that a
logit in log2 units is q . k itself.

Counts: with q = 0 every weight is 1, the normaliser is the number of keys, an
integer below 2^24 and so exact in fp32, and the log-sum-exp its logarithm: one
step of the logarithm, the products' two roundings, 2^-22 of it, taken as 2^-21.
A slot left out or taken twice moves it by 1 / n.  Values that are 1 in one dim a
chunk and 0 elsewhere, held exactly, count each dim's slots: sums exact, the
division 2^-23 (taken as 2^-20), the output's rounding 2^-8 (half a step of
bf16).

Marks: keys are zero but for marked slots, each 6 in a dim of its own; a row's
query holds two marked dims, so that its logits are x and y at these slots, 0
elsewhere, all exact in bf16 (weights powers of two).  A row is then
(sum of v + (2^x - 1) v_a + (2^y - 1) v_b) / (n + 2^x + 2^y - 2): terms and
weights exact, fp32 sums of n terms in any order off by less than n 2^-24 of the
sum of their magnitudes, the output's rounding 2^-8; the log-sum-exp's parts
round as above, and its reference's product with ln 2: 2^-20 beside the sum's n
2^-24."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda"


def _D():
    import paper_2609_03311_amd as D
    return D


class Long:
    """A store of two documents, the second of `slots`, and pairs of `tokens`
    on it."""

    def __init__(self, slots, hkv, d, rep, tokens, seed=0):
        D = _D()
        self.slots, self.hkv, self.d, self.rep = slots, hkv, d, rep
        self.tokens, self.hq, self.n = tokens, hkv * rep, len(tokens)
        self.gen = torch.Generator().manual_seed(seed)
        self.lens = [45, slots]
        self.at = torch.tensor([0, 45, 45 + slots], device=DEV)
        self.store = D.dopr_store_create(1, hkv, d,
                                         np.asarray(self.lens, np.int32),
                                         format=D.DOPR_STORE_FP4)
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(tokens)]),
                               dtype=torch.int32)
        self.total = int(self.cu[-1])
        # the document's slots and, behind them, the tokens' own
        self.k = torch.zeros((slots, hkv, d))
        self.v = torch.zeros((slots, hkv, d))
        self.own_k = torch.zeros((self.total, hkv, d))
        self.own_v = torch.zeros((self.total, hkv, d))

    def put(self):
        D = _D()
        other = torch.full((45, self.hkv, self.d), 6.0)
        D.dopr_store_put(self.store, 0,
                         torch.tensor([0, 1], dtype=torch.int32, device=DEV),
                         self.at,
                         *(torch.cat((other, x)).to(DEV, torch.bfloat16)
                           for x in (self.k, self.v)))

    def call(self, q, variant=0):
        D = _D()
        shape = dict(max_tokens=max(self.tokens), total_tokens=self.total)
        need = D.dopr_prefix_attn_workspace(
            self.store, n_pairs=self.n, n_q_heads=self.hq,
            kernel_variant=variant, **shape)
        ws = torch.full((max(need, 256),), 255, dtype=torch.uint8, device=DEV)
        out = torch.full((self.total, self.hq, self.d), float("nan"),
                         dtype=torch.bfloat16, device=DEV)
        lse = torch.full((self.total, self.hq), float("nan"), device=DEV)
        D.dopr_prefix_attn(
            self.store, 0, torch.ones(self.n, dtype=torch.int32, device=DEV),
            self.cu.to(DEV), *(x.to(DEV, torch.bfloat16) for x in
                               (q, self.own_k, self.own_v)), None, None, out,
            ws, lse=lse, softmax_scale=math.log(2.0), kernel_variant=variant,
            rope_inv_freq=torch.zeros(self.d // 2, device=DEV), **shape)
        assert D.dopr_check_status(self.store) == D.DOPR_OK
        return out.cpu().double(), lse.cpu().double()

    def places(self):
        """(first token, token, number of keys) of every row."""
        for p in range(self.n):
            a = int(self.cu[p])
            for j in range(self.tokens[p]):
                yield a, j, self.slots + j + 1


# (kv heads, q heads each, tokens of the pairs)  A few units are shared by blocks
# of four waves, more by one of four, of two, and many are one wave's: single
# tokens, and several
SHAPES = [(1, 1, [1]), (2, 3, [1, 1]), (1, 4, [1] * 40), (2, 2, [1] * 300),
          (4, 2, [1] * 500), (1, 8, [3]), (2, 5, [2, 17]),
          (1, 3, [40, 3] * 6), (2, 4, [30] * 40), (2, 8, [30] * 60),
          (4, 8, [30] * 40)]
LENGTHS = [1, 33, 1023, 1024, 1025, 2047, 2049, 3000, 4096, 4097, 6016, 6017,
           20001, 20033, 70001]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("variant", [0, 8, 6])
def test_every_key_counts_once(d, shape, variant):
    """Variants 8 and 6: the planned kernels, whose batches hold up to seven of
    a 4-bit store's chunks, or none."""
    hkv, rep, tokens = SHAPES[shape]
    for slots in LENGTHS if len(tokens) < 40 else LENGTHS[:-3]:
        r = Long(slots, hkv, d, rep, tokens)
        chunk = torch.arange(slots) // 32
        r.v[torch.arange(slots), :, chunk % d] = 1.0
        for a, j, _ in r.places():
            r.own_v[a + j, :, (7 * j) % d] = 1.0
        r.put()
        out, lse = r.call(torch.zeros(r.total, r.hq, d), variant)
        prefix = torch.bincount(chunk % d, minlength=d).double()
        own = torch.zeros(max(tokens), d).double()
        own[torch.arange(max(tokens)), 7 * torch.arange(max(tokens)) % d] = 1
        own = own.cumsum(0)
        for a, j, n in r.places():
            want = (prefix + own[j]) / n
            got = out[a + j]
            assert ((got - want).abs() <= (2.0 ** -8 + 2.0 ** -20)
                    * want).all(), (slots, j)
            log = math.log(n)
            assert ((lse[a + j] - log).abs() <= 2.0 ** -21 * log).all(), (
                slots, j, (lse[a + j] - log).abs().max())


def _borders(slots, share):
    """The first and last slots of a part of the chunks, `share` of them or the
    document's ends and a few between."""
    chunks = (slots + 31) // 32
    starts = np.unique(np.linspace(0, chunks - 1, share).astype(int))
    first = 32 * starts
    last = np.minimum(first + 31, slots - 1)
    return np.unique(np.concatenate([first, last, [0, slots - 1]]))


def _marked(r, x, drop, seed):
    """Marks r's borders in turn, as many a call as it has dims and rows for."""
    D, d = _D(), r.d
    rng = np.random.default_rng(seed)
    last = max(r.tokens)
    room = min(d - last, r.rep * sum(r.tokens))
    r.v = torch.randint(-4, 5, r.v.shape, generator=r.gen).float()
    r.v[::32] = -6.0  # (so that the others are held as they are)
    r.own_v = torch.randint(-4, 5, r.own_v.shape, generator=r.gen).float()
    # own keys: token j of a pair in dim d - 1 - j
    for a, j, _ in r.places():
        r.own_k[a + j, :, d - 1 - j] = 6.0
    todo = _borders(r.slots, 40)
    rows = list(r.places())
    sums = r.v.double().sum(0), r.v.double().abs().sum(0)
    for at in range(0, len(todo), room):
        marks = todo[at:at + room]
        r.k.zero_()
        for i, s in enumerate(marks):
            r.k[s, :, i] = 6.0
        r.put()
        q = torch.zeros(r.total, r.hq, d)
        plan = {}
        turn = 0
        for a, j, n in rows:
            for h in range(r.hq):
                i = turn % len(marks)
                turn += 1
                # the other: another mark, or a key of its own up to itself
                own = rng.random() < 0.3
                o = int(rng.integers(j + 1)) if own else int(
                    rng.integers(len(marks)))
                if not own and o == i:
                    own, o = True, j
                lower = drop * int(rng.integers(4)) / 6
                top, low = (x / 6, x / 6 - lower)
                if rng.random() < 0.5:
                    top, low = low, top
                q[a + j, h, i] = top
                q[a + j, h, d - 1 - o if own else o] = low
                plan[a + j, h] = (i, own, o, 6 * top, 6 * low)
        out, lse = r.call(q)
        for a, j, n in rows:
            own_v = r.own_v[a:a + j + 1].double()
            seen, size = sums[0] + own_v.sum(0), sums[1] + own_v.abs().sum(0)
            for h in range(r.hq):
                i, own, o, u, w = plan[a + j, h]
                g = h // r.rep
                va = r.v[marks[i], g].double()
                vb = (r.own_v[a + o, g] if own else r.v[marks[o], g]).double()
                fa, fb = 2.0 ** u - 1, 2.0 ** w - 1
                total = n + fa + fb
                want = (seen[g] + fa * va + fb * vb) / total
                slack = 2.0 ** -24 * n * (
                    size[g] + fa * va.abs() + fb * vb.abs()) / total
                off = (out[a + j, h] - want).abs()
                assert (off <= 2.0 ** -8 * want.abs() + slack).all(), (
                    r.slots, int(marks[i]), own, o, u, w, off.max())
                log = math.log(total)
                assert abs(lse[a + j, h] - log) <= (2.0 ** -20 * log
                                                    + 2.0 ** -24 * n), (
                    r.slots, int(marks[i]), lse[a + j, h], log)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hkv,rep,tokens", [
    (1, 30, [1]), (2, 16, [1, 1]), (1, 60, [1] * 6), (1, 10, [3]),
    (2, 4, [2, 17])])
@pytest.mark.parametrize("x", [12, 36, 72])
def test_marked_slots_are_found(d, hkv, rep, tokens, x):
    """x: weights of 2^12 among the others, of 2^36, and over the bound of the
    softmax without a reference."""
    for slots in (1025, 2047, 4097, 6017, 20001):
        _marked(Long(slots, hkv, d, rep, tokens, seed=slots), x, 3, slots)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hkv,rep,tokens", [(1, 16, [1]), (2, 6, [3])])
@pytest.mark.parametrize("gain", [0.5, 2.0])
def test_marked_slots_with_qk_norm(d, hkv, rep, tokens, gain):
    """Two marked slots of equal logits, 18 (natural log units) above the rest:
    half of each value, however q^ was rounded.  The rest has at most n e^-17.8
    (2^-8 of 18 for that rounding) of twice the largest magnitude, 6.  Gains of
    the keys inside and outside the range without a reference."""
    D = _D()
    for slots in (1025, 4097, 20001):
        r = Long(slots, hkv, d, rep, tokens, seed=slots)
        r.v = torch.randint(-4, 5, r.v.shape, generator=r.gen).float()
        r.v[::32] = -6.0
        todo = _borders(slots, 30)
        for at in range(0, len(todo) - 1, d):
            marks = todo[at:at + d]
            r.k.zero_()
            for i, s in enumerate(marks):
                r.k[s, :, i] = 6.0
            r.put()
            q = torch.zeros(r.total, r.hq, d)
            pick = {}
            turn = 0
            for a, j, _ in r.places():
                for h in range(r.hq):
                    i, o = turn % len(marks), (turn + 5) % len(marks)
                    turn += 1
                    q[a + j, h, i] = q[a + j, h, o] = 1.0
                    pick[a + j, h] = (i, o)
            ones = torch.ones(d, dtype=torch.bfloat16, device=DEV)
            kw = gain * ones
            shape = dict(max_tokens=max(tokens), total_tokens=r.total)
            ws = torch.full((max(256, D.dopr_prefix_attn_workspace(
                r.store, n_pairs=r.n, n_q_heads=r.hq, **shape)),), 255,
                dtype=torch.uint8, device=DEV)
            out = torch.full((r.total, r.hq, d), float("nan"),
                             dtype=torch.bfloat16, device=DEV)
            # q^ is sqrt(d / 2) at a marked dim: logits of 18 and 0 at this
            # scale.  (Own keys are zeros, normed: zeros.)
            D.dopr_prefix_attn(
                r.store, 0, torch.ones(r.n, dtype=torch.int32, device=DEV),
                r.cu.to(DEV), *(x.to(DEV, torch.bfloat16) for x in
                                (q, r.own_k, r.own_v)), ones, kw, out, ws,
                softmax_scale=3 / (d / 2) ** 0.5,
                rope_inv_freq=torch.zeros(d // 2, device=DEV), **shape)
            assert D.dopr_check_status(r.store) == D.DOPR_OK
            out = out.cpu().double()
            for (t, h), (i, o) in pick.items():
                g = h // rep
                # (a single mark left: both of its dims are one)
                want = (r.v[marks[i], g] + r.v[marks[o], g]).double() / 2
                rest = 12 * (slots + 3) * math.exp(-17.8)
                assert ((out[t, h] - want).abs() <= 2.0 ** -8 * want.abs()
                        + rest).all(), (slots, t, h)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("pairs", [300, 600])
def test_many_single_tokens_against_64_bits(d, pairs):
    """Units of two waves, and of one: the rows of some of the pairs."""
    from test_gpu_fp4_token import Tokens
    docs = [p % 6 for p in range(pairs)]
    for norm in (True, False):
        t = Tokens([0, 33, 64, 257, -1, 700], docs, 8, 4, d, norm=norm,
                   seed=pairs, freq=norm)
        t.check(*t.call(), pairs=range(0, pairs, 35))
        assert _D().dopr_check_status(t.store) == _D().DOPR_ERR_DOC_RANGE
