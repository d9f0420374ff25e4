"""The 8-bit key/value cache: store and eviction bit for bit against the one right answer in 64 bits, attention over it within
the bounds of the kernels' roundings (tests/exact_reference.py), and all of it together as a serving loop uses it."""
import math

import numpy as np
import pytest
import torch

import paper_2507_02957_amd as csat
from tests import exact_reference as ref
from tests.gpu_harness import DEV, tdtype, to_np
from tests.test_gpu_exact_attention import dev_ints, offsets

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


class Serving:
    """A pool with sequences in it: B rows of a page table in no order, codes and scales of earlier use in every slot."""

    def __init__(self, B, Hq, Hkv, d, page, max_pages, dtype, seed=0, spare=2, tables=1):
        g = np.random.default_rng(seed)
        self.B, self.Hq, self.Hkv, self.d, self.page, self.dtype, self.max_pages = B, Hq, Hkv, d, page, dtype, max_pages
        self.pages = B * max_pages * tables + spare
        shape = (self.pages, Hkv, page, d)
        self.K, self.V = (torch.from_numpy((100 * g.standard_normal(shape)).astype(np.float32)).clamp(-448, 448).to(F8) for _ in "KV")
        self.K, self.V = self.K.to(DEV), self.V.to(DEV).transpose(2, 3).contiguous()
        self.Ks, self.Vs = (torch.from_numpy(2.0 ** g.integers(-8, -5, shape[:2])).float().to(DEV) for _ in "KV")
        order = g.permutation(self.pages)[:B * max_pages * tables].reshape(tables, B, max_pages)
        self.tables = [dev_ints(t.tolist()) for t in order]
        self.lengths = [dev_ints([0] * B) for _ in range(tables)]
        self.scale = 1.0 / math.sqrt(d)
        self.g = g

    def cache(self, i=0, max_len=None):
        return csat.make_cache(self.K, self.V, self.Ks, self.Vs, self.tables[i], self.lengths[i], max_len)

    def reference(self):
        return ref.Cache(self.K.double().cpu().numpy(), self.V.double().cpu().numpy().swapaxes(2, 3), to_np(self.Ks), to_np(self.Vs))

    def same_as(self, r):
        for name in "KV":
            x = getattr(self, name).double().cpu().numpy()
            x = x if name == "K" else x.swapaxes(2, 3)
            ref.check(name, x, r.x[name], 0.0)
            ref.check(name + "s", to_np(getattr(self, name + "s")), r.s[name], 0.0)

    def rows(self, n, heads, spread=1.0):
        x = torch.from_numpy((spread * self.g.standard_normal((n, heads, self.d))).astype(np.float32))
        return x.to(tdtype(self.dtype)).to(DEV)

    def dims(self, n_q, n_k, max_q, max_k, causal=True, **t):
        return csat.make_packed_dims(self.B, self.Hq, self.Hkv, self.d, max(n_q, 1), max(n_k, 1), max(max_q, 1), max(max_k, 1), self.dtype, causal, **t)

    def store(self, lens, K=None, V=None, i=0, spread=1.0, reference=None):
        """Lengths grow by lens; the new rows, packed behind two rows of nobody."""
        off = offsets(lens, 2)
        n = off[-1] + 1
        K = self.rows(n, self.Hkv, spread) if K is None else K
        V = self.rows(n, self.Hkv, spread) if V is None else V
        before = self.lengths[i].tolist()
        self.lengths[i] += dev_ints(lens)
        csat.csat_cache_store(self.dims(1, n, 1, max(lens), K=K, V=V), self.cache(i), K, V, dev_ints(off))
        torch.cuda.synchronize()
        if reference is not None:
            t = self.tables[i].tolist()
            for b in range(self.B):
                for name, x in (("K", K), ("V", V)):
                    reference.store(name, t[b], before[b], to_np(x[off[b]:off[b + 1]]).reshape(-1, self.Hkv, self.d))
        return K, V

    def attend(self, q_lens, i=0, causal=True, W=None, decay=0.0, max_len=None, Q=None):
        off = offsets(q_lens, 1)
        n = off[-1] + 2
        Q = self.rows(n, self.Hq, 2.0) if Q is None else Q
        O = torch.full((n, self.Hq, self.d), 7.0, dtype=tdtype(self.dtype), device=DEV)
        lse = torch.full((self.Hq, n), 7.0, device=DEV)
        d, c = self.dims(n, 1, max(q_lens), 1, causal, Q=Q, O=O), self.cache(i, max_len)
        ws = torch.full((csat.csat_cache_workspace_bytes(d, c),), 255, dtype=torch.uint8, device=DEV)
        csat.csat_cache_attention(d, c, Q, dev_ints(off), self.scale, decay, O, lse, W, ws)
        torch.cuda.synchronize()
        return Q, O, lse, off

    def check_attention(self, r, Q, O, lse, off, i=0, causal=True, W=None, W_before=None, decay=0.0):
        t, lens, G = self.tables[i].tolist(), self.lengths[i].tolist(), self.Hq // self.Hkv
        O, lse, Qn = to_np(O), to_np(lse), to_np(Q)
        untouched = np.ones(O.shape[0], dtype=bool)
        for b in range(self.B):
            q0, q1, L = off[b], off[b + 1], lens[b]
            untouched[q0:q1] = False
            for h in range(self.Hkv):
                K, V = r.tokens("K", t[b], L, h), r.tokens("V", t[b], L, h)
                total, bound = np.zeros(L), np.zeros(L)
                for a in range(h * G, h * G + G):
                    o, l, p, do, dl, dp = ref.attend(Qn[q0:q1, a], K, V, ref.limits(q1 - q0, L, causal), self.scale, self.dtype)
                    ref.check(f"O[{b}, {a}]", O[q0:q1, a], o, do)
                    ref.check(f"lse[{b}, {a}]", lse[a, q0:q1], l, dl)
                    total += p.sum(0)
                    bound += dp.sum(0)
                if W is not None:
                    was = W_before[b, h, :L] * decay if decay else 0.0
                    ref.check(f"W[{b}, {h}]", to_np(W[b, h, :L]), was + total, bound + 2.0 ** -22 * (np.abs(was) + total))
                    ref.check("W behind", to_np(W[b, h, L:]), W_before[b, h, L:], 0.0)
        assert (O[untouched] == 7.0).all() and (lse[:, untouched] == 7.0).all()

    def weights(self, fill=0.0, i=0):
        return torch.full((self.B, self.Hkv, self.max_pages * self.page), fill, device=DEV)


STORES = [
    # page, d, Hkv, dtype, new tokens per sequence, call by call
    (16, 16, 1, "bf16", [[1], [1], [14], [1], [40]]),
    (64, 128, 2, "bf16", [[70, 0, 3], [1, 1, 1], [0, 64, 0], [1, 0, 61], [1, 1, 1]]),
    (32, 80, 3, "f32", [[33, 5], [1, 27], [30, 1], [1, 1]]),
    (128, 256, 1, "f32", [[1, 300], [200, 1], [1, 1]]),
    (128, 96, 2, "bf16", [[127, 129], [1, 1], [130, 2]]),
]


@pytest.mark.parametrize("case", range(len(STORES)))
def test_store(case):
    """Blocks filled at once and a token at a time, with tokens that make a block's scale grow; slots behind the last token and
    pages of nobody keep their bits."""
    page, d, Hkv, dtype, calls = STORES[case]
    s = Serving(len(calls[0]), Hkv, Hkv, d, page, -(-max(sum(c[b] for c in calls) for b in range(len(calls[0]))) // page) + 1, dtype, seed=case)
    r = s.reference()
    for spread, lens in zip((1.0, 30.0, 0.01, 1000.0, 1e6), calls):
        s.store(lens, spread=spread, reference=r)
        s.same_as(r)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_store_of_every_magnitude(dtype):
    """Values at and next to the middles between two codes, zeros of both signs, subnormal codes, infinities and NaN, blocks of
    zeros, the smallest and largest scales."""
    s = Serving(1, 1, 1, 256, 16, 8, dtype)
    r = s.reference()
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(F8).double()
    x = torch.zeros(2 + 16 * 7 + 1, 1, 256, dtype=torch.float64)
    x[2:18, 0] = codes
    mid = (codes[:126] + codes[1:127]) / 2
    x[18:34, 0, :126], x[18:34, 0, 126:252] = mid, -mid
    if dtype == "f32":
        x[18:26, 0, :126] *= 1 + 2.0 ** -23
        x[26:34, 0, :126] *= 1 - 2.0 ** -23
    x[34, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, 3.0])
    x[50:66, 0] = -0.0
    x[66:82, 0] = 3e-38 * torch.randn(16, 256, dtype=torch.float64)
    x[82:98, 0, 0] = 3.3e38
    x[98, 0, :2] = torch.tensor([448.0, 449.0])
    x = x.to(torch.float32).to(tdtype(dtype)).to(DEV)
    s.store([16 * 7], x, x.flip(-1).contiguous(), reference=r)
    s.same_as(r)
    assert s.Ks[s.tables[0][0, 3], 0].item() == 2.0 ** -118


ATTENDS = [
    # page, d, Hq, Hkv, dtype, lengths, rows, causal
    (64, 128, 8, 2, "bf16", [1, 63, 64, 65], [1, 1, 1, 1], True),
    (16, 64, 3, 3, "bf16", [200, 0, 17], [1, 1, 1], True),
    (32, 80, 7, 1, "f32", [100, 129], [1, 1], True),
    (128, 256, 4, 2, "f32", [300, 5], [1, 2], True),
    (64, 128, 16, 2, "bf16", [130, 40, 3], [8, 1, 5], True),      # several new tokens, more of them than there are
    (64, 96, 40, 1, "bf16", [90, 260], [3, 0], False),             # 120 rows to a key head
    (16, 16, 2, 1, "f32", [33, 50], [4, 2], False),
]


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("case", range(len(ATTENDS)))
def test_attention(case, weights):
    page, d, Hq, Hkv, dtype, lens, rows, causal = ATTENDS[case]
    s = Serving(len(lens), Hq, Hkv, d, page, -(-max(lens) // page) + 1, dtype, seed=case)
    s.lengths[0] += dev_ints(lens)
    W = s.weights(float("nan")) if weights else None                       # decay 0: not read
    got = s.attend(rows, causal=causal, W=W)
    before = np.full(s.weights().shape, np.nan)
    s.check_attention(s.reference(), *got, causal=causal, W=W, W_before=before)
    if weights:
        for decay in (1.0, 0.5):
            before = to_np(torch.nan_to_num(W, nan=3.0))
            W = torch.nan_to_num(W, nan=3.0)
            got = s.attend(rows, causal=causal, W=W, decay=decay)
            s.check_attention(s.reference(), *got, causal=causal, W=W, W_before=before, decay=decay)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_in_shares(dtype):
    """Long sequences of few heads, next to a short and an empty one, with and without weights."""
    s = Serving(3, 4, 1, 64, 64, 80, dtype)
    s.lengths[0] += dev_ints([5000, 0, 100])
    r = s.reference()
    got = s.attend([1, 1, 1])
    assert csat.csat_profile_launch_form("key_shares") > 1
    s.check_attention(r, *got)
    W = s.weights(0.0)
    again = s.attend([1, 1, 1], W=W, Q=got[0])
    assert torch.equal(got[1], again[1]) and torch.equal(got[2], again[2])
    s.check_attention(r, *again, W=W, W_before=np.zeros(W.shape))
    few = s.attend([1, 1, 1], max_len=5000, Q=got[0])
    s.check_attention(r, *few)


def test_attention_in_many_shares():
    """More shares than a wavefront has lanes, with weights, next to a sequence of one token."""
    s = Serving(2, 2, 1, 16, 128, 330, "bf16")
    s.lengths[0] += dev_ints([42000, 1])
    W = s.weights(2.0)
    got = s.attend([2, 1], W=W, decay=0.5)
    assert csat.csat_profile_launch_form("key_shares") > 64
    s.check_attention(s.reference(), *got, W=W, W_before=np.full(W.shape, 2.0), decay=0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_codes(dtype):
    """NaN codes behind the last token and in tokens that a row does not see have no effect; a row that sees one is NaN there."""
    s = Serving(2, 4, 2, 64, 32, 4, dtype)
    s.lengths[0] += dev_ints([70, 39])
    got = s.attend([4, 4])
    t = s.tables[0].tolist()
    K, V = s.K.view(torch.uint8), s.V.view(torch.uint8)
    K[t[0][2], :, 6:], V[t[0][2], :, :, 6:] = 0x7f, 0xff
    K[t[1][1], :, 7:], V[t[1][1], :, :, 7:] = 0xff, 0x7f
    K[t[1][2]], V[t[1][2]] = 0x7f, 0x7f
    again = s.attend([4, 4], Q=got[0])
    assert torch.equal(got[1], again[1]) and torch.equal(got[2], again[2])
    V[t[0][2], 0, 5, 4] = 0x7f                  # the second to last token: seen by the last two rows
    V[t[1][0], 1, 9, 3] = 0xff                  # seen by all
    K[t[1][1], 0, 6] = 0x7f                     # the last token's key: the last row
    again = s.attend([4, 4], Q=got[0])
    s.check_attention(s.reference(), *again)


def _poisoned(s, O, lse, off, b):
    assert torch.isnan(O[off[b]:off[b + 1]]).all() and torch.isnan(lse[:, off[b]:off[b + 1]]).all()


def test_bad_pages_and_lengths():
    """What only the device sees: the sequence concerned is NaN, is not stored to and not evicted; the others are right."""
    for bad in ("page", "low", "length", "negative"):
        s = Serving(3, 2, 1, 32, 16, 6, "bf16", tables=2)
        s.lengths[0] += dev_ints([50, 40, 60])
        if bad in ("page", "low"):
            s.tables[0][1, 1] = s.pages if bad == "page" else -1
        else:
            s.lengths[0][1] = 97 if bad == "length" else -3
        s.tables[0][0, 4:] = 1 << 30             # (not needed: not read)
        W = s.weights(1.0)
        Q, O, lse, off = s.attend([1, 2, 1], W=W)
        _poisoned(s, O, lse, off, 1)
        keep = [0, 2]
        r = s.reference()
        good = Serving.__new__(Serving)
        good.__dict__.update(s.__dict__)
        good.B, good.tables, good.lengths = 1, [None], [None]
        for b in keep:
            good.tables[0], good.lengths[0] = s.tables[0][b:b + 1], s.lengths[0][b:b + 1]
            o, l = torch.full_like(O, 7.0), torch.full_like(lse, 7.0)
            o[off[b]:off[b + 1]], l[:, off[b]:off[b + 1]] = O[off[b]:off[b + 1]], lse[:, off[b]:off[b + 1]]
            good.check_attention(r, Q, o, l, [off[b], off[b + 1]])
        # eviction
        kept = torch.zeros(3, 1, 30, dtype=torch.int32, device=DEV)
        W, W_to = torch.rand(s.weights().shape, device=DEV), s.weights(5.0)
        before = s.reference()
        csat.csat_cache_evict(s.dims(1, 1, 1, 1), s.cache(0), s.cache(1), W, W_to, 30, 3, kept)
        torch.cuda.synchronize()
        assert s.lengths[1].tolist() == [30, -1, 30]
        assert (kept[1] == -1).all() and (W_to[1] == 5.0).all() and (kept[0] >= 0).all()
        after = s.reference()
        for p in s.tables[1][1].tolist():
            assert np.array_equal(before.x["K"][p], after.x["K"][p]) and np.array_equal(before.s["V"][p], after.s["V"][p])
        Q, O, lse, off = s.attend([1, 1, 1], i=1)
        _poisoned(s, O, lse, off, 1)
        assert torch.isfinite(O[off[0]:off[1]].float()).all()
        # store: two more tokens each
        r = s.reference()
        if bad in ("page", "low"):
            s.lengths[0][1] = 20                 # (the new tokens' page is the bad one)
        lens = s.lengths[0].tolist()
        K = s.rows(6, 1)
        s.lengths[0][0] += 2
        s.lengths[0][2] += 2
        csat.csat_cache_store(s.dims(1, 6, 1, 2, K=K, V=K), s.cache(0), K, K, dev_ints([0, 2, 4, 6]))
        torch.cuda.synchronize()
        t = s.tables[0].tolist()
        for b in keep:
            for name in "KV":
                r.store(name, t[b], lens[b], to_np(K[2 * b:2 * b + 2]))
        s.same_as(r)


def evict_and_check(s, W, budget, recent):
    before = s.reference()
    n = min(budget, s.max_pages * s.page)
    W_to, kept = s.weights(5.0), torch.full((s.B, s.Hkv, budget), 9, dtype=torch.int32, device=DEV)
    csat.csat_cache_evict(s.dims(1, 1, 1, 1), s.cache(0), s.cache(1), W, W_to, budget, recent, kept)
    torch.cuda.synchronize()
    t, to, lens, P = s.tables[0].tolist(), s.tables[1].tolist(), s.lengths[0].tolist(), s.page
    want = s.reference()
    want.x, want.s = {k: v.copy() for k, v in before.x.items()}, {k: v.copy() for k, v in before.s.items()}
    assert s.lengths[1].tolist() == [min(x, budget) for x in lens]
    Wn, W_ton, keptn = to_np(W), to_np(W_to), kept.cpu().numpy()
    for b in range(s.B):
        for h in range(s.Hkv):
            at = ref.keep(Wn[b, h, :lens[b]].tolist(), budget, recent)
            assert keptn[b, h].tolist() == at + [-1] * (budget - len(at)), (b, h)
            ref.check("W_to", W_ton[b, h], np.concatenate([Wn[b, h, at], np.full(W_ton.shape[2] - len(at), 5.0)]), 0.0)
            for name in "KV":
                rows = before.tokens(name, t[b], lens[b], h)[at]
                for j in range(-(-len(at) // P)):
                    part = rows[j * P:(j + 1) * P]
                    want.s[name][to[b][j], h] = ref.block_scale(part)
                    want.x[name][to[b][j], h, :len(part)] = ref.e4m3(part / want.s[name][to[b][j], h])
    s.same_as(want)
    return W_to, n


@pytest.mark.parametrize("page,d,Hkv,lens,budget,recent", [
    (16, 16, 1, [1, 0, 40], 1, 0), (16, 16, 1, [1, 5, 40], 1, 1), (64, 128, 2, [300, 129], 128, 17), (32, 80, 3, [100, 64, 33], 64, 64),
    (128, 96, 1, [500, 130], 131, 0), (64, 64, 2, [70, 20], 500, 30), (16, 256, 1, [2000], 1500, 100)])
def test_eviction(page, d, Hkv, lens, budget, recent):
    s = Serving(len(lens), Hkv, Hkv, d, page, max(-(-max(lens) // page), -(-budget // page)), "bf16", tables=2)
    s.lengths[0] += dev_ints(lens)
    s.Ks *= torch.exp2(torch.randint(-12, 12, s.Ks.shape, device=DEV).float())
    W = torch.exp(3 * torch.randn(s.weights().shape, device=DEV))
    evict_and_check(s, W, budget, recent)


@pytest.mark.parametrize("levels", [0, 7])
def test_eviction_of_long_sequences(levels):
    """Longer than the selection holds in registers; weights of their own and ones with many ties."""
    s = Serving(2, 1, 1, 16, 128, 160, "bf16", tables=2)
    s.lengths[0] += dev_ints([20000, 8193])
    W = torch.exp(3 * torch.randn(s.weights().shape, device=DEV)) if levels == 0 else torch.randint(0, levels, s.weights().shape, device=DEV).float()
    evict_and_check(s, W, 8191, 100)


@pytest.mark.parametrize("kind", ["zeros", "equal", "few", "odd", "close"])
def test_eviction_of_equal_and_odd_weights(kind):
    """Ties go to the lowest slot, -0 is 0, NaN counts as the largest, infinities and negative weights have their place."""
    s = Serving(2, 2, 2, 16, 16, 130, "bf16", tables=2)
    s.lengths[0] += dev_ints([2000, 777])
    W = torch.zeros_like(s.weights())
    if kind == "equal":
        W += 0.25
    elif kind == "few":
        W += torch.randint(0, 3, W.shape, device=DEV) * 0.5
        W[:, :, ::7] = -0.0
    elif kind == "odd":
        W += torch.randn(W.shape, device=DEV)
        for i, x in enumerate((math.nan, math.inf, -math.inf, -math.nan, 1e-44, -1e-44)):
            W[:, :, i::97] = x
    elif kind == "close":
        W += 1.0 + torch.randint(0, 40, W.shape, device=DEV) * 2.0 ** -23
    s.K.view(torch.uint8)[:, :, 3, 5] = 0x7f            # NaN codes stay NaN and do not count for a scale
    evict_and_check(s, W, 700, 50)


def test_far_pages():
    """Pages whose byte offsets pass 32 bits, in a pool of over 4 GB each of K and V."""
    Hkv, page, d = 8, 128, 256
    s = Serving(1, Hkv, Hkv, d, page, 2, "bf16", tables=2)
    small, lens = s.reference(), [200]
    s.lengths[0] += dev_ints(lens)
    got = s.attend([1])
    pages = (1 << 32) // (Hkv * page * d) + 40
    K, V = (torch.zeros(pages, *shape, dtype=torch.uint8, device=DEV) for shape in ((Hkv, page, d), (Hkv, d, page)))
    Ks, Vs = (torch.ones(pages, Hkv, device=DEV) for _ in "KV")
    far = [pages - 1 - i for i in range(s.pages)]
    K[far], V[far], Ks[far], Vs[far] = s.K.view(torch.uint8), s.V.view(torch.uint8), s.Ks, s.Vs
    s.K, s.V, s.Ks, s.Vs, s.pages = K.view(F8), V.view(F8), Ks, Vs, pages
    s.tables = [pages - 1 - t for t in s.tables]
    again = s.attend([1], Q=got[0])
    assert torch.equal(got[1], again[1])
    near = far[::-1]

    def bring():
        x, y = (c.view(torch.uint8)[near].view(F8).double().cpu().numpy() for c in (s.K, s.V))
        return ref.Cache(x, y.swapaxes(2, 3), to_np(s.Ks[near]), to_np(s.Vs[near]))
    x = s.rows(3, Hkv)
    s.lengths[0] += 3
    csat.csat_cache_store(s.dims(1, 3, 1, 3, K=x, V=x), s.cache(0), x, x, dev_ints([0, 3]))
    t = (pages - 1 - s.tables[0]).tolist()
    for name in "KV":
        small.store(name, t[0], 200, to_np(x))
    after = bring()
    for name in "KV":
        assert np.array_equal(after.x[name][::-1], small.x[name], equal_nan=True) and np.array_equal(after.s[name][::-1], small.s[name])
    W, W_to, kept = torch.rand(1, Hkv, 256, device=DEV), torch.zeros(1, Hkv, 256, device=DEV), torch.zeros(1, Hkv, 150, dtype=torch.int32, device=DEV)
    csat.csat_cache_evict(s.dims(1, 1, 1, 1), s.cache(0), s.cache(1), W, W_to, 150, 10, kept)
    Q, O, lse, off = s.attend([1], i=1)
    r = bring()
    r.x, r.s = {k: v[::-1] for k, v in r.x.items()}, {k: v[::-1] for k, v in r.s.items()}
    s.tables = [pages - 1 - t for t in s.tables]
    s.check_attention(r, Q, O, lse, off, i=1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_serving_loop(dtype):
    """A batch's prompts, their keys and values into the cache, decode steps that collect weights, an eviction, and decode on: a
    captured step replayed with growing lengths against the same step called eagerly."""
    B, Hq, Hkv, d, page = 3, 8, 2, 64, 16
    s = Serving(B, Hq, Hkv, d, page, 10, dtype, tables=2)
    lens, off = [70, 33, 100], offsets([70, 33, 100])
    n = off[-1]
    Q, K, V = s.rows(n, Hq, 2.0), s.rows(n, Hkv), s.rows(n, Hkv)
    O, lse = torch.zeros(n, Hq, d, dtype=tdtype(dtype), device=DEV), torch.zeros(Hq, n, device=DEV)
    dims = s.dims(n, n, max(lens), max(lens))
    ws = torch.empty(csat.csat_prompt_workspace_bytes(dims), dtype=torch.uint8, device=DEV)
    o = dev_ints(off)
    r = s.reference()
    csat.csat_prompt_attention(dims, Q, K, V, o, o, s.scale, O, lse, ws)
    s.lengths[0] += dev_ints(lens)
    csat.csat_cache_store(dims, s.cache(0), K, V, o)
    t = s.tables[0].tolist()
    for b in range(B):
        r.store("K", t[b], 0, to_np(K[off[b]:off[b + 1]]))
        r.store("V", t[b], 0, to_np(V[off[b]:off[b + 1]]))
    want = ref.packed(to_np(Q), to_np(K), to_np(V), off, off, s.scale, True, dtype, np.zeros((n, Hq, d)), np.zeros((Hq, n)))
    ref.check("prompt", to_np(O), want[0], want[2])
    s.same_as(r)
    # the last eight rows of every prompt say what it looks at
    W = s.weights()
    got = s.attend([8, 8, 8], W=W)
    s.check_attention(r, *got, W=W, W_before=np.zeros(W.shape))
    # decode steps from a captured graph: q, k, v in, lengths grow on the device
    q, k, v = s.rows(B, Hq, 2.0), s.rows(B, Hkv), s.rows(B, Hkv)
    out, l = torch.zeros(B, Hq, d, dtype=tdtype(dtype), device=DEV), torch.zeros(Hq, B, device=DEV)
    step = s.dims(B, B, 1, 1)
    one = dev_ints(range(B + 1))
    ones = dev_ints([1] * B)
    cache = s.cache(0)
    ws = torch.empty(csat.csat_cache_workspace_bytes(step, cache), dtype=torch.uint8, device=DEV)

    def decode():
        s.lengths[0].add_(ones)
        csat.csat_cache_store(step, cache, k, v, one)
        csat.csat_cache_attention(step, cache, q, one, s.scale, 0.9, out, l, W, ws)
    graph = torch.cuda.CUDAGraph()
    saved = [x.clone() for x in (s.K.view(torch.uint8), s.V.view(torch.uint8), s.Ks, s.Vs, s.lengths[0], W)]
    with torch.cuda.graph(graph):
        decode()
    for x, y in zip((s.K.view(torch.uint8), s.V.view(torch.uint8), s.Ks, s.Vs, s.lengths[0], W), saved):
        x.copy_(y)
    for i in range(6):
        q.copy_(s.rows(B, Hq, 2.0)), k.copy_(s.rows(B, Hkv, 3.0 ** i)), v.copy_(s.rows(B, Hkv, 2.0 ** i))
        before, lens = to_np(W), s.lengths[0].tolist()
        graph.replay() if i % 2 == 0 else decode()
        torch.cuda.synchronize()
        assert s.lengths[0].tolist() == [x + 1 for x in lens]
        for b in range(B):
            r.store("K", t[b], lens[b], to_np(k[b:b + 1]))
            r.store("V", t[b], lens[b], to_np(v[b:b + 1]))
        s.same_as(r)
        s.check_attention(r, q, out, l, list(range(B + 1)), W=W, W_before=before, decay=float(np.float32(0.9)))
    W_to, _ = evict_and_check(s, W, 60, 12)
    r = s.reference()
    s.store([1, 1, 1], i=1, reference=None)
    r = s.reference()
    got = s.attend([1, 1, 1], i=1, W=W_to, decay=1.0, Q=s.rows(6, Hq, 2.0))
    s.check_attention(r, *got, i=1)


def test_shared_pages_and_two_streams():
    """Two sequences that begin with the same pages, each with weights of its own; two calls at once with their own workspaces."""
    s = Serving(2, 4, 2, 64, 16, 6, "bf16")
    s.tables[0][1, :3] = s.tables[0][0, :3]
    s.lengths[0] += dev_ints([60, 75])
    W = s.weights()
    got = s.attend([1, 1], W=W)
    r = s.reference()
    s.check_attention(r, *got, W=W, W_before=np.zeros(W.shape))
    s.store([1, 1], reference=r)
    s.same_as(r)
    want = s.attend([1, 1], W=W, Q=got[0])[1:3]
    dims, cache = s.dims(got[0].shape[0], 1, 1, 1), s.cache()
    off = dev_ints(got[3])
    runs = []
    for _ in range(2):
        runs.append((torch.cuda.Stream(), torch.full_like(want[0], 7.0), torch.full_like(want[1], 7.0), s.weights(),
                     torch.empty(csat.csat_cache_workspace_bytes(dims, cache), dtype=torch.uint8, device=DEV)))
    torch.cuda.synchronize()
    for st, O, lse, w, ws in runs * 3:
        csat.csat_cache_attention(dims, cache, got[0], off, s.scale, 0.0, O, lse, w, ws, st)
    torch.cuda.synchronize()
    for st, O, lse, w, ws in runs:
        assert torch.equal(O, want[0]) and torch.equal(lse, want[1]) and torch.equal(w, runs[0][3])
