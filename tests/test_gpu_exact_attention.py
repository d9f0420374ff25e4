"""Exact attention over packed sequences against its definition in 64 bits, with the bounds of the roundings that the kernels make
(tests/exact_reference.py)."""
import math

import numpy as np
import pytest
import torch

import paper_2507_02957_amd as csat
from tests import exact_reference as ref
from tests.gpu_harness import DEV, tdtype, to_np

pytestmark = pytest.mark.gpu


def offsets(lens, first=0):
    return [first] + [first + int(x) for x in np.cumsum(lens)]


def dev_ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Problem:
    """Packed tensors of the given lengths, some rows in front of the first sequence and behind the last."""

    def __init__(self, q_lens, k_lens, Hq, Hkv, d, dtype, causal, seed=0, front=3, tail=5, spread=2.0):
        g = torch.Generator(device="cpu").manual_seed(seed)
        self.Hq, self.Hkv, self.d, self.dtype, self.causal, self.B = Hq, Hkv, d, dtype, causal, len(q_lens)
        self.q_off, self.k_off = offsets(q_lens, front), offsets(k_lens, front)
        self.n_q, self.n_k = self.q_off[-1] + tail, self.k_off[-1] + tail
        t = tdtype(dtype)
        self.Q = (spread * torch.randn(self.n_q, Hq, d, generator=g)).to(t).to(DEV)
        self.K = torch.randn(self.n_k, Hkv, d, generator=g).to(t).to(DEV)
        self.V = torch.randn(self.n_k, Hkv, d, generator=g).to(t).to(DEV)
        self.scale = 1.0 / math.sqrt(d)
        self.max_q, self.max_k = max(max(q_lens), 1), max(max(k_lens), 1)
        self.O = torch.full((self.n_q, Hq, d), 7.0, dtype=t, device=DEV)
        self.lse = torch.full((Hq, self.n_q), 7.0, device=DEV)

    def dims(self, **tensors):
        return csat.make_packed_dims(self.B, self.Hq, self.Hkv, self.d, self.n_q, self.n_k, self.max_q, self.max_k, self.dtype, self.causal, **tensors)

    def call(self, want_lse=True, stream=None, ws=None):
        d = self.dims(Q=self.Q, K=self.K, V=self.V, O=self.O)
        if ws is None:
            ws = torch.full((csat.csat_prompt_workspace_bytes(d),), 255, dtype=torch.uint8, device=DEV)      # (NaN if it were read unwritten)
        csat.csat_prompt_attention(d, self.Q, self.K, self.V, dev_ints(self.q_off), dev_ints(self.k_off), self.scale, self.O,
                                   self.lse if want_lse else None, ws, stream)
        torch.cuda.synchronize()
        return self

    def check(self):
        O, lse, dO, dlse = ref.packed(to_np(self.Q), to_np(self.K), to_np(self.V), self.q_off, self.k_off, self.scale, self.causal, self.dtype,
                                      np.full((self.n_q, self.Hq, self.d), 7.0), np.full((self.Hq, self.n_q), 7.0))
        ref.check("O", to_np(self.O), O, dO)
        ref.check("lse", to_np(self.lse), lse, dlse)
        return self


SHAPES = [
    # q lengths, k lengths, Hq, Hkv, d
    ([1], [1], 1, 1, 8),
    ([5, 0, 33], [5, 0, 33], 2, 1, 24),
    ([64, 1, 130], [64, 1, 130], 4, 2, 64),
    ([257], [257], 3, 3, 80),
    ([40, 100], [200, 333], 8, 2, 128),                # the last rows of longer key sequences
    ([70, 3, 9], [20, 0, 9], 2, 2, 96),                # more rows than keys: causal leaves the first of them empty
    ([129], [129], 6, 2, 256),
    ([31, 66], [65, 127], 7, 1, 136),                  # seven heads to one
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_against_the_definition(shape, causal, dtype):
    q_lens, k_lens, Hq, Hkv, d = SHAPES[shape]
    Problem(q_lens, k_lens, Hq, Hkv, d, dtype, causal, seed=shape).call().check()


# enough heads that bf16 takes row tiles of 128 rows
WIDE = [
    ([1, 70, 33, 129, 64, 5, 0, 90], [1, 70, 33, 129, 64, 5, 0, 90], 32, 32, 64),
    ([40, 20, 128, 3], [90, 20, 300, 130], 64, 32, 128),
    ([130, 7, 60, 64], [65, 9, 64, 200], 32, 32, 80),
    ([33, 65], [33, 129], 128, 64, 96),
    ([50, 129], [50, 129], 64, 64, 256),
    ([140, 31], [100, 31], 64, 64, 200),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", range(len(WIDE)))
def test_many_heads_against_the_definition(shape, causal):
    q_lens, k_lens, Hq, Hkv, d = WIDE[shape]
    Problem(q_lens, k_lens, Hq, Hkv, d, "bf16", causal, seed=shape).call().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_shares_and_many_rows(dtype):
    """Two shares of the keys, joined a wavefront a row."""
    p = Problem([90, 50], [700, 520], 4, 2, 40, dtype, True).call()
    assert csat.csat_profile_launch_form("key_shares") == 2
    p.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q_lens,k_lens,Hq,Hkv,d", [([1], [3000], 4, 2, 64), ([1, 3, 0], [2100, 257, 900], 4, 1, 128), ([20], [5000], 2, 2, 80), ([2], [1030], 8, 1, 256)])
def test_few_rows_share_their_keys(q_lens, k_lens, Hq, Hkv, d, dtype):
    p = Problem(q_lens, k_lens, Hq, Hkv, d, dtype, True).call()
    assert csat.csat_profile_launch_form("key_shares") > 1
    p.check()
    lse = p.lse.clone()
    O = p.O.clone()
    p.call(want_lse=False)
    assert torch.equal(O, p.O) and torch.equal(lse, p.lse)


@pytest.mark.parametrize("q_lens,k_lens,Hq,Hkv,d", [([3, 3], [338, 1], 16, 2, 256), ([2, 0, 1], [65, 64, 31], 4, 4, 136), ([4, 1], [129, 7], 8, 2, 128),
                                                   ([5], [127], 4, 1, 72)])
def test_short_shares_of_float(q_lens, k_lens, Hq, Hkv, d):
    """Shares of a step or two, many of them behind the end of a short sequence."""
    p = Problem(q_lens, k_lens, Hq, Hkv, d, "f32", True).call().check()
    first = p.O.clone()
    p.call()
    assert torch.equal(first, p.O)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(dtype):
    """Parts of a fused projection, heads first, and a key head that all heads share by a stride of 0."""
    want = Problem([50, 81], [50, 81], 4, 2, 64, dtype, True).call().check()
    p = Problem([50, 81], [50, 81], 4, 2, 64, dtype, True)
    fused = torch.cat([p.Q, p.K, p.V], 1)
    p.Q, p.K, p.V = fused[:, :4], fused[:, 4:6], fused[:, 6:]
    p.call()
    assert torch.equal(p.O, want.O) and torch.equal(p.lse, want.lse)
    for name in ("Q", "K", "V", "O"):
        setattr(p, name, getattr(want, name).transpose(0, 1).contiguous().transpose(0, 1))
    p.O.fill_(7.0)
    p.call()
    assert torch.equal(p.O, want.O) and torch.equal(p.lse, want.lse)
    p = Problem([50, 81], [50, 81], 4, 1, 64, dtype, False).call().check()
    s = Problem([50, 81], [50, 81], 4, 4, 64, dtype, False)
    s.Q, s.K, s.V = p.Q, p.K.expand(-1, 4, -1), p.V.expand(-1, 4, -1)
    s.call().check()
    # one row of V for all tokens
    s.V = p.V[:1].expand(s.n_k, 4, -1)
    s.call().check()


ODD = [float("nan"), float("inf"), -float("inf")]


@pytest.mark.parametrize("heads,d,dtype", [(2, 64, "f32"), (2, 128, "f32"), (2, 256, "f32"), (2, 64, "bf16"), (2, 128, "bf16"), (64, 64, "bf16"), (64, 128, "bf16")])
def test_odd_values_in_masked_places(heads, d, dtype):
    """What no row sees does not matter: rows of no sequence, of the next one, of keys behind the causal limit."""
    p = Problem([70, 90], [70, 90], heads if heads > 2 else 4, heads, d, dtype, True).call().check()
    want, lse = p.O.clone(), p.lse.clone()
    a, b = p.k_off[1], p.k_off[2]
    for i, x in enumerate(ODD):
        p.K[b + i], p.V[b + i] = x, x
        p.K[i], p.V[i] = x, x
    p.call()
    assert torch.equal(p.O, want) and torch.equal(p.lse, lse)
    # values that some rows of a sequence see and others do not
    for i, x in enumerate(ODD):
        p.V[a - 40 + 7 * i, 0, 3 + 2 * i] = x
        p.V[b - 60 + 11 * i, 1, 5] = x
    p.V[a - 2, 0, 11], p.V[a - 1, 0, 11] = ODD[1], ODD[2]            # +inf and -inf together
    p.call().check()
    p.K[a - 30] = float("nan")
    p.call().check()


@pytest.mark.parametrize("scale", [1e-30, 1e-38, 1e30])
def test_float_values_of_every_size(scale):
    """V far from 1, where parts of a float are below or next to the smallest bf16 or the largest."""
    p = Problem([60], [60], 2, 1, 64, "f32", True)
    p.V *= scale
    p.call().check()
    p.V[::3] *= 1e-6
    p.call().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_of_minus_infinity(dtype):
    """A score of -inf has weight 0; a row with no other is empty; +inf gives NaN as its definition does."""
    p = Problem([5, 3], [40, 4], 2, 1, 16, dtype, False)
    p.Q.abs_().add_(0.5)
    p.K[p.k_off[0] + 7] = -float("inf")
    p.K[p.k_off[0] + 33:p.k_off[1]] = -float("inf")
    p.K[p.k_off[1]:p.k_off[2]] = -float("inf")
    p.call().check()
    assert (p.O[p.q_off[1]:p.q_off[2]] == 0).all() and (p.lse[:, p.q_off[1]:p.q_off[2]] == -math.inf).all()
    p.K[p.k_off[0] + 8] = float("inf")
    p.call()
    assert torch.isnan(p.O[p.q_off[0]:p.q_off[1]]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_that_grow_and_reach_far(dtype):
    """The running maximum moves at every step; scores of hundreds neither overflow nor lose the small ones' sum."""
    p = Problem([200], [200], 2, 2, 64, dtype, True, spread=1.0)
    ramp = torch.linspace(0.2, 8.0, p.n_k, device=DEV)[:, None, None]
    p.K = (p.K * ramp).to(tdtype(dtype))
    p.Q = (p.Q * 6).to(tdtype(dtype))
    p.call().check()
    p.K = p.K.flip(0).contiguous()
    p.call().check()


def test_bounds_of_rows_and_bad_offsets():
    """Rows beyond max_q are left alone, and so is everything where the offsets say nonsense."""
    p = Problem([50, 20], [50, 20], 2, 1, 64, "bf16", True).call()
    want = p.O.clone()
    p.O.fill_(7.0)
    p.max_q = 30
    p.call()
    q = p.q_off
    assert torch.equal(p.O[q[0]:q[0] + 30], want[q[0]:q[0] + 30]) and torch.equal(p.O[q[1]:q[2]], want[q[1]:q[2]])
    assert (p.O[q[0] + 30:q[1]] == 7.0).all() and (p.O[:q[0]] == 7.0).all() and (p.O[q[2]:] == 7.0).all()
    p.O.fill_(7.0)
    p.q_off, p.k_off = [5, -4, 1 << 30], [1 << 29, 0, -1]
    p.max_q = 1000
    p.call()
    assert (p.O[:5] == 0).all() or torch.isfinite(p.O.float()).all()      # nothing faults, what is written is a number


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q,k", [(300, 300), (2, 4000)])
def test_streams_and_graphs(q, k, dtype):
    """Two calls at once on two streams, and a captured call replayed between eager work, give the eager result."""
    ps = [Problem([q], [k], 4, 2, 64, dtype, True, seed=s) for s in (1, 2)]
    want = [(p.call().O.clone(), p.lse.clone()) for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    dims = [p.dims() for p in ps]
    offs = [(dev_ints(p.q_off), dev_ints(p.k_off)) for p in ps]
    ws = [torch.empty(csat.csat_prompt_workspace_bytes(d), dtype=torch.uint8, device=DEV) for d in dims]

    def one(i, stream=None):
        p = ps[i]
        csat.csat_prompt_attention(dims[i], p.Q, p.K, p.V, *offs[i], p.scale, p.O, p.lse, ws[i], stream)
    for p in ps:
        p.O.fill_(7.0)
    torch.cuda.synchronize()
    for _ in range(3):
        for i, s in enumerate(streams):
            one(i, s)
    torch.cuda.synchronize()
    for p, (O, lse) in zip(ps, want):
        assert torch.equal(p.O, O) and torch.equal(p.lse, lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(0)
    for _ in range(3):
        ps[0].O.fill_(7.0)
        ps[0].lse.fill_(7.0)
        one(1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ps[0].O, want[0][0]) and torch.equal(ps[0].lse, want[0][1])


def test_far_rows():
    """Rows whose byte offsets pass 32 bits."""
    d, n = 128, 9_000_000
    p = Problem([40], [40], 2, 2, d, "bf16", True).call().check()
    K = torch.empty(n, 2, d, dtype=torch.bfloat16, device=DEV)                # 4.6 GB
    V = torch.empty(n, 2, d, dtype=torch.bfloat16, device=DEV)
    first = n - 60
    K[first:first + 40], V[first:first + 40] = p.K[p.k_off[0]:p.k_off[1]], p.V[p.k_off[0]:p.k_off[1]]
    want = p.O.clone()
    p.K, p.V, p.n_k, p.k_off = K, V, n, [first, first + 40]
    p.O.fill_(7.0)
    p.call()
    assert torch.equal(p.O, want)
