"""Dense attention over packed sequences (lsrm_attn_forward, lsrm_attn_backward) and its relative position bias against
the definition in float64 (attn_ref)."""
import numpy as np
import pytest
import torch

import attn_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_05182_amd import binding
    return binding


def rows(n, h, d, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((n, h, d), generator=g) * scale).to(torch.bfloat16).cuda()


def int32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


class Problem:
    """q_lens, k_lens: lengths (k_lens None: self attention).  slots: rows of every sequence's slot are `slots` more than its
    length, filled with NaN.  edge: rows before the first and behind the last sequence, NaN too."""

    def __init__(self, B, q_lens, k_lens=None, h=2, hk=None, d=64, causal=False, bounds=None, slots=0, edge=0, fused=False, seed=1,
                 scale=0.0, spread=1.0, bias=None):
        self.B, self.causal, self.bounds, self.scale = B, causal, bounds, scale
        hk = hk or h
        self.self_attention = k_lens is None
        k_lens = q_lens if k_lens is None else k_lens
        self.q_lens, self.k_lens = list(q_lens), list(k_lens)
        self.q_off = R.lengths_to_offsets([x + slots for x in q_lens], edge)
        self.k_off = R.lengths_to_offsets([x + slots for x in k_lens], edge)
        n_q, n_k = int(self.q_off[-1]) + edge, int(self.k_off[-1]) + edge
        if fused:
            x = rows(n_q, h + 2 * hk, d, seed, spread)
            self.q, self.k, self.v = x[:, :h], x[:, h:h + hk], x[:, h + hk:]
            x = torch.full_like(x, 7.0)
            self.dq, self.dk, self.dv = x[:, :h], x[:, h:h + hk], x[:, h + hk:]
        else:
            self.q, self.k, self.v = rows(n_q, h, d, seed, spread), rows(n_k, hk, d, seed + 1), rows(n_k, hk, d, seed + 2)
            self.dq, self.dk, self.dv = (torch.full_like(x, 7.0) for x in (self.q, self.k, self.v))
        self.dout = rows(n_q, h, d, seed + 3)
        self.q_rows = [(int(o), l) for o, l in zip(self.q_off, q_lens)]
        self.k_rows = [(int(o), l) for o, l in zip(self.k_off, k_lens)]
        self.q_in = self._inside(self.q_rows, n_q)
        self.k_in = self._inside(self.k_rows, n_k)
        self.host = {x: np.nan_to_num(R.f64(getattr(self, x))) for x in ("q", "k", "v", "dout")}
        for x, inside in ((self.q, self.q_in), (self.k, self.k_in), (self.v, self.k_in), (self.dout, self.q_in)):
            x[~inside.cuda()] = float("nan")
        self.bias = self.dbias = None
        if bounds is not None:
            self.bias = torch.randn((h, len(bounds) + 1), generator=torch.Generator().manual_seed(seed + 4)).to(torch.bfloat16).cuda() if bias is None else bias
            self.dbias = torch.full_like(self.bias, 7.0)
        self.out = torch.full((n_q, h, d), 7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((n_q, h), 7.0, device="cuda")
        lens = slots > 0
        self.p = B.make_attn_params(self.q, self.k, self.v, int32(self.q_off), None if self.self_attention else int32(self.k_off),
                                    int32(q_lens) if lens else None, int32(k_lens) if lens and not self.self_attention else None,
                                    causal, scale, bounds)

    @staticmethod
    def _inside(spans, n):
        x = torch.zeros(n, dtype=torch.bool)
        for a, l in spans:
            x[a:a + l] = True
        return x

    def workspace(self, which):
        ws = self.B.alloc_attn_workspace(self.p, which)
        return ws if ws is None else ws.fill_(0xFF)

    def forward(self, stream=None):
        self.B.lsrm_attn_forward(self.p, self.q, self.k, self.v, self.out, self.lse, self.workspace(self.B.LSRM_WS_FORWARD), self.bias, stream)

    def backward(self, stream=None):
        self.B.lsrm_attn_backward(self.p, self.q, self.k, self.v, self.out, self.lse, self.dout, self.dq, self.dk, self.dv,
                                  self.workspace(self.B.LSRM_WS_BACKWARD), self.bias, self.dbias, stream)

    def check(self, train=True):
        val, err = R.attention(self.host["q"], self.host["k"], self.host["v"], self.q_rows, self.k_rows, self.causal, self.scale,
                               None if self.bias is None else R.f64(self.bias), self.bounds or (), self.host["dout"] if train else None)
        torch.cuda.synchronize()
        names = ["out", "lse"] + (["dq", "dk", "dv"] if train else []) + (["dbias"] if train and self.bias is not None else [])
        for name in names:
            R.check(name, R.f64(getattr(self, name)), val[name], err[name])
        # rows of a slot behind its length: zeros; rows of no sequence: as they were
        for name in names:
            if name == "dbias":
                continue
            t, off, inside = getattr(self, name), self.q_off if name in ("out", "lse", "dq") else self.k_off, self.q_in if name in ("out", "lse", "dq") else self.k_in
            behind = ~inside
            behind[:off[0]] = behind[off[-1]:] = False
            outside = torch.ones_like(inside)
            outside[off[0]:off[-1]] = False
            assert (t[behind.cuda()] == (float("-inf") if name == "lse" else 0)).all(), f"{name}: rows behind a length"
            assert (t[outside.cuda()] == 7.0).all(), f"{name}: rows of no sequence"
        return self


def all_forward_kernels():
    """(name, problem): sizes at which a forward call takes each of its ways"""
    return [
        ("few", dict(q_lens=[40, 1, 70], h=4, hk=2)),
        ("few, cut", dict(q_lens=[2, 1, 3], k_lens=[3000, 1025, 2000], h=4, hk=2)),
        ("many", dict(q_lens=[333, 5, 1030, 128], h=16)),
        ("many, cut", dict(q_lens=[700, 1500], k_lens=[1400, 2100], h=2, hk=1)),
    ]


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("way", [0, 1, 2, 3], ids=[name for name, _ in all_forward_kernels()])
def test_every_way(B, way, bias, causal, d):
    x = Problem(B, d=d, causal=causal, seed=101, bounds=[-200, -64, -20, -3, 0, 1, 9, 100] if bias else None, **all_forward_kernels()[way][1])
    x.forward()
    x.backward()
    x.check()


@pytest.mark.parametrize("way", [0, 1, 2, 3], ids=[name for name, _ in all_forward_kernels()])
def test_every_way_with_slots(B, way):
    """rows of slots behind their lengths hold NaN; so do rows before the first and behind the last sequence"""
    x = Problem(B, d=64, causal=True, slots=133, edge=70, bounds=[-30, -1, 0], seed=102, **all_forward_kernels()[way][1])
    x.forward()
    x.backward()
    x.check()


@pytest.mark.parametrize("h", [2, 16])
def test_more_queries_than_keys(B, h):
    """causal: the first queries of a sequence see nothing"""
    x = Problem(B, [600, 900, 130], [100, 899, 1], h=h, d=64, causal=True, seed=103)
    x.forward()
    x.backward()
    x.check()


def test_many_rows_of_many_sequences(B):
    """more sequences than a wavefront has lanes, each of several tiles"""
    rng = np.random.default_rng(8)
    x = Problem(B, rng.integers(0, 300, 90), h=8, hk=8, d=32, causal=True, seed=104, slots=11, edge=300)
    x.forward()
    x.backward()
    x.check()


@pytest.mark.parametrize("lengths", [[50, 9], [1500, 900]], ids=str)
def test_head_major(B, lengths):
    """[heads, rows, channels] underneath"""
    x = Problem(B, lengths, h=8, hk=4, d=64, causal=True, seed=108)
    for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        t = getattr(x, name)
        setattr(x, name, t.transpose(0, 1).contiguous().transpose(0, 1))
    x.p = B.make_attn_params(x.q, x.k, x.v, int32(x.q_off), causal=True, out=x.out)
    x.forward()
    x.backward()
    x.check()


def test_rows_far_apart(B):
    """strides at their limit: offsets within a tile pass 2^31 bytes, those of the whole tensor 2^32"""
    n, step = 150, 1 << 24
    buf = torch.empty((n - 1) * step + 4 * 64, dtype=torch.bfloat16, device="cuda")
    x = Problem(B, [n], h=2, d=64, seed=105)
    for name, head in (("q", 0), ("k", 0), ("v", 2)):
        far = buf.as_strided((n, 2, 64), (step, 64, 1), head * 64)
        if name != "q":
            far.copy_(getattr(x, name))
            setattr(x, name, far)
    x.p = B.make_attn_params(x.q, x.k, x.v, int32(x.q_off), int32(x.k_off))
    x.dk, x.dv = torch.empty_like(buf).as_strided((n, 2, 64), (step, 64, 1)), buf.new_empty(buf.shape).as_strided((n, 2, 64), (step, 64, 1))
    x.forward()
    x.backward()
    x.check()


def test_two_at_once(B):
    """two problems on two streams, workspaces of their own"""
    xs = [Problem(B, [2000], h=2, d=64, seed=106, causal=True), Problem(B, [1] * 3, [4000, 100, 2500], h=8, hk=1, d=128, seed=107, causal=True)]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    spaces = [(x.workspace(B.LSRM_WS_FORWARD), x.workspace(B.LSRM_WS_BACKWARD)) for x in xs]
    torch.cuda.synchronize()
    for _ in range(4):
        for x, st, (wf, wb) in zip(xs, streams, spaces):
            B.lsrm_attn_forward(x.p, x.q, x.k, x.v, x.out, x.lse, wf, x.bias, st)
            B.lsrm_attn_backward(x.p, x.q, x.k, x.v, x.out, x.lse, x.dout, x.dq, x.dk, x.dv, wb, stream=st)
    for x in xs:
        x.check()


def test_offsets_that_do_not_fit(B):
    """beyond the tensors, descending, lengths past their slots: no access leaves the tensors (what comes out is not specified), and sequences
    that are described well beside them are right"""
    q, k, v = rows(100, 4, 64, 1), rows(120, 2, 64, 2), rows(120, 2, 64, 3)
    for q_off, k_off, q_len, k_len in (([0, 40, 1 << 29], [0, 50, 1 << 30], None, None), ([-7, 40, 30], [60, 50, 120], None, None),
                                       ([0, 40, 100], [0, 50, 120], [1 << 20, 60], [99, -4]), ([90, 95, 2000], [119, 119, 119], None, None)):
        for n_seq, causal in ((2, False), (2, True), (70, True)):
            pad = [0] * (n_seq - 2)
            args = [int32(list(o) + [o[-1]] * len(pad)) for o in (q_off, k_off)] + [None if l is None else int32(l + pad) for l in (q_len, k_len)]
            p = B.make_attn_params(q, k, v, *args, causal=causal)
            out, lse = torch.zeros_like(q), torch.zeros((100, 4), device="cuda")
            dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
            B.lsrm_attn_forward(p, q, k, v, out, lse, B.alloc_attn_workspace(p, B.LSRM_WS_FORWARD))
            B.lsrm_attn_backward(p, q, k, v, out, lse, q, dq, dk, dv, B.alloc_attn_workspace(p, B.LSRM_WS_BACKWARD))
            torch.cuda.synchronize()


LENGTHS = [[1], [2], [31], [32], [33], [64, 1, 65], [127, 128, 129], [0, 5, 0, 70, 0], [200, 3]]


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_self_attention(B, lengths, causal, d):
    x = Problem(B, lengths, h=2, d=d, causal=causal)
    x.forward()
    x.check(train=False)
    x.backward()
    x.check()


@pytest.mark.parametrize("h,hk", [(1, 1), (3, 1), (6, 2), (8, 2), (16, 1), (40, 1)])
@pytest.mark.parametrize("causal", [False, True])
def test_grouped_heads(B, h, hk, causal):
    x = Problem(B, [37, 70, 1], h=h, hk=hk, d=32, causal=causal, seed=11)
    x.forward()
    x.backward()
    x.check()


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_queries_and_keys_of_different_lengths(B, causal, d):
    """more queries than keys (causal: the first see none), fewer, none of either"""
    x = Problem(B, [50, 3, 0, 40, 7, 90], [20, 200, 9, 0, 8, 65], h=4, hk=2, d=d, causal=causal, seed=21)
    x.forward()
    x.backward()
    x.check()


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("h,hk", [(4, 4), (16, 2)])
def test_many_workgroups(B, d, h, hk):
    """enough rows that wavefronts share their tiles"""
    x = Problem(B, [900, 300, 2050], h=h, hk=hk, d=d, causal=True, seed=31) if h == 16 else Problem(B, [1500, 2700, 4100], h=h, d=d, seed=31)
    x.forward()
    x.backward()
    x.check()


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("queries", [1, 3])
@pytest.mark.parametrize("bias", [False, True])
def test_single_tokens_over_a_cache(B, d, queries, bias):
    """few queries, long keys of different lengths in slots with NaN behind them"""
    keys = [1000, 5000, queries, 129, 4097]
    x = Problem(B, [queries] * 5, keys, h=16, hk=2, d=d, causal=True, slots=77, edge=3, seed=41,
                bounds=B.lsrm_rel_bucket_bounds(16, 128, False) if bias else None)
    x.forward()
    x.check(train=False)


@pytest.mark.parametrize("n_seq", [1, 65, 700])
def test_numbers_of_sequences(B, n_seq):
    rng = np.random.default_rng(n_seq)
    x = Problem(B, rng.integers(0, 6, n_seq), rng.integers(0, 40, n_seq), h=2, d=32, seed=51)
    x.forward()
    x.backward()
    x.check()


def test_many_sequences_split(B):
    """more sequences than a wavefront has lanes, keys cut into parts"""
    rng = np.random.default_rng(5)
    x = Problem(B, [1] * 150, rng.integers(1, 1500, 150), h=2, hk=1, d=64, causal=True, seed=52)
    x.forward()
    x.check(train=False)


@pytest.mark.parametrize("d", [32, 128])
def test_padded_batch(B, d):
    """slots longer than their sequences, NaN in the padding and around"""
    x = Problem(B, [20, 0, 90, 33], h=4, hk=2, d=d, causal=True, slots=45, edge=9, seed=61)
    x.forward()
    x.backward()
    x.check()


def test_slices_of_a_projection(B):
    x = Problem(B, [70, 131], h=4, hk=2, d=64, fused=True, seed=71)
    assert not x.q.is_contiguous()
    x.forward()
    x.backward()
    x.check()


BOUNDS = {"two-sided": (16, 128, True), "behind": (32, 128, False), "coarse": (2, 2, True)}


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("kind", list(BOUNDS))
def test_bias(B, kind, causal, d):
    x = Problem(B, [5, 200, 333], h=4, hk=2, d=d, causal=causal, bounds=B.lsrm_rel_bucket_bounds(*BOUNDS[kind]), seed=81)
    x.forward()
    x.backward()
    x.check()


@pytest.mark.parametrize("bounds", [[], [0], [-400, 600], [-3, 1, 5, 6]], ids=str)
def test_bias_with_other_bounds(B, bounds):
    x = Problem(B, [100, 900], h=2, d=64, bounds=bounds, seed=82)
    x.forward()
    x.backward()
    x.check()


def test_bias_of_a_large_group(B):
    """the largest expanded biases: 32 heads on one; the widest span of one head"""
    for h, hk, bounds in ((32, 1, list(range(-189, 2, 5))), (8, 1, [-700, -2, 322])):
        assert bounds[-1] - bounds[0] == 1022 or (h // hk) * (bounds[-1] - bounds[0] + 130) == 10240
        x = Problem(B, [150, 2300 if h == 8 else 90], h=h, hk=hk, d=64, bounds=bounds, seed=83)
        x.forward()
        x.backward()
        x.check()


def test_bias_that_masks(B):
    """-inf and the type's lowest value mask a bucket; a row whose keys are all masked gives zeros"""
    bias = torch.zeros((2, 4), dtype=torch.bfloat16)
    bias[0, 0] = float("-inf")
    bias[0, 3] = torch.finfo(torch.bfloat16).min
    bias[1] = float("-inf")
    x = Problem(B, [3, 100], h=2, d=32, bounds=[-5, 0, 9], seed=84, bias=bias.cuda())
    x.forward()
    assert (x.out[:, 1] == 0).all() and (x.lse[:, 1] == float("-inf")).all()
    x.backward()
    x.check()


def test_long_keys_far_bias(B):
    """nearly all keys lie in the far buckets, whose gradients are sums that nearly cancel"""
    x = Problem(B, [2500], h=2, d=64, bounds=B.lsrm_rel_bucket_bounds(8, 16, True), seed=85)
    x.forward()
    x.backward()
    x.check()


@pytest.mark.parametrize("spread", [0.0, 8.0])
def test_extreme_scores(B, spread):
    """all scores equal; scores of +-100, so that rows have one key"""
    x = Problem(B, [90, 300], h=2, d=64, causal=True, seed=91, spread=spread)
    x.forward()
    x.backward()
    x.check()


def test_scores_that_rise(B):
    """the maximum grows from tile to tile by more than any one step allows"""
    x = Problem(B, [1, 40], [2000, 700], h=1, d=32, seed=92)
    ramp = torch.linspace(0.1, 12, 2700).to(torch.bfloat16)
    x.q.fill_(1.0)
    x.k.copy_(ramp[:, None, None].expand(2700, 1, 32).cuda())
    x.host["q"], x.host["k"] = R.f64(x.q), R.f64(x.k)
    x.forward()
    x.backward()
    x.check()


def test_scale(B):
    x = Problem(B, [100], h=2, d=64, scale=0.5, seed=93)
    x.forward()
    x.backward()
    x.check()


def test_without_lse_and_bias_gradient(B):
    x = Problem(B, [60, 61], h=2, d=64, bounds=[-2, 3], seed=94)
    x.forward()
    out = x.out.clone()
    x.out.fill_(3.0)
    B.lsrm_attn_forward(x.p, x.q, x.k, x.v, x.out, None, x.workspace(B.LSRM_WS_FORWARD), x.bias)
    assert torch.equal(out, x.out)
    x.backward()
    x.check()
    dq, dbias = x.dq.clone(), x.dbias
    x.dbias = None
    x.dq.fill_(5.0)
    x.backward()
    assert torch.equal(dq, x.dq)
    x.dbias = dbias


def test_nothing_to_do(B):
    """no sequences, no rows: the bias' gradient is zero, other tensors are left alone"""
    x = Problem(B, [], h=2, d=64, bounds=[-1, 1], edge=4)
    x.forward()
    x.backward()
    torch.cuda.synchronize()
    assert (x.dbias == 0).all() and (x.out == 7).all() and (x.dk == 7).all()
    x = Problem(B, [0, 0], [3, 0], h=2, d=64, bounds=[-1, 1])
    x.forward()
    x.backward()
    torch.cuda.synchronize()
    assert (x.dbias == 0).all() and (x.dk == 0).all() and (x.dv == 0).all()


def test_same_bits_every_time(B):
    for kw in (dict(q_lens=[1] * 4, k_lens=[3000] * 4, causal=True), dict(q_lens=[300, 1000], bounds=[-40, -3, 0, 2, 50])):
        x = Problem(B, h=4, hk=2, d=64, seed=95, **kw)
        first = None
        for _ in range(3):
            x.forward()
            x.backward()
            torch.cuda.synchronize()
            now = [t.clone() for t in (x.out, x.lse, x.dq, x.dk, x.dv) + ((x.dbias,) if x.bias is not None else ())]
            assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
            first = now


def test_other_stream(B):
    x = Problem(B, [400, 100], h=4, d=64, seed=96)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    x.forward(st)
    x.backward(st)
    st.synchronize()
    x.check()


def test_captured_and_replayed(B):
    """two problems of their own workspaces in one graph, replayed between eager work; lengths change under the graph"""
    xs = [Problem(B, [300, 20], h=4, hk=2, d=64, causal=True, bounds=[-20, -2, 0], seed=97),
          Problem(B, [1, 1], [2000, 700], h=8, hk=1, d=128, causal=True, slots=64, seed=98)]
    for x in xs:
        x.ws = [x.workspace(B.LSRM_WS_FORWARD), x.workspace(B.LSRM_WS_BACKWARD)]

    def step():
        for x in xs:
            B.lsrm_attn_forward(x.p, x.q, x.k, x.v, x.out, x.lse, x.ws[0], x.bias)
            B.lsrm_attn_backward(x.p, x.q, x.k, x.v, x.out, x.lse, x.dout, x.dq, x.dk, x.dv, x.ws[1], x.bias, x.dbias)

    def results():
        torch.cuda.synchronize()
        return [t.clone() for x in xs for t in (x.out, x.lse, x.dq, x.dk, x.dv)] + [xs[0].dbias.clone()]

    step()
    want = results()
    for x in xs:
        x.check()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for n in range(3):
        for x in xs:
            x.out.fill_(float("nan"))
            x.dk.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        got = results()
        keep = [torch.where(torch.isnan(a), b, a) if i % 5 == 0 else a for i, (a, b) in enumerate(zip(got, want))]
        assert all(torch.equal(a, b) for a, b in zip(keep, want)), n
        torch.ones(1000, device="cuda").sum().item()
    # the cache grows: the same graph, other lengths
    x = xs[1]
    x.p._keepalive[3].copy_(int32([2050, 64]))
    torch.cuda.synchronize()
    x.k[x.k.isnan()] = 0.5
    x.v[x.v.isnan()] = 0.25
    x.host["k"], x.host["v"] = R.f64(x.k), R.f64(x.v)
    graph.replay()
    torch.cuda.synchronize()
    val, err = R.attention(x.host["q"], x.host["k"], x.host["v"], x.q_rows, [(0, 2050), (2064, 64)], True)
    R.check("out", R.f64(x.out), val["out"], err["out"])


def test_beside_the_sparse_layer(B):
    """dense attention of the tokens of a scene, then the sparse layer over its result: one stream, no waiting in between"""
    from gpu_util import params_for
    from paper_2604_05182_amd import inputs as I
    import oracle
    cfg = I.small_config(name="dense-then-sparse", n_obj=512, n_views=2, grid=16, heads=2, d=64, topk=4, window=128, seed=5)
    x = Problem(B, [cfg.n_obj, cfg.n_img], h=2, d=64, seed=99)
    p = params_for(B, cfg)
    idx = torch.empty((cfg.nb, cfg.topk), dtype=torch.int32, device="cuda")
    kc = torch.empty((cfg.nb, 2, 64), dtype=torch.bfloat16, device="cuda")
    vc, out = torch.empty_like(kc), torch.empty_like(x.out)
    pos, cams = I.make_points(cfg), I.make_cameras(cfg)
    gates = I.make_gates(cfg)
    x.forward()
    B.lsrm_route_blocks(p, torch.from_numpy(pos).cuda(), torch.from_numpy(cams).cuda(), idx, None, B.alloc_workspace(p, B.LSRM_WS_ROUTE))
    B.lsrm_nsa_compress(p, x.k, x.out, kc, vc)
    B.lsrm_nsa_forward(p, x.q, x.k, x.out, kc, vc, idx, torch.from_numpy(gates).cuda(), out, None, None, B.alloc_workspace(p, B.LSRM_WS_FORWARD))
    torch.cuda.synchronize()
    x.check(train=False)
    q, k, v = (t.float().cpu().numpy() for t in (x.q, x.k, x.out))
    ref = oracle.nsa_forward(q, k, v, oracle.pool(k), oracle.pool(v), idx.cpu().numpy(), gates, cfg.seg_offsets(), cfg.window)
    assert np.abs(out.float().cpu().numpy() - ref).max() <= 2e-2


def test_one_row_of_a_large_cache(B):
    """One key in a head-major cache whose heads lie 2^23 elements apart"""
    n, h, d = 1 << 16, 4, 128
    cache = torch.full((2, h, n, d), float("nan"), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    k, v = cache[0, :1], cache[1, :1]
    k.copy_(rows(1, h, d, 1))
    v.copy_(rows(1, h, d, 2))
    q = rows(1, h, d, 3)
    out = torch.empty_like(q)
    p = B.make_attn_params(q, k, v, int32([0, 1]), int32([0, 1]), causal=True)
    B.lsrm_attn_forward(p, q, k, v, out, None, B.alloc_attn_workspace(p, B.LSRM_WS_FORWARD))
    assert torch.equal(out, v)  # one key: its probability is one


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("case", [
    dict(q_lens=[257, 100, 30, 1, 180], h=8, hk=4),               # few keys to a workgroup
    dict(q_lens=[1, 40, 0, 5], k_lens=[33, 0, 64, 200], h=6, hk=1),  # the same; fewer tiles of queries than wavefronts, none at all
    dict(q_lens=[640, 520], h=32),                                # 128 rows and keys
    dict(q_lens=[2048], h=8, hk=2),                               # dK, dV: walks cut
    dict(q_lens=[70], k_lens=[6000], h=2, hk=1),                  # dQ: walks cut
    dict(q_lens=[6000], k_lens=[70], h=2, hk=1),
], ids=["few", "few, short", "many", "grouped", "few queries", "few keys"])
def test_every_way_backward(B, case, bias, causal, d):
    x = Problem(B, d=d, causal=causal, seed=103, slots=9, edge=3, bounds=[-90, -17, -1, 0, 1, 40] if bias else None, **case)
    x.forward()
    x.backward()
    x.check()
