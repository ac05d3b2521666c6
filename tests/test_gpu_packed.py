"""GPU parity of packed attention, rotary axes and dropout against the oracle in 64 bits, at the sizes, strides and values where they can go wrong.

Tolerances count roundings.  bf16: half a step is 2^-8 of a value.  O is rounded once, and each probability once before it is summed, so
|O - exact| <= 2^-8 (|O| + sum P |V|); likewise a gradient with |dS| or P in the place of P.  What is computed in fp32 before those roundings (a product's d terms, the
exponential, a difference dP - rowsum(dO O)) is off by at most FP32 = 2^-14 of the magnitudes summed: (d + 4) 2^-24 < 2^-16 for a product, and the exponent's argument,
below 64 in these inputs, carries 2^-24 * 64 + (d + 4) 2^-24 * 64 / sqrt(d) < 2^-15 into every probability."""
import math

import numpy as np
import pytest
import torch

import paper_2411_01075_amd as C
from oracle import packed as opacked

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
FP32 = 2.0 ** -14
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
LIB = {"bf16": C.BF16, "f32": C.F32}
MARK = 7.0      # in every place that a call may not touch


def _starts(lengths, before=0):
    return [before + int(v) for v in np.concatenate([[0], np.cumsum(lengths)])]


class Packed:
    """Buffers of one call: rows before and behind the samples and columns past the rows hold MARK."""

    def __init__(self, dtype, heads, kv_heads, d, causal, lengths, before=0, behind=0, gap=0, seed=0, scale=0.0, std=1.0):
        self.dtype, self.heads, self.kv_heads, self.d, self.causal = dtype, heads, kv_heads, d, causal
        self.starts = _starts(lengths, before)
        self.rows = self.starts[-1] + behind
        self.width, self.o_width = (heads + 2 * kv_heads) * d, heads * d
        self.desc = C.packed_desc(heads, kv_heads, d, causal, LIB[dtype], self.rows, self.width + gap, self.o_width + gap, scale)
        self.scale = scale or 1 / math.sqrt(d)
        self.plan = C.cephalo_packed_plan(self.desc, self.starts).cuda()
        rng = np.random.default_rng(seed)
        def buffer(width, inner):
            t = torch.full((self.rows, width + gap), MARK, dtype=TORCH[dtype])
            t[before:self.starts[-1], :width] = torch.from_numpy(inner).to(TORCH[dtype])
            return t.cuda()
        n = self.starts[-1] - before
        self.qkv = buffer(self.width, std * rng.standard_normal((n, self.width)))
        self.dO = buffer(self.o_width, rng.standard_normal((n, self.o_width)))
        self.O = torch.full_like(self.dO, MARK)
        self.dqkv = torch.full_like(self.qkv, MARK)
        self.lse = torch.full((heads, self.rows), MARK, device="cuda")
        self.workspace = torch.full((C.cephalo_op_attention_packed_bwd_workspace(self.desc),), 0xAB, dtype=torch.uint8, device="cuda")

    def forward(self, **kw):
        C.cephalo_op_attention_packed_fwd(self.desc, self.plan, self.qkv, self.O, self.lse, **kw)

    def backward(self, **kw):
        C.cephalo_op_attention_packed_bwd(self.desc, self.plan, self.qkv, self.O, self.dO, self.lse, self.dqkv, self.workspace, **kw)

    def host(self, t, width):
        return t.double().cpu().numpy()[:, :width]

    def untouched(self, t, width):
        t = t.float().cpu().numpy()
        return (t[:self.starts[0]] == MARK).all() and (t[self.starts[-1]:] == MARK).all() and (t[:, width:] == MARK).all()


def _within(name, got, want, bound):
    off = np.abs(got - want) - bound
    assert np.isfinite(got).all(), "%s has non-finite values" % name
    assert off.max() <= 0, "%s: off by %.3e where %.3e is allowed" % (name, np.abs(got - want).flat[off.argmax()], bound.flat[off.argmax()])


def _check(c):
    half = HALF[c.dtype]
    x = c.host(c.qkv, c.width)
    inside = slice(c.starts[0], c.starts[-1])
    c.forward()
    torch.cuda.synchronize()
    O, lse, mag = opacked.attention_fwd(x, c.starts, c.heads, c.kv_heads, c.d, c.causal, c.scale)
    _within("O", c.host(c.O, c.o_width)[inside], O[inside], (half * (np.abs(O) + mag) + FP32 * mag)[inside])
    got = c.lse.double().cpu().numpy()
    _within("lse", got[:, inside], lse[:, inside], FP32 * (1 + np.abs(lse[:, inside])))
    assert (got[:, :inside.start] == MARK).all() and (got[:, inside.stop:] == MARK).all()
    assert c.untouched(c.O, c.o_width)
    # the backward as a function of what it is given: the forward's own O and lse
    c.backward()
    torch.cuda.synchronize()
    grad, weighted, parts = opacked.attention_bwd(x, c.host(c.O, c.o_width), c.host(c.dO, c.o_width), got, c.starts, c.heads, c.kv_heads, c.d, c.causal, c.scale)
    _within("dqkv", c.host(c.dqkv, c.width)[inside], grad[inside], (half * (np.abs(grad) + weighted) + FP32 * parts)[inside])
    assert c.untouched(c.dqkv, c.width)


HEADS = [(4, 4, 64), (4, 2, 64), (5, 1, 64), (8, 1, 128), (12, 4, 128), (3, 3, 104), (6, 2, 32), (2, 2, 8), (4, 1, 40), (2, 1, 72)]
LENGTHS = [[1], [0, 1, 0, 2], [63, 64, 65], [127, 128, 129, 1], [300, 5, 0, 513], [31, 32, 33, 95, 96, 97, 16, 17]]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("heads,kv_heads,d", HEADS)
def test_bf16_attention(heads, kv_heads, d, lengths, causal):
    print("packed", heads, kv_heads, d, lengths, causal, flush=True)
    _check(Packed("bf16", heads, kv_heads, d, causal, lengths, seed=d + len(lengths)))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 2, 64), (3, 3, 24), (2, 1, 100), (5, 1, 7), (4, 4, 128)])
def test_f32_attention(heads, kv_heads, d, lengths, causal):
    print("packed f32", heads, kv_heads, d, lengths, causal, flush=True)
    _check(Packed("f32", heads, kv_heads, d, causal, lengths, seed=d + len(lengths)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 2, 64), (4, 1, 128), (2, 2, 40)])
def test_rows_and_columns_that_belong_to_no_sample_stay_as_they_are(heads, kv_heads, d, causal, dtype):
    _check(Packed(dtype, heads, kv_heads, d, causal, [130, 0, 70, 1], before=3, behind=61, gap=24))


@pytest.mark.parametrize("heads,kv_heads,d", [(4, 2, 64), (4, 1, 128)])
def test_a_scale_of_the_caller_s_and_sharp_scores(heads, kv_heads, d):
    """Scores of standard deviation 6: rows where one key takes nearly all, and a maximum that moves from tile to tile."""
    _check(Packed("bf16", heads, kv_heads, d, True, [333, 100], scale=6 / math.sqrt(d)))
    _check(Packed("f32", heads, kv_heads, d, False, [333, 100], scale=0.37))


@pytest.mark.parametrize("dtype,d", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_the_smallest_scale(dtype, d):
    """Scores of nearly zero: every key counts alike, and the gradients of the scores' factors are of the scale's size."""
    _check(Packed(dtype, 4, 2, d, True, [333, 100], scale=1e-30))


@pytest.mark.parametrize("dtype,heads,kv_heads,d", [("bf16", 16, 1, 128), ("bf16", 16, 1, 64), ("bf16", 10, 2, 24), ("f32", 8, 1, 64), ("f32", 6, 1, 50)])
@pytest.mark.parametrize("causal", [True, False])
def test_walks_in_pieces(dtype, heads, kv_heads, d, causal):
    """Few keys under many heads: their queries are cut into pieces whose sums are joined."""
    c = Packed(dtype, heads, kv_heads, d, causal, [700, 3, 260], gap=8)
    assert c.desc.joins > 0
    _check(c)


def test_long_samples():
    _check(Packed("bf16", 2, 1, 128, True, [2500, 700]))
    _check(Packed("bf16", 2, 1, 64, False, [1, 2111]))


FULL = [700, 333, 129, 1, 600, 0, 260]                      # 20 tiles of 128 rows
FULLER = FULL + [640, 697, 512]                             # 35


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,heads,kv_heads,d,lengths", [
    ("bf16", 32, 8, 128, FULL), ("bf16", 32, 8, 104, FULL), ("bf16", 40, 8, 64, FULLER), ("bf16", 40, 8, 24, FULLER),
    ("bf16", 40, 1, 128, FULL), ("bf16", 80, 1, 64, FULL), ("f32", 16, 4, 64, FULL), ("f32", 16, 4, 100, FULL), ("f32", 16, 1, 40, FULL)])
def test_launches_that_fill_the_chip(dtype, heads, kv_heads, d, lengths, causal):
    """More blocks than compute units: 128 queries a block and a backward in two launches, where the small calls above split blocks and take one."""
    print("packed full", dtype, heads, kv_heads, d, causal, flush=True)
    c = Packed(dtype, heads, kv_heads, d, causal, lengths, before=2, behind=5, gap=8, seed=heads + d)
    tiles = sum((n + 127) // 128 for n in lengths)
    assert c.desc.tiles == tiles
    if dtype == "bf16":
        assert tiles * heads > 256 and tiles * (heads + kv_heads) > (1536 if d <= 64 else 768)
    assert kv_heads > 1 or c.desc.joins > 0
    _check(c)
    eager = [t.clone() for t in (c.O, c.lse, c.dqkv)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward(); c.backward()
    for _ in range(3):
        for t in (c.O, c.lse, c.dqkv):
            t.fill_(MARK)
        c.workspace.fill_(0xCD)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (c.O, c.lse, c.dqkv)))


def test_rows_far_apart_pass_32_bits():
    """Rows of 2 MiB: the samples lie behind 4 GiB, in the projection and in its gradient."""
    heads, kv_heads, d, pitch, first, lengths = 4, 2, 64, 1 << 20, 2090, [70, 30]
    rows = first + 100
    starts = _starts(lengths, first)
    desc = C.packed_desc(heads, kv_heads, d, True, C.BF16, rows, pitch)
    plan = C.cephalo_packed_plan(desc, starts).cuda()
    small = Packed("bf16", heads, kv_heads, d, True, lengths)
    small.forward(); small.backward()
    qkv, dqkv = (torch.empty(rows, pitch, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    qkv[first:, :small.width] = small.qkv
    O, dO, lse = torch.zeros(rows, heads * d, dtype=torch.bfloat16, device="cuda"), torch.zeros(rows, heads * d, dtype=torch.bfloat16, device="cuda"), torch.zeros(heads, rows, device="cuda")
    dO[first:] = small.dO
    workspace = torch.empty(C.cephalo_op_attention_packed_bwd_workspace(desc), dtype=torch.uint8, device="cuda")
    C.cephalo_op_attention_packed_fwd(desc, plan, qkv, O, lse)
    C.cephalo_op_attention_packed_bwd(desc, plan, qkv, O, dO, lse, dqkv, workspace)
    torch.cuda.synchronize()
    assert torch.equal(O[first:], small.O) and torch.equal(lse[:, first:], small.lse)
    assert torch.equal(dqkv[first:, :small.width], small.dqkv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_no_value_crosses_from_sample_to_sample(d, causal, dtype):
    """One sample of infinities and not-a-numbers: its neighbours' results keep their bits."""
    lengths, results = [100, 77, 130], []
    for bad in (False, True):
        c = Packed(dtype, 4, 2, d, causal, lengths)
        if bad:
            c.qkv[100:177] = float("nan")
            c.qkv[101:177:3] = float("inf")
            c.dO[100:177] = float("-inf")
        c.forward(); c.backward()
        results.append((c.O, c.lse.t().contiguous(), c.dqkv))
    torch.cuda.synchronize()
    for a, b in zip(*results):
        assert torch.equal(a[:100], b[:100]) and torch.equal(a[177:], b[177:])


def test_a_sample_among_others_is_the_sample_alone():
    """How the work is divided, and with it the order of additions, goes by all samples of a list: both results lie within the bounds that _check takes of the
    exact one, so they differ by at most the sum of the two."""
    for dtype in ("bf16", "f32"):
        alone = Packed(dtype, 4, 2, 64, True, [200], seed=3)
        among = Packed(dtype, 4, 2, 64, True, [7, 200, 300, 1], seed=4)
        among.qkv[7:207], among.dO[7:207] = alone.qkv, alone.dO
        for c in (alone, among):
            c.forward()
            c.backward()
        torch.cuda.synchronize()
        x, half = alone.host(alone.qkv, alone.width), HALF[dtype]
        O, lse, mag = opacked.attention_fwd(x, [0, 200], 4, 2, 64, True)
        off = half * (np.abs(O) + mag) + FP32 * mag
        _within("O", among.host(among.O, 256)[7:207], alone.host(alone.O, 256), 2 * off)
        # the gradients are functions of O too, which may differ by 2 off: rowsum(dO O) by sum |dO| 2 off, dS by P times that
        got = [c.lse.double().cpu().numpy() for c in (alone, among)]
        _within("lse", got[1][:, 7:207], got[0], 2 * FP32 * (1 + np.abs(lse)))
        grads = [opacked.attention_bwd(x, o, alone.host(alone.dO, 256), l, [0, 200], 4, 2, 64, True)
                 for o, l in ((alone.host(alone.O, 256), got[0]), (among.host(among.O, 256)[7:207], got[1][:, 7:207]))]
        bounds = [half * (np.abs(g) + w) + FP32 * p for g, w, p in grads]
        _within("dqkv", among.host(among.dqkv, 512)[7:207] - alone.host(alone.dqkv, 512), grads[1][0] - grads[0][0], bounds[0] + bounds[1])


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_the_same_bits_twice_and_under_a_captured_graph(dtype, d):
    c = Packed(dtype, 8, 2, d, True, [257, 1, 120])
    c.forward(); c.backward()
    torch.cuda.synchronize()
    first = [t.clone() for t in (c.O, c.lse, c.dqkv)]
    fresh = Packed(dtype, 8, 2, d, True, [257, 1, 120], seed=9)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward(); c.backward()
    inputs = [(c.qkv.clone(), c.dO.clone()), (fresh.qkv.clone(), fresh.dO.clone())]
    fresh.forward(); fresh.backward()
    torch.cuda.synchronize()
    second = [t.clone() for t in (fresh.O, fresh.lse, fresh.dqkv)]
    for k in (0, 1, 0, 1):
        c.qkv.copy_(inputs[k][0]); c.dO.copy_(inputs[k][1])
        for t in (c.O, c.lse, c.dqkv):
            t.fill_(MARK)
        c.workspace.fill_(0xCD)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((c.O, c.lse, c.dqkv), (first, second)[k]):
            assert torch.equal(got, want)
        float((c.dqkv.float() ** 2).sum())      # the program's own work between the replays


def test_on_a_stream_of_its_own():
    a, b = Packed("bf16", 4, 2, 64, True, [300, 20]), Packed("bf16", 4, 2, 64, True, [300, 20])
    a.forward(); a.backward()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.forward(stream=s); b.backward(stream=s)
    s.synchronize(); torch.cuda.synchronize()
    assert torch.equal(a.O, b.O) and torch.equal(a.dqkv, b.dqkv)


def test_a_list_of_other_samples_reaches_no_row_outside_the_buffers():
    """The list's entries are checked against the rows that the call names: of a longer set's list only what fits is done."""
    big = Packed("bf16", 4, 2, 64, True, [40, 500])
    c = Packed("bf16", 4, 2, 64, True, [40, 60])
    for field in ("longest", "tiles", "key_items", "joins", "slots", "plan_bytes"):
        setattr(c.desc, field, getattr(big.desc, field))
    c.desc.longest, c.plan = 60, big.plan
    c.workspace = torch.empty(C.cephalo_op_attention_packed_bwd_workspace(c.desc), dtype=torch.uint8, device="cuda")
    c.forward(); c.backward()
    torch.cuda.synchronize()
    alone = Packed("bf16", 4, 2, 64, True, [40, 60])
    alone.forward()
    torch.cuda.synchronize()
    assert torch.equal(c.O[:40], alone.O[:40]) and bool((c.O[40:] == MARK).all())


# ---- rotary axes ------------------------------------------------------------------------------------------------------------

# An angle's fraction of a turn is rounded to 24 bits (2^-25 of a turn: pi 2^-24), a sine or cosine is off by at most two steps (2^-23): 2^-21 of |even| + |odd| covers
# both, the products and the sum.
def _rotary(dtype, heads, d, dims, rows, inverse, gap=0, in_place=False, far=0, base=10000.0, seed=0):
    rng = np.random.default_rng(seed + rows)
    positions = rng.integers(0, 3000, (rows, len(dims))) + far
    x = torch.full((max(rows, 1), heads * d + gap), MARK, dtype=TORCH[dtype])
    x[:rows, :heads * d] = torch.from_numpy(rng.standard_normal((rows, heads * d))).to(TORCH[dtype])
    src = x.cuda()
    dst = src if in_place else torch.full_like(src, MARK)
    C.cephalo_op_rotary_axes(LIB[dtype], src, heads * d + gap, dst, heads * d + gap, torch.from_numpy(positions.astype(np.int32)).cuda(), rows, dims, heads, d, base, inverse)
    torch.cuda.synchronize()
    x = x.double().numpy()[:rows, :heads * d]
    want = opacked.rotary(x, positions, dims, heads, d, base, inverse)
    pairs = np.abs(x.reshape(-1, 2)).sum(1)[:, None].repeat(2, 1).reshape(x.shape)
    _within("rotary", dst.double().cpu().numpy()[:rows, :heads * d], want, HALF[dtype] * np.abs(want) + 2.0 ** -21 * pairs)
    assert (dst.float().cpu().numpy()[:, heads * d:] == MARK).all()
    turned = sum(dims)
    same = lambda t: t.reshape(rows, heads, d)[..., turned:]      # noqa: E731
    assert np.array_equal(same(dst.double().cpu().numpy()[:rows, :heads * d]), same(x))


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,d,dims", [(4, 64, [64]), (1, 8, [4, 4]), (25, 64, [22, 22, 20]), (40, 128, [32, 48, 48]), (3, 80, [40, 0, 20]), (7, 104, [52, 52]), (300, 32, [16, 16]), (2, 128, [2, 30])])
@pytest.mark.parametrize("rows", [1, 197])
def test_rotary_axes(heads, d, dims, rows, dtype, inverse):
    _rotary(dtype, heads, d, dims, rows, inverse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_in_place_with_gaps_and_at_far_positions(dtype):
    _rotary(dtype, 6, 64, [20, 22, 22], 133, False, gap=40, in_place=True)
    _rotary(dtype, 6, 64, [64], 50, True, far=2 ** 31 - 4000)
    _rotary(dtype, 6, 64, [32, 32], 50, False, far=-700000, base=500000.0)
    _rotary(dtype, 3, 64, [64], 20011, False)


def test_columns_that_are_not_turned_keep_infinities_to_themselves():
    x = torch.ones(3, 16, device="cuda")
    x[:, 8] = float("inf"); x[1, 13] = float("nan")
    y = torch.empty_like(x)
    C.cephalo_op_rotary_axes(C.F32, x, 16, y, 16, torch.full((3, 1), 5, dtype=torch.int32, device="cuda"), 3, [8], 1, 16)
    torch.cuda.synchronize()
    assert torch.equal(y[:, 8:].nan_to_num(3.0), x[:, 8:].nan_to_num(3.0)) and torch.isfinite(y[:, :8]).all()


# ---- dropout ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 2047, 2048, 2056, 131 * 257])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999])
def test_dropout(dtype, n, p):
    seed, first = 0x9ABCDEF012345678, 8 * (2 ** 33 + 5)
    rng = np.random.default_rng(n)
    branch = torch.from_numpy(rng.standard_normal(n)).to(TORCH[dtype]).cuda()
    resid, dy = (torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda() for _ in range(2))
    out, dbranch = torch.full((n + 8,), MARK, device="cuda"), torch.full((n + 8,), MARK, dtype=TORCH[dtype], device="cuda")
    C.cephalo_op_dropout_add(LIB[dtype], branch, resid, out, n, p, seed, first)
    C.cephalo_op_dropout_bwd(LIB[dtype], dy, dbranch, n, p, seed, first)
    torch.cuda.synchronize()
    factor = opacked.dropout_factors(n, p, seed, first)
    got, back = out.double().cpu().numpy(), dbranch.double().cpu().numpy()
    b, r, g = (t.double().cpu().numpy() for t in (branch, resid, dy))
    # the scale, the product and the sum are rounded to 24 bits each, the gradient's product to the branch's type
    _within("out", got[:n], r + factor * b, 2.0 ** -24 * (np.abs(r + factor * b) + 2 * np.abs(factor * b)) * 1.01)
    _within("dbranch", back[:n], factor * g, (HALF[dtype] + 2.0 ** -23) * np.abs(factor * g) * 1.01)
    assert ((got[:n] == r) >= (factor == 0)).all() and (back[:n][factor == 0] == 0).all()
    assert (got[n:] == MARK).all() and (back[n:] == MARK).all()


def test_dropped_elements_may_hold_anything_and_out_may_be_resid():
    n, seed = 4096, 77
    factor = torch.from_numpy(opacked.dropout_factors(n, 0.5, seed)).cuda()
    branch, resid = torch.ones(n, device="cuda"), torch.randn(n, device="cuda")
    branch[factor == 0] = float("nan")
    want = resid + (factor > 0) * 2.0
    C.cephalo_op_dropout_add(C.F32, branch, resid, resid, n, 0.5, seed)
    torch.cuda.synchronize()
    assert torch.equal(resid, want)


def test_parts_of_a_tensor_drop_what_one_call_drops_and_a_counter_moves_the_words():
    n, seed = 5000, 5
    x = torch.randn(n, device="cuda")
    whole, parts, moved = (torch.empty(n, device="cuda") for _ in range(3))
    C.cephalo_op_dropout_bwd(C.F32, x, whole, n, 0.3, seed, 800)
    C.cephalo_op_dropout_bwd(C.F32, x[:1600], parts[:1600], 1600, 0.3, seed, 800)
    C.cephalo_op_dropout_bwd(C.F32, x[1600:], parts[1600:], n - 1600, 0.3, seed, 2400)
    counter = torch.tensor([0], device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        C.cephalo_op_dropout_bwd(C.F32, x, moved, n, 0.3, seed, 0, counter)
    torch.cuda.synchronize()
    assert torch.equal(whole, parts)
    for at in (800, 16, 800, 2 ** 40):
        counter.fill_(at)
        graph.replay()
        torch.cuda.synchronize()
        want = torch.from_numpy(opacked.dropout_factors(n, 0.3, seed, at)).cuda()
        assert torch.equal(moved != 0, want > 0) and (at != 800 or torch.equal(moved, whole))


# ---- together ---------------------------------------------------------------------------------------------------------------

def test_the_attention_half_of_a_layer_forward_and_backward():
    """qkv -> rotary -> attention -> projection -> dropout -> residual, and all the way back, on packed samples in fp32, against the oracle chained in 64 bits.

    The framework's own fp32 tolerance: 1e-4 of the largest value and, on average, of the average one."""
    heads, kv_heads, d, lengths, H = 6, 2, 32, [50, 1, 129], 192
    starts, rows, width, p, seed = _starts(lengths), sum(lengths), (6 + 4) * 32, 0.2, 31
    dims, rng = [16, 8, 8], np.random.default_rng(0)
    f32 = lambda *shape: rng.standard_normal(shape).astype(np.float32)      # noqa: E731
    qkv, W, resid, dy, positions = f32(rows, width), f32(H, heads * d) * 0.1, f32(rows, H), f32(rows, H), rng.integers(0, 40, (rows, 3)).astype(np.int32)
    g = {k: torch.from_numpy(v).cuda() for k, v in dict(qkv=qkv, W=W, resid=resid, dy=dy, positions=positions).items()}
    new = lambda *shape: torch.full(shape, MARK, device="cuda")      # noqa: E731
    desc = C.packed_desc(heads, kv_heads, d, True, C.F32, rows)
    plan = C.cephalo_packed_plan(desc, starts).cuda()
    turned, O, lse, branch, out = g["qkv"].clone(), new(rows, heads * d), new(heads, rows), new(rows, H), new(rows, H)
    turn = lambda t, inverse: C.cephalo_op_rotary_axes(C.F32, t, width, t, width, g["positions"], rows, dims, heads + kv_heads, d, 10000.0, inverse)      # noqa: E731
    turn(turned, False)
    C.cephalo_op_attention_packed_fwd(desc, plan, turned, O, lse)
    C.cephalo_op_gemm(C.F32, O, heads * d, 1, g["W"], heads * d, 1, rows, H, heads * d, C.EPI_NONE, branch)
    C.cephalo_op_dropout_add(C.F32, branch, g["resid"], out, rows * H, p, seed)
    dbranch, dO, dqkv = new(rows, H), new(rows, heads * d), new(rows, width)
    C.cephalo_op_dropout_bwd(C.F32, g["dy"], dbranch, rows * H, p, seed)
    C.cephalo_op_gemm(C.F32, dbranch, H, 1, g["W"], 1, heads * d, rows, heads * d, H, C.EPI_NONE, dO)
    workspace = torch.empty(C.cephalo_op_attention_packed_bwd_workspace(desc), dtype=torch.uint8, device="cuda")
    C.cephalo_op_attention_packed_bwd(desc, plan, turned, O, dO, lse, dqkv, workspace)
    turn(dqkv, True)
    torch.cuda.synchronize()

    q64 = qkv.astype(np.float64)
    n = (heads + kv_heads) * d
    t64 = np.concatenate([opacked.rotary(q64[:, :n], positions, dims, heads + kv_heads, d), q64[:, n:]], axis=1)
    O64, lse64, _ = opacked.attention_fwd(t64, starts, heads, kv_heads, d, True)
    factor = opacked.dropout_factors(rows * H, p, seed).reshape(rows, H)
    out64 = resid + factor * (O64 @ W.astype(np.float64).T)
    grad, _, _ = opacked.attention_bwd(t64, O64, (factor * dy) @ W.astype(np.float64), lse64, starts, heads, kv_heads, d, True)
    grad = np.concatenate([opacked.rotary(grad[:, :n], positions, dims, heads + kv_heads, d, inverse=True), grad[:, n:]], axis=1)
    for name, got, want in (("out", out, out64), ("dqkv", dqkv, grad)):
        off = np.abs(got.double().cpu().numpy() - want)
        assert off.max() <= 1e-4 * np.abs(want).max() and off.mean() <= 1e-4 * np.abs(want).mean(), (name, off.max(), off.mean())


# ---- the largest score ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,heads,kv_heads,d,rows", [("bf16", 2, 1, 32, 150), ("bf16", 2, 1, 64, 150), ("bf16", 2, 2, 128, 150), ("bf16", 40, 10, 64, 1100), ("bf16", 20, 5, 128, 1100), ("f32", 2, 1, 64, 150)])
@pytest.mark.parametrize("causal", [True, False])
def test_the_largest_score_in_any_place_of_a_tile(dtype, heads, kv_heads, d, rows, causal):
    """One key whose score is 300 above all others', in each place of 16 and in several tiles: rows that see it take its values.  (Weights e^-300: zero in 32 bits.)"""
    for place in list(range(16)) + [16 + 5, 64 + 12, 128 + 3]:
        c = Packed(dtype, heads, kv_heads, d, causal, [rows], scale=1.0)
        x = torch.zeros(rows, heads + 2 * kv_heads, d, dtype=TORCH[dtype], device="cuda")
        x[:, :heads, 3], x[place, heads:heads + kv_heads, 3] = 20, 15
        x[:, heads + kv_heads:] = c.qkv.reshape(rows, -1, d)[:, heads + kv_heads:]
        c.qkv[:] = x.reshape(rows, -1)
        c.forward()
        torch.cuda.synchronize()
        see = range(place, rows) if causal else range(rows)
        want = x[place, heads + kv_heads:].repeat_interleave(heads // kv_heads, 0).reshape(-1)
        assert torch.equal(c.O[see.start:], want.expand(len(see), -1)), (place, dtype)
        assert (c.lse[:, see.start:] - 300).abs().max() <= 300 * FP32, place
        assert torch.isfinite(c.O.float()).all() and (c.lse[:, :see.start] < 10).all()


# ---- scores far from zero -----------------------------------------------------------------------------------------------------

# Whole numbers: every product and every partial sum below 2^24 is exact, so the scores are what the definition says and rows have ties.  What is left of the error: the
# scale times log2(e) is off by 2^-23 of itself, which counts on differences of scores that matter (below 64 in the exponent), and lse is rounded three times.
def _whole(dtype, heads, kv_heads, d, causal, lengths, scale, most=3, seed=0):
    c = Packed(dtype, heads, kv_heads, d, causal, lengths, scale=scale, seed=seed)
    c.scale = float(np.float32(scale))
    rng = np.random.default_rng(seed)
    c.qkv[:, :(heads + kv_heads) * d] = torch.from_numpy(rng.integers(-most, most + 1, (c.rows, (heads + kv_heads) * d))).to(TORCH[dtype]).cuda()
    return c


def _check_forward(c):
    c.forward()
    torch.cuda.synchronize()
    O, lse, mag = opacked.attention_fwd(c.host(c.qkv, c.width), c.starts, c.heads, c.kv_heads, c.d, c.causal, c.scale)
    _within("O", c.host(c.O, c.o_width), O, HALF[c.dtype] * (np.abs(O) + mag) + FP32 * mag)
    _within("lse", c.lse.double().cpu().numpy(), lse, FP32 * (1 + np.abs(lse)))


@pytest.mark.parametrize("dtype,heads,kv_heads,d,lengths", [("bf16", 4, 2, 64, [333, 100]), ("bf16", 4, 2, 128, [333, 100]), ("bf16", 4, 2, 24, [333, 100]), ("bf16", 20, 5, 64, FULL),
                                                            ("bf16", 16, 4, 128, FULL), ("f32", 4, 2, 64, [333, 100]), ("f32", 2, 1, 100, [200])])
@pytest.mark.parametrize("scale", [1e3, 1e6, 3e7, 1e9, 1e20, 1e30])
def test_the_forward_at_any_finite_scores(dtype, heads, kv_heads, d, lengths, scale):
    """Rows where the keys of the largest score share the weight, exactly."""
    for causal in (True, False):
        _check_forward(_whole(dtype, heads, kv_heads, d, causal, lengths, scale))


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_the_forward_of_large_queries_and_keys(dtype, d):
    """The default scale, scores up to 1e30."""
    for size in (2.0 ** 12, 2.0 ** 20, 2.0 ** 45):
        c = _whole(dtype, 4, 2, d, True, [333, 100], 0.0)
        c.scale = 1 / math.sqrt(d)
        c.qkv[:, :(4 + 2) * d] *= size
        _check_forward(c)


@pytest.mark.parametrize("dtype,heads,kv_heads,d", [("bf16", 4, 2, 64), ("bf16", 40, 4, 64), ("bf16", 4, 2, 128), ("bf16", 16, 4, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("offset,scale", [(0x58B902, 2.0), (1 << 23, 2.0), (-(1 << 23), 2.0), (0x5C5D00, 0.25), (0x58B902, 64.0), (-0x58B902, 64.0)])
def test_weights_of_scores_that_lie_close_together_far_from_zero(dtype, heads, kv_heads, d, offset, scale):
    """Scores of offset + small whole numbers that rise along the keys (causal rows raise their maximum on the way), weights of more than one key in a row."""
    c = _whole(dtype, heads, kv_heads, d, True, [700, 90] if heads < 16 else FULL, scale, most=1)
    n, sign = heads + kv_heads, 1 if offset > 0 else -1
    x = torch.zeros(c.rows, n, d, dtype=TORCH[dtype])
    digits = [abs(offset) >> 16, abs(offset) >> 8 & 255, abs(offset) & 255]
    for j, v in enumerate(digits):                         # offset = sum of digit * 256^j: 256 * (digit * 256), 16 * (digit * 16), 1 * digit
        x[:, :heads, j], x[:, heads:, j] = (256, 16, 1)[j], sign * v * (256, 16, 1)[j]
    x[:, :heads, 3] = 1
    rng = np.random.default_rng(5)
    x[:, heads:, 3] = torch.from_numpy(np.minimum(np.arange(c.rows) // 8, 100)[:, None] + rng.integers(-3, 4, (c.rows, kv_heads))).to(TORCH[dtype])
    c.qkv[:, :n * d] = x.reshape(c.rows, n * d).cuda()
    _check_forward(c)


def _check_sharp(c):
    """Of forward and backward at large scores: every weight may carry the factor exp(w), w = (d + 8) 2^-24 s, s the larger of |lse| and the scale times sum |q| |k|.  (A score is a sum of d
    terms and at most four more, -lse / scale and the roundings of scale log2(e) and of lse log2(e) among them, each rounded to 2^-24 of at most 2 s.)  What lies below 2^-126 may count as zero: a weight, a dS, one of n products or of their sums, each times what follows it."""
    x, half = c.host(c.qkv, c.width), HALF[c.dtype]
    c.forward(); c.backward()
    torch.cuda.synchronize()
    O, lse, mag = opacked.attention_fwd(x, c.starts, c.heads, c.kv_heads, c.d, c.causal, c.scale)
    r = np.abs(x).reshape(c.rows, c.heads + 2 * c.kv_heads, c.d)
    s = max(np.abs(lse).max(), c.scale * max((r[:, a] @ r[:, c.heads + a * c.kv_heads // c.heads].T).max() for a in range(c.heads)))
    w = math.expm1((c.d + 8) * 2.0 ** -24 * s)
    dO, X = c.host(c.dO, c.o_width), np.abs(x).max()
    dP = 2 * c.d * np.abs(dO).max() * X
    zero = 2 * 2.0 ** -126 * c.rows * (c.heads // c.kv_heads)
    _within("O", c.host(c.O, c.o_width), O, half * (np.abs(O) + mag) + (FP32 + 2 * w) * mag + zero * (X + 1))
    got = c.lse.double().cpu().numpy()
    _within("lse", got, lse, FP32 + w + 2.0 ** -22 * s)
    grad, weighted, parts = opacked.attention_bwd(x, c.host(c.O, c.o_width), dO, got, c.starts, c.heads, c.kv_heads, c.d, c.causal, c.scale)
    zero *= np.abs(dO).max() + 1 + c.scale * (dP * X + X + 1)
    _within("dqkv", c.host(c.dqkv, c.width), grad, half * (np.abs(grad) + weighted) + (FP32 + 2 * w) * parts + zero)
    return zero / np.abs(grad).max(), w


@pytest.mark.parametrize("dtype,heads,kv_heads,d,lengths", [("bf16", 4, 2, 32, [333, 100]), ("bf16", 4, 2, 64, [333, 100]), ("bf16", 4, 2, 128, [333, 100]), ("bf16", 40, 8, 64, FULLER),
                                                            ("bf16", 32, 8, 128, FULL), ("f32", 4, 2, 64, [333, 100]), ("f32", 4, 2, 100, [333, 100])])
@pytest.mark.parametrize("scale", [1.0, 16.0, 128.0])
def test_gradients_at_large_scores_keep_the_stated_accuracy(dtype, heads, kv_heads, d, lengths, scale):
    for causal in (True, False):
        _check_sharp(Packed(dtype, heads, kv_heads, d, causal, lengths, scale=scale))


@pytest.mark.parametrize("dtype,heads,kv_heads,d,lengths", [("bf16", 4, 2, 32, [333, 100]), ("bf16", 4, 2, 64, [333, 100]), ("bf16", 4, 2, 128, [333, 100]), ("bf16", 40, 8, 64, FULLER),
                                                            ("bf16", 32, 8, 128, FULL), ("f32", 4, 2, 64, [333, 100]), ("f32", 4, 2, 100, [333, 100])])
@pytest.mark.parametrize("scale,std", [(float(np.float32(1e30)), 1e-15), (float(np.float32(1e-30)), 1e15), (1e6, 1e-3)])
def test_both_ends_of_the_scale_with_ordinary_scores(dtype, heads, kv_heads, d, lengths, scale, std):
    """Queries, keys and values of a size that brings the scores back to ordinary ones."""
    zero, w = _check_sharp(Packed(dtype, heads, kv_heads, d, True, lengths, scale=float(np.float32(scale)), std=std))
    assert zero < 1e-4 and w < 1e-2


@pytest.mark.parametrize("dtype,heads,kv_heads,d,lengths", [("bf16", 4, 2, 32, [333, 100]), ("bf16", 4, 2, 64, [333, 100]), ("bf16", 4, 2, 104, [333, 100]), ("bf16", 40, 8, 64, FULLER),
                                                            ("bf16", 32, 8, 128, FULL), ("f32", 4, 2, 64, [333, 100]), ("f32", 4, 2, 80, [333, 100])])
def test_hidden_keys_with_scores_beyond_any_that_a_row_sees(dtype, heads, kv_heads, d, lengths):
    """Every 17th key forty times as long: a row before it, which does not see it, would give it a weight that 32 bits do not hold."""
    for causal in (True, False):
        c = Packed(dtype, heads, kv_heads, d, causal, lengths, scale=1.0)
        c.qkv[5::17, heads * d:(heads + kv_heads) * d] *= 40
        _check_sharp(c)


# ---- forms that the cases above do not reach ----------------------------------------------------------------------------------

@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,d,lengths", [(4, 2, 72, LENGTHS[2]), (4, 2, 80, LENGTHS[3]), (4, 4, 96, LENGTHS[4]), (5, 1, 90, LENGTHS[5]), (4, 2, 65, LENGTHS[1]), (2, 1, 80, [1]),
                                                      (8, 1, 80, [700, 3, 260]), (8, 1, 66, [700, 3, 260]), (16, 4, 80, FULL), (16, 4, 90, FULL)])
def test_f32_heads_of_65_to_96(heads, kv_heads, d, lengths, causal):
    """The width between: eight wavefronts a block, places of the workspace 128 wide."""
    print("packed f32", heads, kv_heads, d, lengths, causal, flush=True)
    c = Packed("f32", heads, kv_heads, d, causal, lengths, before=1, behind=3, gap=5 if d % 2 else 4, seed=d)
    assert kv_heads > 1 or max(lengths) < 700 or c.desc.joins > 0
    _check(c)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,heads,d,dims,rows", [("bf16", 40, 128, [32, 48, 48], 3301), ("f32", 25, 64, [22, 22, 20], 5301)])
def test_rotary_results_that_go_past_the_caches(dtype, heads, d, dims, rows, in_place):
    """Above 32 MiB."""
    assert rows * heads * d * (2 if dtype == "bf16" else 4) > 32 << 20
    _rotary(dtype, heads, d, dims, rows, in_place, gap=16, in_place=in_place)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropout_results_that_go_past_the_caches(dtype):
    n, p, seed, first = (1 << 24) + 6149, 0.3, 12345, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    branch = torch.randn(n, generator=g, device="cuda").to(TORCH[dtype])
    resid, dy = (torch.randn(n, generator=g, device="cuda") for _ in range(2))
    out, dbranch = torch.full((n + 8,), MARK, device="cuda"), torch.full((n + 8,), MARK, dtype=TORCH[dtype], device="cuda")
    assert out.numel() * 4 > 32 << 20 and dbranch.numel() * dbranch.element_size() > 32 << 20
    C.cephalo_op_dropout_add(LIB[dtype], branch, resid, out, n, p, seed, first)
    C.cephalo_op_dropout_bwd(LIB[dtype], dy, dbranch, n, p, seed, first)
    torch.cuda.synchronize()
    factor = torch.from_numpy(opacked.dropout_factors(n, p, seed, first)).cuda()
    for got, want, bound in ((out, resid + factor * branch.double(), 2.0 ** -24 * ((resid + factor * branch.double()).abs() + 2 * (factor * branch.double()).abs())),
                             (dbranch, factor * dy.double(), (HALF[dtype] + 2.0 ** -23) * (factor * dy.double()).abs())):
        assert bool(((got[:n].double() - want).abs() <= bound * 1.01).all()) and bool((got[n:] == MARK).all())
    assert bool((out[:n][factor == 0] == resid[factor == 0]).all()) and bool((dbranch[:n][factor == 0] == 0).all())
    out[:n] = resid
    C.cephalo_op_dropout_add(LIB[dtype], branch, out, out, n, p, seed, first)
    again = torch.empty(n, device="cuda")
    C.cephalo_op_dropout_add(LIB[dtype], branch, resid, again, n, p, seed, first)
    torch.cuda.synchronize()
    assert torch.equal(out[:n], again)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("bf16", 24), ("f32", 64), ("f32", 80), ("f32", 100)])
@pytest.mark.parametrize("causal", [True, False])
def test_a_list_of_other_samples_writes_nothing_but_the_samples_that_fit(dtype, d, causal):
    """A longer set's list, with joins: the sample that both sets begin with is done, forward and backward, and no other row is written, neither behind the buffers' rows nor in them."""
    heads, kv_heads, behind = 16, 1, 700
    big, small = (Packed(dtype, heads, kv_heads, d, causal, [300, n], seed=1) for n in (500, 60))
    c = Packed(dtype, heads, kv_heads, d, causal, [300, 60], behind=behind, seed=1)
    c.desc, c.plan = small.desc, big.plan                 # 360 rows
    for field in ("tiles", "key_items", "joins", "slots", "plan_bytes"):
        setattr(c.desc, field, getattr(big.desc, field))
    assert c.desc.joins > 0 and c.desc.tokens == 360 and c.rows == 360 + behind
    c.lse = torch.full((heads * 360 + 4096,), MARK, device="cuda")
    need = C.cephalo_op_attention_packed_bwd_workspace(c.desc)
    c.workspace = torch.full((need + 65536,), 0xAB, dtype=torch.uint8, device="cuda")
    c.forward(); c.backward()
    torch.cuda.synchronize()
    assert bool((c.O[300:] == MARK).all()) and bool((c.dqkv[300:] == MARK).all()) and bool((c.workspace[need:] == 0xAB).all())
    lse = c.lse[:heads * 360].reshape(heads, 360)
    assert bool((lse[:, 300:] == MARK).all()) and bool((c.lse[heads * 360:] == MARK).all())
    x, half = c.host(c.qkv, c.width)[:300], HALF[dtype]
    O, want, mag = opacked.attention_fwd(x, [0, 300], heads, kv_heads, d, causal)
    _within("O", c.host(c.O, c.o_width)[:300], O, half * (np.abs(O) + mag) + FP32 * mag)
    got = lse[:, :300].double().cpu().numpy()
    _within("lse", got, want, FP32 * (1 + np.abs(want)))
    grad, weighted, parts = opacked.attention_bwd(x, c.host(c.O, c.o_width)[:300], c.host(c.dO, c.o_width)[:300], got, [0, 300], heads, kv_heads, d, causal)
    _within("dqkv", c.host(c.dqkv, c.width)[:300], grad, half * (np.abs(grad) + weighted) + FP32 * parts)


# ---- views ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_attention_on_columns_of_wider_tensors(dtype, d):
    c, v = (Packed(dtype, 4, 2, d, True, [130, 0, 70, 1], before=3, behind=6) for _ in range(2))
    c.forward(); c.backward()
    wide = {n: torch.full((c.rows + 2, getattr(c, n).shape[1] + 48), MARK, dtype=TORCH[dtype], device="cuda") for n in ("qkv", "O", "dO", "dqkv")}
    part = {n: t[1:-1, 16:-32] for n, t in wide.items()}
    part["qkv"].copy_(c.qkv); part["dO"].copy_(c.dO)
    v.desc.qkv_pitch, v.desc.o_pitch = wide["qkv"].stride(0), wide["O"].stride(0)
    for n in wide:
        setattr(v, n, part[n].unflatten(1, (-1, d)) if n == "O" else part[n])
    v.forward(); v.backward()
    torch.cuda.synchronize()
    assert torch.equal(part["O"], c.O) and torch.equal(v.lse, c.lse) and torch.equal(part["dqkv"], c.dqkv)
    for n, t in wide.items():
        assert bool((t[0] == MARK).all()) and bool((t[-1] == MARK).all()) and bool((t[:, :16] == MARK).all()) and bool((t[:, -32:] == MARK).all()), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_on_the_keys_of_a_projection_in_place(dtype):
    heads, kv_heads, d, rows = 4, 2, 64, 77
    qkv = torch.randn(rows, (heads + 2 * kv_heads) * d, device="cuda").to(TORCH[dtype])
    positions = torch.arange(rows, dtype=torch.int32, device="cuda")[:, None].contiguous()
    keys, before = qkv[:, heads * d:(heads + kv_heads) * d], qkv.clone()
    want = torch.empty(rows, kv_heads * d, dtype=TORCH[dtype], device="cuda")
    C.cephalo_op_rotary_axes(LIB[dtype], keys.contiguous(), kv_heads * d, want, kv_heads * d, positions, rows, [64], kv_heads, d)
    C.cephalo_op_rotary_axes(LIB[dtype], keys, qkv.stride(0), keys, qkv.stride(0), positions, rows, [64], kv_heads, d)
    torch.cuda.synchronize()
    assert torch.equal(keys, want)
    assert torch.equal(qkv[:, :heads * d], before[:, :heads * d]) and torch.equal(qkv[:, (heads + kv_heads) * d:], before[:, (heads + kv_heads) * d:])


def test_views_that_do_not_cover_the_rows_are_refused():
    x = torch.zeros(8, 48, device="cuda")
    p = torch.zeros(8, 1, dtype=torch.int32, device="cuda")
    call = lambda src, rows=8, pitch=48: C.cephalo_op_rotary_axes(C.F32, src, pitch, src, pitch, p, rows, [16], 1, 16)      # noqa: E731
    call(x[:, 16:32]); call(x[:, 32:]); call(x[1:, 32:], rows=7); call(x[:, 16:32], rows=1); call(x[:, 16:32], rows=0)
    for bad in (lambda: call(x[:, 16:31]), lambda: call(x[:7, 16:32]), lambda: call(x[:, 16:32], pitch=40), lambda: call(x[::2, 16:32], rows=4), lambda: call(x.t()[16:32].t()[:, ::2]),
                lambda: call(x[:, 16:32].double()), lambda: call(x.cpu()[:, 16:32])):
        with pytest.raises(C.CephaloError, match="expected"):
            bad()
    torch.cuda.synchronize()


# ---- side by side and captured ------------------------------------------------------------------------------------------------

def test_calls_on_two_streams_at_once():
    """Different samples, a workspace and a plan of their own: what each gives is what it gives alone."""
    cases = [Packed("bf16", 16, 4, 64, True, FULL, seed=1), Packed("bf16", 8, 2, 128, False, [257, 1, 120], seed=2)]
    want = []
    for c in cases:
        c.forward(); c.backward()
        torch.cuda.synchronize()
        want.append([t.clone() for t in (c.O, c.lse, c.dqkv)])
        for t in (c.O, c.lse, c.dqkv):
            t.fill_(MARK)
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(cases, streams):
            c.forward(stream=s); c.backward(stream=s)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert all(torch.equal(a, b) for a, b in zip(w, (c.O, c.lse, c.dqkv)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_operators_together_in_a_graph_with_the_program_s_work_between_replays(dtype):
    """Rotary, attention, dropout and the way back; new inputs and new words at each replay, against the same calls made eagerly."""
    heads, kv_heads, d, lengths, p, seed = 8, 2, 64, [130, 1, 77], 0.25, 5
    c = Packed(dtype, heads, kv_heads, d, True, lengths)
    rows, turned, back = c.rows, torch.empty_like(c.qkv), torch.empty_like(c.qkv)
    positions = torch.stack([torch.arange(rows), torch.arange(rows) // 7], 1).to(torch.int32).cuda()
    resid = torch.randn(rows, heads * d, device="cuda")
    out, counter = torch.empty_like(resid), torch.zeros(1, dtype=torch.int64, device="cuda")
    source, n = c.qkv.clone(), rows * heads * d
    c.qkv = turned
    dy = torch.randn(rows, heads * d, device="cuda")

    def step():
        turned.copy_(source)
        C.cephalo_op_rotary_axes(LIB[dtype], turned, c.width, turned, c.width, positions, rows, [32, 32], heads + kv_heads, d)
        c.forward()
        C.cephalo_op_dropout_add(LIB[dtype], c.O, resid, out, n, p, seed, 0, counter)
        C.cephalo_op_dropout_bwd(LIB[dtype], dy, c.dO, n, p, seed, 0, counter)
        c.backward()
        back.copy_(c.dqkv)
        C.cephalo_op_rotary_axes(LIB[dtype], back, c.width, back, c.width, positions, rows, [32, 32], heads + kv_heads, d, inverse=True)

    inputs, results = [torch.randn(rows, c.width, device="cuda").to(TORCH[dtype]) for _ in range(3)], []
    for k, x in enumerate(inputs):
        source.copy_(x); counter.fill_(800 * k)
        step()
        torch.cuda.synchronize()
        results.append([t.clone() for t in (out, c.dO, back)])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in (0, 1, 2, 1, 0):
        source.copy_(inputs[k]); counter.fill_(800 * k)
        for t in (out, c.dO, back, c.O, c.lse, c.dqkv):
            t.fill_(MARK)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results[k], (out, c.dO, back)))
        float((back.float() ** 2).sum())
    assert not torch.equal(results[0][1] != 0, results[1][1] != 0)
