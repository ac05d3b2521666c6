"""Pins of the oracle of packed attention, rotary axes and dropout; the work list; refusals.  Nothing here launches a kernel."""
import ctypes
import itertools

import numpy as np
import pytest
import torch

import paper_2411_01075_amd as C
from oracle import layer as olayer
from oracle import packed as opacked
from paper_2411_01075_amd import binding

FAKE = ctypes.c_void_p(0x1000)       # never dereferenced: validation fails first


def test_equal_heads_and_lengths_are_the_layer_s_attention():
    rng = np.random.default_rng(1)
    m, S, A, d = 2, 9, 3, 8
    x, dO = rng.standard_normal((m * S, 3 * A * d)), rng.standard_normal((m * S, A * d))
    for causal in (False, True):
        q, k, v = (olayer.split_heads(x.reshape(m, S, 3 * A * d)[..., i * A * d:(i + 1) * A * d], A) for i in range(3))
        want, P = olayer.attention_fwd(q, k, v, causal)
        O, lse, _ = opacked.attention_fwd(x, [0, S, 2 * S], A, A, d, causal)
        assert np.allclose(O, olayer.merge_heads(want).reshape(m * S, A * d), atol=1e-13)
        grads = olayer.attention_bwd(olayer.split_heads(dO.reshape(m, S, A * d), A), q, k, v, P)
        got, _, _ = opacked.attention_bwd(x, O, dO, lse, [0, S, 2 * S], A, A, d, causal)
        assert np.allclose(got, np.concatenate([olayer.merge_heads(t) for t in grads], axis=-1).reshape(m * S, 3 * A * d), atol=1e-12)


@pytest.mark.parametrize("heads,kv_heads,causal", [(4, 2, True), (3, 1, False), (2, 2, True)])
def test_gradients_are_the_definition_s_by_autograd_and_by_differences(heads, kv_heads, causal):
    rng = np.random.default_rng(heads)
    d, starts, n = 6, [1, 5, 5, 6, 13], 14
    x, dO = rng.standard_normal((n, (heads + 2 * kv_heads) * d)), rng.standard_normal((n, heads * d))
    O, lse, _ = opacked.attention_fwd(x, starts, heads, kv_heads, d, causal)
    grad, _, _ = opacked.attention_bwd(x, O, dO, lse, starts, heads, kv_heads, d, causal)
    t = torch.from_numpy(x).requires_grad_()
    w = t.reshape(n, -1, d)
    loss = torch.zeros((), dtype=torch.float64)
    for lo, hi in zip(starts, starts[1:]):
        if lo == hi:
            continue
        for a in range(heads):
            g = a // (heads // kv_heads)
            z = w[lo:hi, a] @ w[lo:hi, heads + g].T / d ** 0.5
            if causal:
                z = z + torch.full((hi - lo, hi - lo), -np.inf, dtype=torch.float64).triu(1)
            loss = loss + (torch.softmax(z, 1) @ w[lo:hi, heads + kv_heads + g] * torch.from_numpy(dO).reshape(n, heads, d)[lo:hi, a]).sum()
    loss.backward()
    assert np.allclose(grad, t.grad.numpy(), atol=1e-12)
    f = lambda y: (opacked.attention_fwd(y, starts, heads, kv_heads, d, causal)[0] * dO).sum()      # noqa: E731
    for _ in range(5):
        v = rng.standard_normal(x.shape)
        step = 1e-5
        assert abs((f(x + step * v) - f(x - step * v)) / (2 * step) - (grad * v).sum()) < 1e-7 * np.abs(grad * v).sum()


def test_rotary_turns_pairs_by_their_axis_and_back():
    rng = np.random.default_rng(2)
    x, pos = rng.standard_normal((5, 2 * 10)), rng.integers(0, 100, (5, 2))
    y = opacked.rotary(x, pos, [4, 2], 2, 10)
    assert np.allclose(opacked.rotary(y, pos, [4, 2], 2, 10, inverse=True), x, atol=1e-13)
    assert np.array_equal(y.reshape(5, 2, 10)[..., 6:], x.reshape(5, 2, 10)[..., 6:])
    angle = pos[3, 0] * 10000.0 ** (-2 / 4)
    e, o = x.reshape(5, 2, 10)[3, 1, 2:4]
    assert np.allclose(y.reshape(5, 2, 10)[3, 1, 2:4], [e * np.cos(angle) - o * np.sin(angle), e * np.sin(angle) + o * np.cos(angle)])
    assert np.allclose(y.reshape(5, 2, 10)[2, 0, 4], x.reshape(5, 2, 10)[2, 0, 4] * np.cos(pos[2, 1]) - x.reshape(5, 2, 10)[2, 0, 5] * np.sin(pos[2, 1]))


def test_words_are_the_published_generator_s():
    # the known answer for counter 0 and key 0
    assert [hex(v) for v in opacked.philox([0], 0)[0]] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    f = opacked.dropout_factors(1 << 16, 0.25, 12345)
    assert set(np.unique(f)) == {0.0, 65536 / 49152}
    assert abs((f > 0).mean() - 0.75) < 6 * np.sqrt(0.25 * 0.75 / f.size)
    assert np.array_equal(opacked.dropout_factors(40, 0.25, 12345, first=16), f[16:56])


# ---- the work list ----------------------------------------------------------------------------------------------------------

def _desc(heads=4, kv_heads=2, d=64, causal=True, dtype=C.BF16, tokens=1000, **kw):
    return C.packed_desc(heads, kv_heads, d, causal, dtype, tokens, **kw)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("starts", [[0, 1], [0, 0], [3, 3, 4, 200, 200, 328, 1000], [0, 128, 256, 1000], [7, 999]])
def test_the_list_holds_every_row_once_and_the_longest_work_first(starts, causal):
    d = _desc(causal=causal)
    plan = C.cephalo_packed_plan(d, starts).numpy()
    lengths = [b - a for a, b in zip(starts, starts[1:])]
    assert (d.samples, d.longest, d.tiles) == (len(lengths), max(lengths), sum((n + 127) // 128 for n in lengths))
    assert d.plan_bytes == 16 * d.tiles + 32 * (d.key_items + d.joins) <= binding.lib().cephalo_packed_plan_bytes(len(lengths), 1000)
    tiles, keys, joins = np.split(plan[:d.plan_bytes // 4], [4 * d.tiles, 4 * d.tiles + 8 * d.key_items])
    want = np.zeros(1000, dtype=int)
    want[starts[0]:starts[-1]] = 1
    seen = np.zeros(1000, dtype=int)
    tiles = tiles.reshape(-1, 4)
    for first, rows, tile, _ in tiles:
        assert first in starts and rows in lengths
        seen[first + tile * 128:min(first + rows, first + tile * 128 + 128)] += 1
    assert np.array_equal(seen, want)
    work = [tile if causal else rows for _, rows, tile, _ in tiles]
    assert work == sorted(work, reverse=True)


@pytest.mark.parametrize("dtype", [C.BF16, C.F32])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,d,starts", [(4, 2, 64, [0, 1]), (16, 1, 128, [0, 700, 700, 701, 1000]), (8, 8, 64, [5, 900]), (2, 1, 32, [0, 2, 100000]), (40, 8, 128, list(range(0, 64000, 37)))])
def test_the_walks_of_the_keys_cover_the_queries_once(heads, kv_heads, d, starts, causal, dtype):
    """Every 128 keys: their items' steps follow one another from 0 to the end, and where there are several each has a place of its own that the join adds in order."""
    desc = C.packed_desc(heads, kv_heads, d, causal, dtype, starts[-1] + 3)
    plan = C.cephalo_packed_plan(desc, starts).numpy()
    _, keys, joins = np.split(plan[:desc.plan_bytes // 4], [4 * desc.tiles, 4 * desc.tiles + 8 * desc.key_items])
    keys, joins = keys.reshape(-1, 8), joins.reshape(-1, 8)
    assert [int(e - b) for _, _, _, b, e, _, _, _ in keys] == sorted((int(e - b) for _, _, _, b, e, _, _, _ in keys), reverse=True)
    by_keys = {}
    for first, rows, tile, begin, end, slot, pieces, _ in keys.tolist():
        by_keys.setdefault((first, rows, tile), []).append((begin, end, slot, pieces))
    assert len(by_keys) == desc.tiles and len(joins) == desc.joins
    joined, used = {(f, r, t): (s, p) for f, r, t, _, _, s, p, _ in joins.tolist()}, set()
    for (first, rows, tile), items in by_keys.items():
        items.sort()
        steps = (rows - (tile * 128 if causal else 0) + 63) // 64 * (heads // kv_heads)
        assert items[0][0] == 0 and items[-1][1] == steps and all(a[1] == b[0] and a[0] < a[1] for a, b in zip(items, items[1:] + [(steps, 0, 0, 0)]))
        assert all(i[3] == len(items) for i in items)
        if len(items) == 1:
            assert items[0][2] == -1
        else:
            slots = [i[2] for i in items]
            assert joined.pop((first, rows, tile)) == (slots[0], len(items)) and slots == list(range(slots[0], slots[0] + len(items)))
            used.update(slots)
    assert not joined and used == set(range(desc.slots))


@pytest.mark.parametrize("dtype", [C.BF16, C.F32])
@pytest.mark.parametrize("d", [32, 128])
def test_the_pieces_of_any_list_have_room(d, dtype):
    """A list's buffer holds 512 pieces beyond one a tile: no set of samples takes more."""
    rng, most = np.random.default_rng(d), 0
    for _ in range(300):
        kv_heads, group = int(rng.choice([1, 1, 2, 8])), int(rng.choice([1, 4, 16, 64]))
        lengths = np.exp(rng.uniform(0, rng.uniform(1, 12), int(rng.integers(1, 200)))).astype(int)
        starts = [0] + np.cumsum(lengths).tolist()
        desc = C.packed_desc(kv_heads * group, kv_heads, d, bool(rng.integers(2)), dtype, starts[-1])
        plan = C.cephalo_packed_plan(desc, starts)
        most = max(most, desc.key_items - desc.tiles)
        assert desc.key_items - desc.tiles < 512 and plan.numel() * 4 <= binding.lib().cephalo_packed_plan_bytes(len(lengths), desc.tokens)
    assert most > (64 if dtype == C.BF16 else 4)


@pytest.mark.parametrize("starts,says", [([0, 5, 4], "ends before it starts"), ([-1, 5], "from row -1"), ([0, 1001], "to 1001"), ([0], "0 samples")])
def test_starts_outside_the_rows_are_refused(starts, says):
    with pytest.raises(C.CephaloError, match=says):
        C.cephalo_packed_plan(_desc(), starts)


@pytest.mark.parametrize("starts", [[0, 2 ** 32 + 5], [2 ** 32, 2 ** 32 + 5], [-2 ** 32, 5], [0, 2 ** 31]])
def test_starts_that_pass_32_bits_are_refused(starts):
    """Not taken modulo 2^32, where they would lie inside the rows."""
    with pytest.raises(C.CephaloError, match="32 bits"):
        C.cephalo_packed_plan(_desc(), starts)


def test_a_list_buffer_that_is_too_small_is_refused():
    d, L = _desc(), binding.lib()
    starts = (ctypes.c_int32 * 3)(0, 500, 1000)
    need = L.cephalo_packed_plan_bytes(2, 1000)
    buf = ctypes.create_string_buffer(need)
    assert L.cephalo_packed_plan(ctypes.byref(d), 2, starts, buf, need - 1) == -3
    assert L.cephalo_packed_plan(ctypes.byref(d), 2, None, buf, need) == -1
    assert L.cephalo_packed_plan(ctypes.byref(d), 2, starts, None, need) == -1
    assert L.cephalo_packed_plan(None, 2, starts, buf, need) == -1
    assert L.cephalo_packed_plan(ctypes.byref(d), 2, starts, buf, need) == 0


# ---- refusals ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw,code", [
    (dict(heads=0), -1), (dict(kv_heads=0), -1), (dict(heads=4, kv_heads=3), -1), (dict(heads=2, kv_heads=4), -1), (dict(d=0), -1), (dict(d=136), -2),
    (dict(d=100), -2), (dict(dtype=2), -1), (dict(causal=2), -1), (dict(tokens=0), -1), (dict(tokens=2 ** 31), -1), (dict(qkv_pitch=511), -1),
    (dict(o_pitch=255), -1), (dict(qkv_pitch=516), -1), (dict(o_pitch=260), -1), (dict(scale=-1.0), -1), (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1)])
def test_a_desc_that_the_kernels_do_not_hold_is_refused(kw, code):
    with pytest.raises(C.CephaloError, match="cephalo error %d" % code):
        C.cephalo_packed_plan(_desc(**kw), [0, 1])
    assert binding.lib().cephalo_op_attention_packed_bwd_workspace(ctypes.byref(_desc(**kw))) == 0


def _calls(d):
    L = binding.lib()
    return (lambda **k: L.cephalo_op_attention_packed_fwd(ctypes.byref(d), *[k.get(n, FAKE) for n in ("plan", "qkv", "O", "lse")], None),
            lambda **k: L.cephalo_op_attention_packed_bwd(ctypes.byref(d), *[k.get(n, FAKE) for n in ("plan", "qkv", "O", "dO", "lse", "dqkv", "workspace")],
                                                          k.get("bytes", 1 << 40), None))


def test_attention_refuses_bad_buffers_and_a_desc_without_a_list():
    d = _desc()
    for call in _calls(d):
        assert call() == -1 and "has not filled" in C.cephalo_last_error()
    C.cephalo_packed_plan(d, [0, 1000])
    fwd, bwd = _calls(d)
    odd = ctypes.c_void_p(0x1008)
    for call, names in ((fwd, ("plan", "qkv", "O", "lse")), (bwd, ("plan", "qkv", "O", "dO", "lse", "dqkv", "workspace"))):
        for n in names:
            assert call(**{n: None}) == -1
            assert call(**{n: odd}) == -1
    need = binding.lib().cephalo_op_attention_packed_bwd_workspace(ctypes.byref(d))
    assert need >= 4 * 1000 * 4
    assert bwd(bytes=need - 1) == -3


def test_a_sample_beyond_a_buffer_offset_is_refused_and_many_such_rows_are_not():
    pitch = 1 << 20
    d = _desc(tokens=5000, qkv_pitch=pitch)
    C.cephalo_packed_plan(d, [0, 2000])
    fwd, bwd = _calls(d)
    assert fwd() == -2 and bwd() == -2 and "2 GiB" in C.cephalo_last_error()
    C.cephalo_packed_plan(d, [0, 800, 1600, 2400])
    assert fwd(plan=None) == -1 and "null" in C.cephalo_last_error()


@pytest.mark.parametrize("dtype,heads,kv_heads,d,most", [(C.F32, 32, 4, 8, 1 << 20), (C.F32, 32, 4, 100, 1 << 21), (C.BF16, 64, 8, 64, 1 << 24), (C.BF16, 64, 64, 8, 1 << 24), (C.BF16, 64, 64, 72, 1 << 23)])
def test_launches_of_too_many_threads_are_refused_before_any(dtype, heads, kv_heads, d, most):
    """Samples of one row, a block for each and each head (fp32: eight): `most` such pairs are 2^32 threads."""
    for samples, ok in ((most // heads - 1, True), (most // heads, False)):
        desc = _desc(heads, kv_heads, d, True, dtype, samples)
        C.cephalo_packed_plan(desc, range(samples + 1))
        assert (desc.tiles, desc.key_items) == (samples, samples)
        fwd, bwd = _calls(desc)
        for call in (fwd, bwd):
            assert call(plan=None) == -1 if ok else call() == -2 and "threads of a launch" in C.cephalo_last_error()
        assert (binding.lib().cephalo_op_attention_packed_bwd_workspace(ctypes.byref(desc)) > 0) == ok


@pytest.mark.parametrize("rows,code", [(2 ** 30, 0), (2 ** 30 + 1, -2), (2 ** 31 - 64, -2), (2 ** 31 - 63, -2), (2 ** 31 - 1, -2)])
def test_samples_whose_rows_pass_the_kernels_counters_are_refused(rows, code):
    """A longer sample's steps would be counted past 2^31."""
    d, L = _desc(1, 1, 4, False, C.F32, rows), binding.lib()
    plan = np.empty(L.cephalo_packed_plan_bytes(1, rows) // 4, np.int32)      # (untouched pages take no memory)
    assert L.cephalo_packed_plan(ctypes.byref(d), 1, (ctypes.c_int32 * 2)(0, rows), plan.ctypes.data, plan.nbytes) == code
    if code == 0:
        keys = plan[4 * d.tiles:4 * d.tiles + 8 * d.key_items].reshape(-1, 8)
        assert (keys[:, 3] >= 0).all() and (keys[:, 4] > keys[:, 3]).all() and keys[:, 4].max() <= (rows + 63) // 64


def test_no_samples_no_launch():
    d = _desc()
    C.cephalo_packed_plan(d, [4, 4, 4])
    fwd, bwd = _calls(d)
    assert d.tiles == 0 and fwd() == 0 and bwd() == 0


def _rotary(dtype=C.BF16, src=FAKE, src_pitch=256, dst=ctypes.c_void_p(0x2000), dst_pitch=256, positions=FAKE, rows=3, dims=(64,), heads=4, d=64, base=1e4, inverse=0, axes=None):
    dims_c = (ctypes.c_int32 * max(len(dims), 1))(*dims)
    return binding.lib().cephalo_op_rotary_axes(dtype, src, src_pitch, dst, dst_pitch, positions, rows, len(dims) if axes is None else axes, dims_c, heads, d, base, inverse, None)


def test_rotary_refusals():
    odd = ctypes.c_void_p(0x1008)
    for kw, code in [(dict(dtype=5), -1), (dict(rows=-1), -1), (dict(heads=0), -1), (dict(d=0), -1), (dict(d=60, src_pitch=240, dst_pitch=240), -2), (dict(d=136, src_pitch=544, dst_pitch=544), -2),
                     (dict(axes=0), -1), (dict(axes=9), -1), (dict(dims=(63,)), -1), (dict(dims=(66,)), -1), (dict(dims=(32, 34)), -1), (dict(dims=(-2, 4)), -1), (dict(dims=(0,)), -1),
                     (dict(base=1.0), -1), (dict(base=float("nan")), -1), (dict(inverse=2), -1), (dict(src_pitch=255), -1), (dict(dst_pitch=248), -1), (dict(src_pitch=260), -1),
                     (dict(src=None), -1), (dict(dst=None), -1), (dict(positions=None), -1), (dict(src=odd), -1), (dict(dst=odd), -1), (dict(positions=odd), -1),
                     (dict(dst=FAKE, dst_pitch=264), -1)]:
        assert _rotary(**kw) == code, kw
    assert _rotary(rows=0, src=None, dst=None, positions=None) == 0


def test_rotary_and_dropout_launches_of_too_many_threads_are_refused():
    for kw in (dict(rows=1 << 24, heads=300, d=128, src_pitch=300 * 128, dst_pitch=300 * 128, dims=(128,)), dict(rows=1 << 28, heads=1, d=128, src_pitch=128, dst_pitch=128, dims=(128,)),
               dict(rows=1 << 62), dict(dtype=C.F32, rows=1 << 27, heads=8, src_pitch=512, dst_pitch=512)):
        assert _rotary(**kw) == -2 and "threads of a launch" in C.cephalo_last_error(), kw
    for kw in (dict(rows=(1 << 24) - 2, heads=300, d=128, src_pitch=300 * 128, dst_pitch=300 * 128, dims=(128,)), dict(rows=(1 << 28) - 32, heads=1, d=128, src_pitch=128, dst_pitch=128, dims=(128,))):
        assert _rotary(positions=None, **kw) == -1 and "null" in C.cephalo_last_error(), kw
    L = binding.lib()
    for n, code in ((2 ** 35 - 2048, -2), (2 ** 41, -2), (2 ** 62, -2), (2 ** 35 - 2049, -1)):
        assert L.cephalo_op_dropout_add(C.BF16, None, FAKE, FAKE, n, 0.1, 1, 0, None, None) == code
        assert L.cephalo_op_dropout_bwd(C.F32, FAKE, None, n, 0.1, 1, 0, None, None) == code


def test_dropout_refusals():
    L = binding.lib()
    add = lambda dtype=C.BF16, branch=FAKE, resid=FAKE, out=FAKE, n=8, p=0.1, first=0, counter=None: L.cephalo_op_dropout_add(dtype, branch, resid, out, n, p, 1, first, counter, None)      # noqa: E731
    bwd = lambda dtype=C.BF16, dy=FAKE, dbranch=FAKE, n=8, p=0.1, first=0, counter=None: L.cephalo_op_dropout_bwd(dtype, dy, dbranch, n, p, 1, first, counter, None)      # noqa: E731
    odd = ctypes.c_void_p(0x1004)
    for call, kw in itertools.product((add, bwd), [dict(dtype=9), dict(n=-1), dict(p=-0.1), dict(p=1.0), dict(p=float("nan")), dict(p=0.999999), dict(first=4), dict(first=-8), dict(counter=odd)]):
        assert call(**kw) == -1, kw
    for kw in (dict(branch=None), dict(resid=None), dict(out=None), dict(branch=odd), dict(resid=odd), dict(out=odd)):
        assert add(**kw) == -1
    for kw in (dict(dy=None), dict(dbranch=None), dict(dy=odd), dict(dbranch=odd)):
        assert bwd(**kw) == -1
    assert add(n=0, branch=None, resid=None, out=None) == 0 and bwd(n=0, dy=None, dbranch=None) == 0


def test_the_binding_refuses_tensors_that_are_too_small_or_of_another_type():
    d = _desc(tokens=10)
    plan = C.cephalo_packed_plan(d, [0, 10])
    qkv, O, lse = torch.zeros(10, 512, dtype=torch.bfloat16), torch.zeros(10, 256, dtype=torch.bfloat16), torch.zeros(4, 10)
    for args in ((plan[:3], qkv, O, lse), (plan.long(), qkv, O, lse), (plan, qkv[:9], O, lse), (plan, qkv.float(), O, lse), (plan, qkv, O[:9], lse), (plan, qkv, O, lse[:3]),
                 (plan, qkv, O, lse.double())):
        with pytest.raises(C.CephaloError, match="expected"):
            C.cephalo_op_attention_packed_fwd(d, *args)
    with pytest.raises(C.CephaloError, match="device tensor"):
        C.cephalo_op_attention_packed_fwd(d, plan, qkv, O, lse)
    x = torch.zeros(16)
    with pytest.raises(C.CephaloError, match="expected"):
        C.cephalo_op_dropout_add(C.BF16, x, x, x, 16, 0.1, 1)
    with pytest.raises(C.CephaloError, match="expected"):
        C.cephalo_op_dropout_bwd(C.F32, x, x, 17, 0.1, 1)
    with pytest.raises(C.CephaloError, match="expected"):
        C.cephalo_op_rotary_axes(C.F32, x, 8, x, 8, torch.zeros(2, 1, dtype=torch.int64), 2, [8], 1, 8)


@pytest.mark.parametrize("scale", [-0.5, 1e-39, 9e-31, 1.1e30, 3e38, float("inf"), float("nan")])
def test_scales_whose_products_pass_32_bits_are_refused(scale):
    with pytest.raises(C.CephaloError):
        C.cephalo_packed_plan(C.packed_desc(2, 2, 64, True, C.BF16, 8, scale=scale), [0, 8])


@pytest.mark.parametrize("scale", [0.0, 1e-30, 1e30])
def test_scales_at_the_ends_are_taken(scale):
    C.cephalo_packed_plan(C.packed_desc(2, 2, 64, True, C.BF16, 8, scale=scale), [0, 8])
