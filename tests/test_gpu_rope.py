"""vpp_rope and vpp_kv_append_rope against the fp64 oracle, element by element."""
import numpy as np
import pytest
import torch

from block_parity import f64, generator, ints, randn
from oracle.ref_block_sparse import ref_rope, rows_of
from paper_2608_26523_b200 import api

pytestmark = pytest.mark.gpu


def frequencies(rot, base=10000.0):
    return torch.tensor(base ** (-2.0 * np.arange(rot // 2) / rot), dtype=torch.float32, device="cuda")


def check(got, x, positions, inv_freq, layout, offset, amplitude, label=""):
    """The result is rounded once (half a step of bf16: 2^-8 of it); what is left of an angle after its reduction in 64 bits is rounded to 32 (at most
    2^-24 of half a turn), cosine and sine are off by 2 steps of 2^-24, and four roundings of 2^-24 follow: below 6e-7 (|a| + |b|)."""
    f = inv_freq.cpu().numpy().astype(np.float64)
    want = ref_rope(f64(x), positions, f, layout, offset, amplitude)
    other = np.zeros_like(want)
    part = np.abs(f64(x))[..., offset:offset + 2 * len(f)]
    h = len(f)
    pairs = part[..., :h] + part[..., h:] if layout == "half" else part[..., 0::2] + part[..., 1::2]
    other[..., offset:offset + 2 * h] = np.concatenate([pairs, pairs], -1) if layout == "half" else np.repeat(pairs, 2, -1)
    err = np.abs(f64(got) - want)
    assert (err <= 2.0 ** -8 * np.abs(want) + 6e-7 * abs(amplitude) * other).all(), (label, err.max())
    keep = np.ones(want.shape[-1], bool)
    keep[offset:offset + 2 * h] = False
    assert (f64(got)[..., keep] == f64(x)[..., keep]).all(), label


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads, dim, rot, offset", [(1, 16, 16, 0), (5, 128, 128, 0), (3, 128, 64, 64), (2, 128, 32, 40), (7, 64, 48, 8), (4, 576, 64, 512),
                                                     (2, 256, 256, 0), (130, 128, 128, 0)])
def test_rotation(layout, heads, dim, rot, offset):
    gen = generator(heads * dim + rot)
    prefix, chunk = [0, 1000, 7, (1 << 20) - 3, 5], [3, 1, 0, 9, 33]
    T = sum(chunk)
    x = randn(gen, T, heads, dim)
    out = torch.full_like(x, float("nan"))
    status = ints([-1])
    f = frequencies(rot)
    api.vpp_rope(x, out, ints(prefix), ints(chunk), f, layout=layout, rot_offset=offset, amplitude=1.25, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    check(out, x, [p for _, p in rows_of(prefix, chunk)], f, layout, offset, 1.25)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_positions_and_slow_frequencies(layout):
    """Positions to 2^31 - 2, frequencies from 1 to 1e-7: the angle is that of 64 bits."""
    gen = generator(5)
    prefix, chunk = [2 ** 31 - 40, 123456789, 2 ** 24 + 1], [39, 2, 1]
    x = randn(gen, 42, 2, 64)
    f = frequencies(64, 1e7)
    out = torch.empty_like(x)
    api.vpp_rope(x, out, ints(prefix), ints(chunk), f, layout=layout)
    check(out, x, [p for _, p in rows_of(prefix, chunk)], f, layout, 0, 1.0)


def test_in_place_and_strided():
    gen = generator(6)
    prefix, chunk = [100, 3], [21, 40]
    fused = randn(gen, 61, 9, 128)
    before = fused.clone()
    f = frequencies(128)
    positions = [p for _, p in rows_of(prefix, chunk)]
    api.vpp_rope(fused[:, 2:7], fused[:, 2:7], ints(prefix), ints(chunk), f)                    # in place, a part of wider rows
    check(fused[:, 2:7], before[:, 2:7], positions, f, "half", 0, 1.0)
    assert torch.equal(fused[:, :2], before[:, :2]) and torch.equal(fused[:, 7:], before[:, 7:])
    heads_first = randn(gen, 5, 61, 128).transpose(0, 1)                                        # strides in another order
    out = torch.full((61, 5, 200), 3.0, dtype=torch.bfloat16, device="cuda")
    api.vpp_rope(heads_first, out[..., 64:192], ints(prefix), ints(chunk), f, layout="interleaved")
    check(out[..., 64:192], heads_first, positions, f, "interleaved", 0, 1.0)
    assert (out[..., :64] == 3).all() and (out[..., 192:] == 3).all()


def test_bad_lengths_write_nothing():
    x = randn(generator(7), 10, 2, 64)
    f = frequencies(64)
    for prefix, chunk in (([0, 0], [5, 4]), ([0, 0], [11, -1]), ([-1, 0], [5, 5]), ([2 ** 31 - 5, 0], [6, 4]), ([0, 0], [2 ** 31 - 1, 2 ** 31 - 1])):
        out = torch.full_like(x, 7.0)
        status = ints([0])
        api.vpp_rope(x, out, ints(prefix), ints(chunk), f, status=status)
        assert int(status) == 1 and (out == 7).all(), (prefix, chunk)


def make_append(seed, prefix, chunk, hq, hkv, dqk, dv, page, alias=False):
    gen = generator(seed)
    T = sum(chunk)
    ends = [p + c for p, c in zip(prefix, chunk)]
    width = max(1, max(-(-e // page) for e in ends))
    R = len(prefix)
    pool = R * width + 3
    table = torch.randperm(pool, generator=gen, device="cuda")[:R * width].to(torch.int32).view(R, width)
    k_cache = torch.full((pool, page, hkv, dqk), 3.0, dtype=torch.bfloat16, device="cuda")
    v_cache = k_cache[..., :dv] if alias else torch.full((pool, page, hkv, dv), 5.0, dtype=torch.bfloat16, device="cuda")
    fused = randn(gen, T, hq * dqk + hkv * (dqk + dv))
    q = fused[:, :hq * dqk].view(T, hq, dqk) if hq else None
    k = fused[:, hq * dqk:(hq + hkv) * dqk].view(T, hkv, dqk)
    v = None if alias else fused[:, (hq + hkv) * dqk:].view(T, hkv, dv)
    return table, k_cache, v_cache, q, k, v


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("prefix, chunk, hq, hkv, dqk, dv, page, rot, offset, alias", [
    ([0], [1], 1, 1, 128, 128, 16, 128, 0, False),
    ([31, 0, 500, 16], [1, 40, 0, 17], 8, 2, 128, 128, 16, 128, 0, False),
    ([1000, 127], [70, 130], 64, 8, 128, 128, 128, 64, 0, False),
    ([77, 5], [5, 64], 0, 3, 128, 64, 64, 32, 96, False),
    ([200, 63], [30, 2], 0, 1, 576, 512, 64, 64, 512, True),
    ([9, 300], [90, 1], 15, 5, 64, 128, 32, 48, 16, False)])
def test_append(layout, prefix, chunk, hq, hkv, dqk, dv, page, rot, offset, alias):
    table, k_cache, v_cache, q, k, v = make_append(11, prefix, chunk, hq, hkv, dqk, dv, page, alias)
    f = frequencies(rot)
    q_out = None if q is None else torch.full((q.shape[0], hq, dqk), float("nan"), dtype=torch.bfloat16, device="cuda")
    status = ints([-1])
    k0, v0 = k_cache.clone(), v_cache.clone()
    api.vpp_kv_append_rope(k, v, k_cache, v_cache, table, ints(prefix), ints(chunk), page, max(p + c for p, c in zip(prefix, chunk)), f, q=q,
                           q_out=q_out, layout=layout, rot_offset=offset, amplitude=0.75, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    where = rows_of(prefix, chunk)
    positions = [p for _, p in where]
    blk = torch.tensor([int(table[r, p // page]) for r, p in where], device="cuda")
    slot = torch.tensor([p % page for _, p in where], device="cuda")
    check(k_cache[blk, slot], k, positions, f, layout, offset, 0.75, "keys")
    if v is not None:
        assert torch.equal(v_cache[blk, slot], v)
    if q is not None:
        check(q_out, q, positions, f, layout, offset, 0.75, "queries")
    k_cache[blk, slot] = k0[blk, slot]             # every other slot is as it was
    assert torch.equal(k_cache, k0)
    if not alias:
        v_cache[blk, slot] = v0[blk, slot]
        assert torch.equal(v_cache, v0)


def test_append_to_a_contiguous_cache_and_queries_in_place():
    prefix, chunk, gen = [10, 0], [6, 20], generator(13)
    k_cache, v_cache = (torch.zeros((2, 32, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v, q = (randn(gen, 26, h, 128) for h in (2, 2, 4))
    before = q.clone()
    f = frequencies(128)
    api.vpp_kv_append_rope(k, v, k_cache, v_cache, None, ints(prefix), ints(chunk), 0, 32, f, q=q, q_out=q)
    where = rows_of(prefix, chunk)
    r, p = torch.tensor([r for r, _ in where], device="cuda"), torch.tensor([p for _, p in where], device="cuda")
    check(k_cache[r, p], k, p.tolist(), f, "half", 0, 1.0)
    assert torch.equal(v_cache[r, p], v)
    check(q, before, p.tolist(), f, "half", 0, 1.0)


def test_append_checks_on_the_device():
    prefix, chunk, page = [10, 5], [30, 20], 16
    table, k_cache, v_cache, q, k, v = make_append(17, prefix, chunk, 4, 2, 128, 128, page)
    f = frequencies(128)

    def call(prefix, chunk, table):
        kc, vc, qo, status = k_cache.clone(), v_cache.clone(), torch.full((50, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda"), ints([0])
        api.vpp_kv_append_rope(k, v, kc, vc, table, ints(prefix), ints(chunk), page, 64, f, q=q, q_out=qo, status=status)
        return int(status), kc, vc, qo

    for bad in (([10, 5], [30, 19]), ([10, -5], [30, 20]), ([20, 5], [30, 20])):        # (48 positions of pages)
        st, kc, vc, qo = call(*bad, table)
        assert st == 1 and torch.equal(kc, k_cache) and torch.equal(vc, v_cache) and (qo == 7).all()
    wrong = table.clone()
    wrong[0, 1] = k_cache.shape[0]
    wrong[1, 0] = -1
    st, kc, vc, qo = call(prefix, chunk, wrong)
    good = call(prefix, chunk, table)
    assert st == 2 and torch.equal(qo, good[3])
    for r, p in rows_of(prefix, chunk):
        b = int(table[r, p // page])
        if int(wrong[r, p // page]) == b:
            assert torch.equal(kc[b, p % page], good[1][b, p % page]) and torch.equal(vc[b, p % page], good[2][b, p % page])
        else:
            assert (kc[b, p % page] == 3).all() and (vc[b, p % page] == 5).all()


def test_append_equals_rotation_then_append():
    """The same bits as the two calls one after the other, over more rows than one wave of blocks takes."""
    prefix, chunk, page = [3000], [5000], 64
    table, k_cache, v_cache, q, k, v = make_append(19, prefix, chunk, 16, 4, 128, 128, page)
    f, p, c = frequencies(128), ints(prefix), ints(chunk)
    k1, v1, q1, k_rot = k_cache.clone(), v_cache.clone(), torch.empty(5000, 16, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(5000, 4, 128, dtype=torch.bfloat16, device="cuda")
    q2 = torch.empty_like(q1)
    api.vpp_kv_append_rope(k, v, k_cache, v_cache, table, p, c, page, 8000, f, q=q, q_out=q2)
    api.vpp_rope(k, k_rot, p, c, f)
    api.vpp_rope(q, q1, p, c, f)
    api.vpp_kv_append(k_rot, v.contiguous(), k1, v1, table, p, c, page, 8000)
    assert torch.equal(k1, k_cache) and torch.equal(v1, v_cache) and torch.equal(q1, q2)


def test_a_pool_past_32_bits():
    """Pages whose byte offsets pass 2^32."""
    page, hkv = 16, 8
    pool = (5 << 30) // (page * hkv * 256)
    k_cache = torch.zeros((pool, page, hkv, 128), dtype=torch.bfloat16, device="cuda")
    v_cache = torch.zeros_like(k_cache)
    table = ints([[pool - 1, 0, pool - 2]])
    gen = generator(23)
    k, v = randn(gen, 40, hkv, 128), randn(gen, 40, hkv, 128)
    f = frequencies(128)
    api.vpp_kv_append_rope(k, v, k_cache, v_cache, table, ints([5]), ints([40]), page, 48, f)
    blk = torch.tensor([int(table[0, p // page]) for p in range(5, 45)], device="cuda")
    slot = torch.tensor([p % page for p in range(5, 45)], device="cuda")
    check(k_cache[blk, slot], k, range(5, 45), f, "half", 0, 1.0)
    assert torch.equal(v_cache[blk, slot], v)
    assert int((k_cache.view(pool, -1) != 0).any(1).sum()) == 3


def test_captured_and_replayed():
    prefix, chunk = [100], [33]
    table, k_cache, v_cache, q, k, v = make_append(29, prefix, chunk, 8, 2, 128, 128, 16)
    f, p, c = frequencies(128), ints(prefix), ints(chunk)
    q_out, status = torch.empty(33, 8, 128, dtype=torch.bfloat16, device="cuda"), ints([0])
    call = lambda: api.vpp_kv_append_rope(k, v, k_cache, v_cache, table, p, c, 16, 133, f, q=q, q_out=q_out, status=status)      # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    k.copy_(randn(generator(31), 33, 2, 128))
    p.fill_(90)
    graph.replay()
    torch.cuda.synchronize()
    assert int(status) == 0
    blk = torch.tensor([int(table[0, x // 16]) for x in range(90, 123)], device="cuda")
    check(k_cache[blk, torch.tensor([x % 16 for x in range(90, 123)], device="cuda")], k, range(90, 123), f, "half", 0, 1.0)
    check(q_out, q, range(90, 123), f, "half", 0, 1.0)
