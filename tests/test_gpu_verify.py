"""The verification-step operators on the GPU against 64-bit restatements (verify_reference.py), at the sizes and masks where
they can go wrong.

Tolerances.  u is half a step of the output's type relative to the value (torch.finfo(t).eps / 2).  An fp32 chain of n
products and sums adds at most about n 2^-24 of the sum of the magnitudes involved; the approximate exp2 / log2 / rsqrt units
are good to 2^-22 relative.  Each test states what it multiplies."""
import math

import numpy as np
import pytest
import torch

import verify_reference as R

pytestmark = pytest.mark.gpu

BF, HF, FF = torch.bfloat16, torch.float16, torch.float32
THETA, EPS = 500000.0, 1e-5


def u_of(dt):
    return torch.finfo(dt).eps / 2


def tiny_of(dt):
    """Half a step of the type's smallest values: IEEE halves step by 2^-24 below 2^-14, the others by less than 2^-126."""
    return 2.0 ** -25 if dt == torch.float16 else 1e-37


def f64(t):
    return t.detach().double().cpu().numpy()


def i32(values):
    return torch.tensor(np.asarray(values), dtype=torch.int32, device="cuda")


def e4m3(codes):
    return f64(codes.view(torch.float8_e4m3fn).float())


# ------------------------------------------------------------------------------------------------------- plan_pages
def plan_case(rng, seqs, past_hi, new_hi, extra_blocks=3, scarce=False):
    past, new = rng.integers(0, past_hi + 1, seqs), rng.integers(0, new_hi + 1, seqs)
    owned = -(-past // 128) + (rng.random(seqs) < 0.3)
    blocks = int(max((past + new + 127) // 128 + 1)) + extra_blocks
    pages = rng.permutation(int(owned.sum()) + 4000)
    table, at = np.full((seqs, blocks), -7), 0
    for b in range(seqs):
        table[b, : owned[b]] = pages[at: at + owned[b]]
        at += owned[b]
    need = int(np.maximum(0, -(-(past + new) // 128) - owned).sum())
    n_free = need // 2 if scarce else need + 5
    return past, new, owned, table, pages[at: at + max(n_free + 3, 4)], n_free, blocks


@pytest.mark.parametrize("seqs,past_hi,new_hi,scarce", [(1, 0, 1, False), (1, 0, 0, False), (1, 500, 700, False), (3, 128, 128, True), (33, 1000, 5, False), (257, 3000, 300, True),
                                                        (1000, 9000, 40, False), (8192, 200, 2, False), (5, 60000, 9000, False)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan_pages(seqs, past_hi, new_hi, scarce, in_place):
    import paper_2410_03960_b200 as P
    past, new, owned, table, free, n_free, blocks = plan_case(np.random.default_rng(seqs + new_hi), seqs, past_hi, new_hi, scarce=scarce)
    want = R.plan(past, new, owned, table, free, n_free, blocks)
    room = int(new.sum()) + 9
    t = i32(table)
    out = {"block_table": t if in_place else torch.full_like(t, 99), "n_owned": i32([-5] * seqs), "n_free": i32([-5]), "cu_new": i32([-5] * (seqs + 1)),
           "slot_map": i32([-55] * room), "positions": i32([-55] * room), "info": i32([0] * 4)}
    got = P.plan_pages(i32(past), i32(new), i32(owned), t, i32(free), i32([n_free]), out=out)
    P.op_status()
    n = int(new.sum())
    for name in ("n_owned", "n_free", "cu_new", "info", "block_table"):
        assert np.array_equal(got[name].cpu().numpy(), want[name]), name
    for name in ("slot_map", "positions"):
        assert np.array_equal(got[name][:n].cpu().numpy(), want[name]), name
        assert (got[name][n:] == -55).all(), "entries behind the last token"


def test_plan_pages_bounds_what_it_finds():
    """Negative counts read as zero, a table row that is too short and a room that is too small cut what does not fit."""
    import paper_2410_03960_b200 as P
    got = P.plan_pages(i32([-3, 250, 100]), i32([-1, 300, 20]), i32([-2, 99, 1]), i32(np.arange(9).reshape(3, 3)), i32([50, 51, 52]), i32([7]), max_tokens=310)
    assert got["cu_new"].tolist() == [0, 0, 300, 320] and got["n_owned"].tolist() == [0, 3, 1] and got["n_free"].tolist() == [3]
    assert got["info"].tolist() == [320, 0, 2, 550]
    slots = got["slot_map"].tolist()
    assert slots[:6] == [4 * 128 + 122 + i for i in range(6)] and slots[134 - 1] == 5 * 128 + 127 and slots[134:300] == [-1] * 166
    assert slots[300:310] == [6 * 128 + 100 + i for i in range(10)]


def test_plan_pages_follows_nothing_where_sums_wrap():
    """Counts of new tokens that no memory could hold: rows stay inside the pages that are there, or are -1."""
    import paper_2410_03960_b200 as P
    for seqs in (3, 5):
        table = torch.arange(seqs * 6, dtype=torch.int32, device="cuda").view(seqs, 6)
        free = i32(range(100, 140))
        out = P.plan_pages(i32([200] * seqs), i32([1 << 30] * seqs), i32([2] * seqs), table, free, i32([40]), max_tokens=700)
        torch.cuda.synchronize()
        out["slot_map"].fill_(-1)
        P.plan_pages(i32([200] * seqs), i32([1 << 30] * seqs), i32([2] * seqs), table, free, i32([40]), out=out)
        rows = out["slot_map"]
        assert ((rows >= -1) & (rows < 140 * 128)).all()
        bt = out["block_table"]
        assert ((bt >= -1) & (bt < 140)).all()
        assert torch.equal(bt[:, :2], table[:, :2])


# ------------------------------------------------------------------------------------------- qk_norm_rope and gradient
def rope_inputs(T, n_q, n_kv, hd, dt, seed, strided=True, max_pos=131072):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = (n_q + 2 * n_kv) * hd + (8 if strided else 0)
    x = (torch.randn((T, width), generator=g, device="cuda") * 1.5).to(dt)
    q, k, v = (x[:, a: a + n * hd].view(T, n, hd) for a, n in ((0, n_q), (n_q * hd, n_kv), ((n_q + n_kv) * hd, n_kv)))
    pos = torch.randint(0, max_pos, (T,), generator=g, device="cuda", dtype=torch.int32)
    gains = tuple((1 + 0.3 * torch.randn(hd, generator=g, device="cuda")).to(dt) for _ in range(2))
    return g, q, k, v, pos, gains


def rope_bound(x, gain, pos, u, hd, y, tiny=1e-37):
    """u |y| for the store; the pair's magnitudes times 2^-24 (sum of hd squares, rsqrt, gain, table entries, two products):
    hd / 32 + 16 roundings cover the pairwise sums and the chain."""
    h = np.abs(R.head_norm(x, gain, EPS))
    lo, hi = h[..., : hd // 2], h[..., hd // 2:]
    return u * np.abs(y) + (hd / 32 + 16) * 2.0 ** -24 * np.concatenate([lo + hi, lo + hi], -1) + tiny


SHAPES = [(1, 1, 1, 2), (3, 4, 2, 32), (7, 6, 2, 64), (5, 5, 1, 80), (33, 32, 8, 128), (4, 10, 2, 256), (2, 3, 3, 250), (129, 8, 8, 128)]


@pytest.mark.parametrize("T,n_q,n_kv,hd", SHAPES)
@pytest.mark.parametrize("dt", [BF, HF, FF])
@pytest.mark.parametrize("norm", ["both", "k", "none"])
def test_qk_norm_rope(T, n_q, n_kv, hd, dt, norm):
    import paper_2410_03960_b200 as P
    g, q, k, v, pos, (qg, kg) = rope_inputs(T, n_q, n_kv, hd, dt, T * hd, strided=T % 2 == 1)
    qg, kg = (qg if norm == "both" else None), (kg if norm != "none" else None)
    cos, sin = P.rope_table(131072, hd, THETA)
    rows = 2 * T + 3
    slots = torch.randperm(rows, generator=g, device="cuda")[:T].to(torch.int32)
    slots[0] = -1                                             # a token whose page is missing
    kc, vc = torch.full((rows, n_kv, hd), 7.0, dtype=dt, device="cuda"), torch.full((rows, n_kv, hd), 9.0, dtype=dt, device="cuda")
    out = P.qk_norm_rope(q, k, v, pos, cos, sin, q_gain=qg, k_gain=kg, eps=EPS, k_cache=kc, v_cache=vc, slot_map=slots)
    P.op_status()
    p, s, u = pos.cpu().numpy(), slots.cpu().numpy(), u_of(dt)
    for x, gain, got, stored in ((q, qg, f64(out), np.ones(T, bool)), (k, kg, f64(kc)[np.maximum(s, 0)], s >= 0)):
        x, gain = f64(x), None if gain is None else f64(gain)
        want = R.rotate(R.head_norm(x, gain, EPS), p, THETA)
        bad = (np.abs(got - want) > rope_bound(x, gain, p, u, hd, want, tiny_of(dt))) & stored[:, None, None]
        assert not bad.any(), np.argwhere(bad)[:4]
    assert torch.equal(vc[slots[1:].long()], v[1:])
    left = np.setdiff1d(np.arange(rows), s[s >= 0])
    assert (kc[left] == 7).all() and (vc[left] == 9).all(), "rows that no token names"


@pytest.mark.parametrize("T,n_q,n_kv,hd", [(1, 1, 1, 16), (5, 6, 2, 64), (17, 32, 8, 128), (3, 4, 4, 256), (3, 5, 1, 80), (2, 2, 64, 128)])
@pytest.mark.parametrize("dt", [BF, HF, FF])
def test_qk_norm_rope_into_an_fp8_cache(T, n_q, n_kv, hd, dt):
    """Scales to fp32 accuracy, codes to half a step of e4m3 (2^-4 of the value, 2^-10 of the scale where it is subnormal); the
    kernel decides from its own fp32 value, whose error is the bound of the plain store."""
    import paper_2410_03960_b200 as P
    g, q, k, v, pos, (qg, kg) = rope_inputs(T, n_q, n_kv, hd, dt, 3 * T + hd)
    if T > 2:
        v[1] = 0.0                                            # an all-zero row
    cos, sin = P.rope_table(131072, hd, THETA)
    rows = T + 4
    slots = torch.randperm(rows, generator=g, device="cuda")[:T].to(torch.int32)
    kc, vc = (torch.full((rows, n_kv, hd), 0x11, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((rows,), 5.0, device="cuda") for _ in range(2))
    P.qk_norm_rope(q, k, v, pos, cos, sin, q_gain=qg, k_gain=kg, eps=EPS, k_cache=kc, v_cache=vc, k_scale=ks, v_scale=vs, slot_map=slots)
    P.op_status()
    p, s = pos.cpu().numpy(), slots.cpu().numpy()
    for x, gain, codes, scales in ((f64(k), f64(kg), kc, ks), (f64(v), None, vc, vs)):
        want = R.rotate(R.head_norm(x, gain, EPS), p, THETA) if gain is not None else x
        err = rope_bound(x, gain, p, 0.0, hd, want) if gain is not None else np.zeros_like(x)
        sc = f64(scales)[s]
        # scale = RN(max(amax, 2^-64) / 448): half a step (2^-24) of that maximum, the floor included -- an all-zero row's scale is
        # 2^-64 / 448 and rounds too, so the relative term multiplies the floored maximum
        amax = np.maximum(np.abs(want).reshape(T, -1).max(1), 2.0 ** -64)
        assert (np.abs(sc * 448 - amax) <= err.reshape(T, -1).max(1) + 2.0 ** -23 * amax).all()
        got = e4m3(codes)[s] * sc[:, None, None]
        assert (np.abs(got - want) <= 2.0 ** -4 * np.abs(want) + (2.0 ** -10 + 2.0 ** -20) * sc[:, None, None] + 2 * err).all()
        left = np.setdiff1d(np.arange(rows), s)
        assert (codes[left] == 0x11).all() and (scales[left] == 5).all()


@pytest.mark.parametrize("n_kv,hd", [(1, 64), (3, 64), (5, 128), (7, 256), (16, 256), (17, 256), (31, 128), (32, 128), (33, 128), (64, 64)])
def test_qk_norm_rope_into_an_fp8_cache_of_other_widths(n_kv, hd):
    """Rows that do not fill their lanes, that fill a block, and that are too wide for one."""
    test_qk_norm_rope_into_an_fp8_cache(11, n_kv, n_kv, hd, BF)


def test_qk_norm_rope_in_place_and_unaligned():
    """q_out = q, keys and values "stored" to plain tensors, and tensors that start off a 16-byte boundary: the same bits."""
    import paper_2410_03960_b200 as P
    T, n_q, n_kv, hd = 37, 8, 2, 128
    _, q, k, v, pos, (qg, kg) = rope_inputs(T, n_q, n_kv, hd, BF, 5)
    cos, sin = P.rope_table(131072, hd, THETA)
    k1, v1 = (torch.empty((T, n_kv, hd), dtype=BF, device="cuda") for _ in range(2))
    ref = P.qk_norm_rope(q, k, v, pos, cos, sin, q_gain=qg, k_gain=kg, k_cache=k1, v_cache=v1)
    flat = torch.empty(T * n_q * hd + 1, dtype=BF, device="cuda")
    off = flat[1:].view(T, n_q, hd)
    off.copy_(q)
    k2, v2 = torch.empty_like(k1), torch.empty_like(v1)
    got = P.qk_norm_rope(off, k, v, pos, cos, sin, q_gain=qg, k_gain=kg, k_cache=k2, v_cache=v2, q_out=off)
    assert got.data_ptr() == off.data_ptr()
    # (two kernels: the same arithmetic up to the order of the sum of squares)
    assert (got.float() - ref.float()).abs().max() <= 2.0 ** -7 * ref.float().abs().max()
    qi = q.clone()
    got = P.qk_norm_rope(qi, k, v, pos, cos, sin, q_gain=qg, k_gain=kg, k_cache=k2, v_cache=v2, q_out=qi)
    assert torch.equal(got, ref) and torch.equal(k1, k2) and torch.equal(v1, v2)
    P.op_status()


@pytest.mark.parametrize("dt", [BF, HF, FF])
@pytest.mark.parametrize("T,n_q,n_kv,hd", [(1, 4, 2, 128), (700, 8, 2, 64), (2100, 4, 4, 128), (90, 3, 2, 80)])
def test_qk_norm_rope_on_its_inputs(T, n_q, n_kv, hd, dt):
    """Queries, keys and values where they are: without a slot map every row is its own place; and the gradients over q and k."""
    import paper_2410_03960_b200 as P
    g, q, k, v, pos, (qg, kg) = rope_inputs(T, n_q, n_kv, hd, dt, T, strided=False)
    q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    cos, sin = P.rope_table(131072, hd, THETA)
    dq, dk = (torch.randn((T, n, hd), generator=g, device="cuda").to(dt) for n in (n_q, n_kv))
    kc, vc = torch.empty_like(k), torch.empty_like(v)
    qo = P.qk_norm_rope(q, k, v, pos, cos, sin, q_gain=qg, k_gain=kg, eps=EPS, k_cache=kc, v_cache=vc)
    q2, k2, v2 = q.clone(), k.clone(), v.clone()
    P.qk_norm_rope(q2, k2, v2, pos, cos, sin, q_gain=qg, k_gain=kg, eps=EPS, k_cache=k2, v_cache=v2, q_out=q2)
    assert torch.equal(q2, qo) and torch.equal(k2, kc) and torch.equal(v2, v) and torch.equal(vc, v)
    want = P.qk_norm_rope_bwd(dq, dk, q, k, pos, cos, sin, q_gain=qg, k_gain=kg, eps=EPS)
    q2, k2 = q.clone(), k.clone()
    got = P.qk_norm_rope_bwd(dq, dk, q2, k2, pos, cos, sin, q_gain=qg, k_gain=kg, eps=EPS, out=(q2, k2))
    P.op_status()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_overlaps_are_refused():
    import paper_2410_03960_b200 as P
    _, q, k, v, pos, _ = rope_inputs(9, 4, 2, 64, BF, 3)
    cos, sin = P.rope_table(131072, 64, THETA)
    flat = torch.empty(9 * 4 * 64 + 64, dtype=BF, device="cuda")
    a, b = flat[:-64].view(9, 4, 64), flat[64:].view(9, 4, 64)
    kc = torch.empty_like(k, memory_format=torch.contiguous_format)
    with pytest.raises(P.SwiftKVError):
        P.qk_norm_rope(a, k, v, pos, cos, sin, k_cache=kc, v_cache=torch.empty_like(kc), q_out=b)
    with pytest.raises(P.SwiftKVError):
        P.qk_norm_rope(q, k, v, pos, cos, sin, k_cache=kc, v_cache=kc)
    c = tree_case(5, [(90, 9)], 4, 2, 64, BF)
    with pytest.raises(P.SwiftKVError):
        run_tree(c, out=c["q"])


def test_qk_norm_rope_reports_bad_indices():
    import paper_2410_03960_b200 as P
    _, q, k, v, pos, _ = rope_inputs(4, 4, 2, 64, BF, 6, max_pos=50)
    cos, sin = P.rope_table(50, 64, THETA)
    for bad_pos, bad_slot in ((50, 0), (-1, 0), (0, 10)):
        pos2, slots = pos.clone(), i32([3, 1, 2, 9])
        pos2[1] = bad_pos
        slots[2] = bad_slot if bad_slot else 2
        kc = torch.zeros((10, 2, 64), dtype=BF, device="cuda")
        P.qk_norm_rope(q, k, v, pos2, cos, sin, k_cache=kc, v_cache=torch.zeros_like(kc), slot_map=slots)
        with pytest.raises(P.SwiftKVError) as e:
            P.op_status()
        assert e.value.code == -6
        P.op_status()                                        # reported once
        assert (kc[0] == 0).all() and (kc[4:9] == 0).all() and (kc[9] != 0).any()


@pytest.mark.parametrize("T,n_q,n_kv,hd", [(1, 1, 1, 2), (3, 4, 2, 32), (9, 6, 2, 64), (33, 32, 8, 128), (4, 10, 2, 256), (2, 3, 3, 250), (700, 8, 1, 128)])
@pytest.mark.parametrize("dt", [BF, HF, FF])
@pytest.mark.parametrize("norm", ["both", "q", "none"])
def test_qk_norm_rope_gradient(T, n_q, n_kv, hd, dt, norm):
    import paper_2410_03960_b200 as P
    g, q, k, v, pos, (qg, kg) = rope_inputs(T, n_q, n_kv, hd, dt, T + hd, strided=T % 2 == 1)
    qg, kg = (qg if norm != "none" else None), (kg if norm == "both" else None)
    dq, dk = ((torch.randn((T, n, hd), generator=g, device="cuda")).to(dt) for n in (n_q, n_kv))
    cos, sin = P.rope_table(131072, hd, THETA)
    got = P.qk_norm_rope_bwd(dq, dk, q, k, pos, cos, sin, q_gain=qg, k_gain=kg, eps=EPS)
    again = P.qk_norm_rope_bwd(dq.clone(), dk.clone(), q, k, pos, cos, sin, q_gain=qg, k_gain=kg, eps=EPS)
    P.op_status()
    p, u = pos.cpu().numpy(), u_of(dt)
    for x, dy, gain, dx, dg in ((q, dq, qg, got[0], got[2]), (k, dk, kg, got[1], got[3])):
        xn, dn, gn = f64(x), f64(dy), None if gain is None else f64(gain)
        want, wg = R.norm_rope_bwd(xn, dn, gn, EPS, p, THETA)
        # the pair's gradient magnitudes, and -- normed -- |x| r times the mean of |dz g xh|, each with the chain's roundings
        a = np.abs(dn)
        pair = np.concatenate([a[..., : hd // 2] + a[..., hd // 2:]] * 2, -1)
        mag = pair
        if gn is not None:
            r = 1 / np.sqrt((xn * xn).mean(-1, keepdims=True) + EPS)
            mag = r * (pair * np.abs(gn) + np.abs(xn) * r * (pair * np.abs(gn) * np.abs(xn) * r).mean(-1, keepdims=True))
        assert (np.abs(f64(dx) - want) <= u * np.abs(want) + (hd / 32 + 24) * 2.0 ** -24 * mag + tiny_of(dt)).all()
        if gn is None:
            assert dg is None
        else:
            # fp32 partial sums: a thread's chain of at most tokens * heads / 32 terms, then a tree
            terms = (pair * np.abs(xn) * r).sum((0, 1))
            assert (np.abs(f64(dg) - wg) <= (24 + T * x.shape[1] / 32) * 2.0 ** -24 * terms + 1e-30).all()
    for a, b in zip(got, again):
        assert (a is None and b is None) or torch.equal(a, b), "repeats bit for bit"
    P.qk_norm_rope_bwd(dq, dk, q, k, pos, cos, sin, q_gain=qg, k_gain=kg, eps=EPS, out=(dq, dk))       # in place
    assert torch.equal(dq, got[0]) and torch.equal(dk, got[1])


def test_qk_norm_rope_gradient_against_differences():
    """Directional derivatives of the 64-bit forward formula: |difference quotient - gradient . direction| is at most the
    quotient's own error (h^2 f''' / 6, about 1e-7 of the terms at h = 1e-4) plus the kernel's 2^-17 of them."""
    import paper_2410_03960_b200 as P
    T, n_q, n_kv, hd = 6, 4, 2, 64
    g, q, k, v, pos, (qg, kg) = rope_inputs(T, n_q, n_kv, hd, FF, 11, strided=False)
    dq, dk = (torch.randn((T, n, hd), generator=g, device="cuda") for n in (n_q, n_kv))
    cos, sin = P.rope_table(131072, hd, THETA)
    gq, gk, gqg, gkg = P.qk_norm_rope_bwd(dq, dk, q, k, pos, cos, sin, q_gain=qg, k_gain=kg, eps=EPS)
    p = pos.cpu().numpy()
    rng = np.random.default_rng(0)
    for x, dy, gain, gx, gg in ((q, dq, qg, gq, gqg), (k, dk, kg, gk, gkg)):
        x, dy, gain = f64(x), f64(dy), f64(gain)
        f = lambda x_, g_: float((R.rotate(R.head_norm(x_, g_, EPS), p, THETA) * dy).sum())  # noqa: E731
        for _ in range(4):
            d, e = rng.standard_normal(x.shape), rng.standard_normal(gain.shape)
            num = (f(x + 1e-4 * d, gain + 1e-4 * e) - f(x - 1e-4 * d, gain - 1e-4 * e)) / 2e-4
            terms = np.abs(f64(gx) * d).sum() + np.abs(f64(gg) * e).sum()
            assert abs(num - (f64(gx) * d).sum() - (f64(gg) * e).sum()) <= (2.0 ** -17 + 1e-6) * terms


# --------------------------------------------------------------------------------------------------- tree_attention
def random_tree(rng, n, words):
    """Ancestor sets as bit rows [n, words] and as a matrix."""
    seen = []
    for i in range(n):
        parent = int(rng.integers(-1, i)) if i else -1
        seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
    bits = np.array([[(m >> (32 * w)) & 0xFFFFFFFF for w in range(words)] for m in seen], dtype=np.uint32).reshape(n, words)
    return bits.view(np.int32), np.array([[bool(m >> j & 1) for j in range(n)] for m in seen]).reshape(n, n)


def tree_case(seed, lens, n_q, n_kv, hd, dt, fp8=False, paged=True, mask=True, strided=False):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    past, new = [a for a, _ in lens], [b for _, b in lens]
    T, words = sum(new), max(1, -(-max(new) // 32))
    cu = np.concatenate([[0], np.cumsum(new)]).astype(int)
    pages = [-(-(p + n) // 128) for p, n in lens]
    n_pages = sum(pages) + 2
    cache_rows = n_pages * 128
    order, at, table, rows, row0 = rng.permutation(n_pages), 0, np.full((len(lens), max(max(pages), 1) + 1), -1), [], []
    for b, (p, n) in enumerate(lens):
        if paged:
            table[b, : pages[b]] = order[at: at + pages[b]]
            rows.append((table[b, np.arange(p + n) // 128] * 128 + np.arange(p + n) % 128) if p + n else np.zeros(0, int))
        else:
            row0.append(at * 128 + int(rng.integers(0, 3)) * 37)
            rows.append(row0[-1] + np.arange(p + n))
        at += pages[b]
    c = dict(T=T, past=past, cu=cu, rows=rows, max_new=max(new), max_kv=max(p + n for p, n in lens), n_q=n_q, n_kv=n_kv, hd=hd, dt=dt, fp8=fp8)
    q = torch.randn((T, n_q * hd + (8 if strided else 0)), generator=g, device="cuda").mul(1.5).to(dt)
    c["q"] = q[:, : n_q * hd].view(T, n_q, hd)
    if fp8:
        c["k"], c["v"] = (torch.randn((cache_rows, n_kv, hd), generator=g, device="cuda").mul(120).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2))
        c["ks"], c["vs"] = ((torch.rand(cache_rows, generator=g, device="cuda") + 0.5) / 120 for _ in range(2))
    else:
        c["k"], c["v"] = (torch.randn((cache_rows, n_kv, hd), generator=g, device="cuda").to(dt) for _ in range(2))
        c["ks"] = c["vs"] = None
    bits, sees = [], []
    for n in new:
        m, s = random_tree(rng, n, words)
        bits.append(m)
        sees.append(s if mask else np.tril(np.ones((n, n), bool)))
    c["mask"] = i32(np.concatenate(bits)) if mask else None
    c["sees"] = sees
    c["table"], c["row0"] = (i32(table), None) if paged else (None, i32(row0))
    return c


def run_tree(c, **kw):
    import paper_2410_03960_b200 as P
    lse = torch.full((c["T"], c["n_q"]), 77.0, device="cuda")
    args = dict(block_table=c["table"], row0=c["row0"], tree_mask=c["mask"], k_scale=c["ks"], v_scale=c["vs"], lse=lse)
    args.update(kw)
    out = P.tree_attention(c["q"], c["k"], c["v"], i32(c["past"]), i32(c["cu"]), c["max_new"], c["max_kv"], **args)
    return out, lse


def check_tree(c, out, lse, scale=None):
    """|out - o| <= u |o| + (u_P + e) A with A = sum p |v|: u_P the rounding of the probabilities to 16 bits (the 16-bit paths; with an
    FP8 cache they carry the rows' scale and are halves: 2^-11 relative, or -- steps of 2^-24 below 2^-14, with a reference that keeps the
    row's largest P at 1 or more -- 2^-25 of that largest: 2^-25 G, the G of verify_reference), e the relative error of a probability: twice that of its exponent, which is the
    products' (hd + 2) 2^-24 of sum |q k| scale, plus 2^-20 for exp2 and the fp32 sums over the keys (pairwise inside a tile, then a
    chain over tiles and splits)."""
    u = u_of(c["dt"])
    if c["fp8"]:
        k, v = e4m3(c["k"]) * f64(c["ks"])[:, None, None], e4m3(c["v"]) * f64(c["vs"])[:, None, None]
        u_p = 2.0 ** -11 if c["dt"] != FF else 0.0
        extra = dict(v_scale=f64(c["vs"]), v_codes=e4m3(c["v"]))
    else:
        k, v = f64(c["k"]), f64(c["v"])
        u_p = u if c["dt"] != FF else 0.0
        extra = {}
    want, wl, A, Z, G = R.tree_attention(f64(c["q"]), k, v, c["past"], c["cu"], c["rows"], c["sees"], scale, **extra)
    dz = (c["hd"] + 2) * 2.0 ** -24 * Z + 2.0 ** -20 + 2.0 ** -24 * np.where(np.isfinite(wl), np.abs(wl), 0) * 4
    keys = c["max_kv"] / 128 + 64
    e = (2 * dz + keys * 2.0 ** -24)[..., None]
    got, gl = f64(out), f64(lse)
    sees = np.isfinite(wl)
    assert np.array_equal(sees, np.isfinite(gl)) and (gl[~sees] == -np.inf).all() and (got[~sees] == 0).all()
    bad = np.abs(got - want) > u * np.abs(want) + (u_p * 1.01 + e) * A + (2.0 ** -25 * G if c["dt"] != FF else 0.0) + tiny_of(c["dt"])
    assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - want).max())
    assert (np.abs(gl - wl)[sees] <= (dz + keys * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(np.where(sees, wl, 0))))[sees]).all()


LENS = [[(0, 1)], [(127, 1)], [(128, 1)], [(0, 33)], [(700, 1), (0, 5), (130, 7)], [(5, 3), (200, 0), (0, 1), (126, 4)], [(1000, 40), (64, 64)], [(2500, 17)]]


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (32, 8, 128)], ids=str)
@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8"])
@pytest.mark.parametrize("paged", [True, False])
def test_tree_attention(lens, heads, kind, paged):
    import paper_2410_03960_b200 as P
    c = tree_case(len(lens) * 100 + lens[0][0], lens, *heads, HF if kind == "f16" else BF, fp8=kind == "fp8", paged=paged, strided=paged)
    check_tree(c, *run_tree(c))
    P.op_status()


@pytest.mark.parametrize("heads", [(7, 1, 128), (10, 2, 128), (3, 1, 64), (24, 2, 128), (16, 1, 128), (65, 1, 128), (200, 1, 64), (5, 5, 128)], ids=str)
@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_tree_attention_group_sizes(heads, kind):
    """Groups that do not divide a tile of 128 query rows, and groups larger than one."""
    c = tree_case(heads[0], [(300, 23), (129, 1), (90, 50)], *heads, BF, fp8=kind == "fp8")
    check_tree(c, *run_tree(c))


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 2, 32), (3, 3, 80), (2, 1, 256), (6, 2, 2), (5, 1, 17)], ids=str)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f32 fp8"])
def test_tree_attention_other_shapes(heads, kind):
    c = tree_case(heads[2], [(300, 9), (0, 3), (1500, 2)], *heads, BF if kind == "bf16" else FF, fp8="fp8" in kind, mask=heads[0] != 3)
    check_tree(c, *run_tree(c))


# many short sequences: several complete (sequence, head) pieces, and parts of others, per block of the grid
MANY = {"few rows": [(300 + 17 * i, 1 + i % 8) for i in range(40)],
        "64 rows": [(100 + 23 * i, 9 + i % 8) for i in range(30)],
        "128 rows": [(100 + 31 * i, 3 + i * 7 % 30) for i in range(30)],
        "one and two groups": [(150 + 43 * i, 150 if i % 6 == 1 else 1 + i % 5) for i in range(24)],
        "three groups": [(150 + 43 * i, 270 if i % 12 == 1 else 3) for i in range(24)]}


@pytest.mark.parametrize("lens", MANY, ids=str)
@pytest.mark.parametrize("heads", [(16, 8, 128), (15, 5, 64), (4, 1, 128)], ids=str)
@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_tree_attention_many_pieces_per_block(lens, heads, kind):
    c = tree_case(len(lens), MANY[lens], *heads, BF, fp8=kind == "fp8")
    check_tree(c, *run_tree(c))


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("max_new", [20, 40, 70, 130, 300])
def test_tree_attention_promised_more_than_comes(kind, max_new):
    """max_new and max_kv far above what the lengths say (a server passes its limits), sequences of nothing among them."""
    import paper_2410_03960_b200 as P
    c = tree_case(max_new, [(300, 3), (0, 0), (1300, 17), (0, 1), (640, 8), (77, 0)], 16, 4, 128, FF if kind == "f32" else BF, fp8=kind == "fp8")
    c["max_new"] = max_new
    keys = c["max_kv"]
    c["max_kv"] = 40000
    out, lse = run_tree(c)
    c["max_kv"] = keys
    check_tree(c, out, lse)
    P.op_status()


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("max_new", [(1 << 29) + 1, 1 << 26, (1 << 31) - 1])
@pytest.mark.parametrize("heads", [(16, 2, 128), (64, 1, 64)], ids=str)
def test_tree_attention_promises_of_any_size(kind, max_new, heads):
    """max_new times the heads of a group beyond 32 bits, and the largest number that there is."""
    import paper_2410_03960_b200 as P
    c = tree_case(max_new % 97, [(300, 3), (0, 20), (640, 1)], *heads, FF if kind == "f32" else BF, fp8=kind == "fp8")
    want, want_lse = run_tree(c)
    out, lse = run_tree(dict(c, max_new=max_new))
    check_tree(c, out, lse)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    P.op_status()


def test_tree_attention_limits_of_a_large_server():
    """256 sequences of one token with limits that no call comes near: the size of the work is the tokens', not the limits'."""
    import paper_2410_03960_b200 as P
    c = tree_case(256, [(i, 1) for i in range(256)], 32, 8, 128, BF)
    keys, c["max_new"], c["max_kv"] = c["max_kv"], 65536, 131072
    out, lse = run_tree(c)
    check_tree(dict(c, max_kv=keys), out, lse)
    P.op_status()


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_tree_attention_any_max_kv(kind):
    import paper_2410_03960_b200 as P
    c = tree_case(77, [(300, 3), (1500, 2)], 16, 4, 128, FF if kind == "f32" else BF, fp8=kind == "fp8")
    out, lse = run_tree(dict(c, max_kv=(1 << 31) - 1))
    check_tree(c, out, lse)
    P.op_status()


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
def test_tree_attention_a_length_that_no_cache_has(kind):
    """A committed length next to 2^31 is cut so that the keys are 2^30, and reported; what lies behind the table reads as zeros, which all
    have score 0: the few hundred rows that are there carry 2^-21 of the probability."""
    import paper_2410_03960_b200 as P
    c = tree_case(78, [(300, 2)], 4, 1, 128, BF, fp8=kind == "fp8")
    c["q"] = c["q"] * 0.01
    out, lse = run_tree(dict(c, past=[(1 << 31) - 200], max_kv=(1 << 31) - 1))
    assert (lse - 30 * math.log(2.0)).abs().max() <= 1e-4 and out.float().abs().max() <= 1e-4
    with pytest.raises(P.SwiftKVError) as e:
        P.op_status()
    assert e.value.code == -6


@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8", "f32"])
@pytest.mark.parametrize("heads", [(4, 1, 128), (6, 2, 64)], ids=str)
def test_tree_attention_prompt_chunks(kind, heads):
    """Chunks of prompts (no mask: causal): many groups of query tiles per sequence, a decode token beside them."""
    c = tree_case(heads[0], [(1400, 900), (3, 300), (801, 1)], *heads, {"bf16": BF, "f16": HF, "fp8": BF, "f32": FF}[kind], fp8=kind == "fp8", mask=False)
    check_tree(c, *run_tree(c))


def test_tree_attention_many_rows_in_the_general_form():
    """fp32 rows enough for every SM: the keys are split less often, so that the partial results stay bounded."""
    import paper_2410_03960_b200 as P
    for lens, n_q, hd in (([(32700, 300)], 16, 16), ([(2000, 700), (1, 2)], 64, 8)):
        c = tree_case(len(lens), lens, n_q, 4, hd, FF, mask=False)
        check_tree(c, *run_tree(c))
    P.op_status()


def test_tree_attention_more_tokens_than_copies_are_kept_for():
    """An FP8 cache and tiles of few rows, but 700, then 2600 of them."""
    for seqs, new in ((700, 1), (1300, 2)):
        c = tree_case(seqs, [(i % 140, new) for i in range(seqs)], 4, 2, 64, BF, fp8=True)
        check_tree(c, *run_tree(c))


@pytest.mark.parametrize("kind", ["bf16", "fp8"])
@pytest.mark.parametrize("hi", [8, 24, 50, 150])
def test_tree_attention_repeats_bit_for_bit(kind, hi):
    """Thirty calls over sequences whose warps of unused rows run ahead of the others into the last tiles of a sequence."""
    c = tree_case(hi, [(400 + 331 * i, 1 + i * 13 % hi) for i in range(16)], 16, 8, 128, BF, fp8=kind == "fp8")
    first, lse = run_tree(c)
    if hi == 24:
        check_tree(c, first, lse)
    for _ in range(30):
        out, l2 = run_tree(c)
        assert torch.equal(out, first) and torch.equal(l2, lse)


@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8", "f32"])
@pytest.mark.parametrize("n", [6, 12, 30, 60])
def test_tree_attention_one_element_of_a_drafted_row(kind, n):
    """An infinity or NaN in one element of a drafted token's K or V.  Who does not see the token keeps the result; who sees it gets it
    everywhere (K) or in that element (V), and keeps the rest of the row."""
    c = tree_case(n, [(250, n), (90, 2)], 16, 4, 128, {"bf16": BF, "f16": HF, "fp8": BF, "f32": FF}[kind], fp8=kind == "fp8")
    row = int(c["rows"][0][251])
    who = torch.tensor(np.flatnonzero(c["sees"][0][:, 1]), device="cuda")
    assert 0 < len(who) < n
    for what in ("k", "v"):
        if what == "v":
            c["v"][row, 2, 17] = 0
        base, _ = run_tree(c)
        kept = c[what][row, 2, 17].clone()
        c[what][row, 2, 17] = 0xFF if kind == "fp8" else float("nan") if what == "k" else float("inf")
        out, _ = run_tree(c)
        c[what][row, 2, 17] = kept
        hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        if what == "k":
            hit[who, 8:12] = True
        else:
            hit[who, 8:12, 17] = True
        assert torch.equal(out[~hit], base[~hit]) and not torch.isfinite(out[hit]).any(), what


@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8", "f32"])
def test_tree_attention_causal_and_scale(kind):
    c = tree_case(3, [(1029, 130), (0, 257), (3, 1)], 8, 2, 128, {"bf16": BF, "f16": HF, "fp8": BF, "f32": FF}[kind], fp8=kind == "fp8", mask=False)
    check_tree(c, *run_tree(c))
    out, lse = run_tree(c, softmax_scale=0.31)
    check_tree(c, out, lse, scale=float(np.float32(0.31)))


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_tree_attention_empty_rows_and_rows_behind(kind):
    """Mask rows of zeros (over no committed token: nothing is seen), mask words beyond the new tokens, untouched rows behind."""
    c = tree_case(8, [(0, 6), (40, 5), (0, 40)], 8, 2, 128, FF if kind == "f32" else BF, fp8=kind == "fp8")
    mask = c["mask"].clone()
    mask[2] = 0
    mask[7] = 0
    mask[11:51] = 0
    mask[30, 1] = -1                           # sees tokens 32 .. 39 and bits past the last one
    c["mask"] = mask
    c["sees"][0][2] = False
    c["sees"][1][1] = False
    c["sees"][2][:] = False
    c["sees"][2][19, 32:] = True
    check_tree(c, *run_tree(c))
    T = c["T"]
    import paper_2410_03960_b200 as P
    wide = dict(c, T=T + 3, q=torch.cat([c["q"], c["q"][:3]]).contiguous())
    out = torch.full((T + 3, 8, 128), 5.0, dtype=c["dt"], device="cuda")
    o, lse = run_tree(dict(wide, mask=torch.cat([mask, mask[:3]])), out=out)
    check_tree(c, o[:T].contiguous(), lse[:T].contiguous())
    assert (o[T:] == 5).all() and (lse[T:] == 77).all()
    P.op_status()


@pytest.mark.parametrize("kind", ["bf16", "f16", "fp8", "f32"])
@pytest.mark.parametrize("lens", [[(250, 6), (0, 9)], [(128, 20)], [(3, 120)]], ids=str)
def test_tree_attention_ignores_what_is_not_seen(kind, lens):
    """NaN and infinities in cache rows behind a sequence's last token, in free pages, and in a drafted token's K and V that others do
    not see: the others' results keep their bits."""
    c = tree_case(21, lens, 8, 2, 128, {"bf16": BF, "f16": HF, "fp8": BF, "f32": FF}[kind], fp8=kind == "fp8")
    # the first sequence's token 1 is seen by nobody but itself
    c["mask"][:, 0] &= ~2
    c["mask"][1, 0] |= 2
    for s in c["sees"]:
        s[:, 1] = False
    c["sees"][0][1, 1] = True
    c["mask"][c["cu"][0] + 1, 0] |= 2
    if len(lens) > 1:
        assert not (c["mask"][c["cu"][1]:, 0] & 2).any()
    clean, clean_lse = run_tree(c)
    check_tree(c, clean, clean_lse)
    used = np.concatenate(c["rows"])
    free = np.setdiff1d(np.arange(c["k"].shape[0]), used)
    hidden = int(c["rows"][0][lens[0][0] + 1])
    d = dict(c, k=c["k"].clone(), v=c["v"].clone())
    if kind == "fp8":
        d["ks"], d["vs"] = c["ks"].clone(), c["vs"].clone()
        for t in (d["k"], d["v"]):
            t[free] = 0x7F                     # the code that stands for no number
            t[hidden] = 0x7E
        for t in (d["ks"], d["vs"]):
            t[free] = float("nan")
            t[hidden] = float("inf")
    else:
        for t in (d["k"], d["v"]):
            t[free] = float("nan")
            t[hidden] = float("inf")
            t[hidden, 0, ::3] = float("nan")
    out, lse = run_tree(d)
    others = [t for t in range(c["T"]) if t != 1]
    assert torch.equal(out[others], clean[others]) and torch.equal(lse[others], clean_lse[others])
    assert not torch.isfinite(out[1].float()).all()          # and the one that sees it does not hide it


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
def test_tree_attention_large_scores(kind):
    """Scores of some hundreds, rising along the keys (every tile moves the reference maximum) and falling."""
    for sign in (1.0, -1.0):
        c = tree_case(31, [(900, 4)], 4, 2, 128, FF if kind == "f32" else BF, fp8=kind == "fp8")
        c["q"] = torch.ones_like(c["q"])
        ramp = torch.linspace(-3, 3, 904, device="cuda") * sign * 10
        rows = torch.as_tensor(c["rows"][0], device="cuda")
        if kind == "fp8":
            c["k"][rows] = 0x38                # 1.0
            c["ks"][rows] = ramp.abs() + 1e-3
            neg = rows[ramp < 0]
            c["k"][neg] = 0xB8
        else:
            c["k"][rows] = ramp[:, None, None].to(c["dt"]).expand(-1, 2, 128)
        check_tree(c, *run_tree(c))


@pytest.mark.parametrize("n", [1, 10, 20, 40])
def test_tree_attention_every_fp8_code(n):
    """All 254 numbers of e4m3, subnormal ones and zeros of both signs among them, in K and V; 4 to 160 rows per KV head (a tile of few
    rows is laid out several times); row scales over many powers of two."""
    for dt in (BF, HF, FF):
        c = tree_case(33, [(700, n), (3, n)], 8, 2, 128, dt, fp8=True)
        numbers = torch.tensor([i for i in range(256) if i & 0x7F != 0x7F], dtype=torch.uint8, device="cuda")
        g = torch.Generator(device="cuda").manual_seed(5)
        for t in (c["k"], c["v"]):
            t.copy_(numbers[torch.randint(0, 254, t.shape, generator=g, device="cuda")])
        c["ks"] = torch.exp2(torch.randint(-14, -8, c["ks"].shape, generator=g, device="cuda").float()) * 1.37
        c["vs"] = torch.exp2(torch.randint(-30, 3, c["vs"].shape, generator=g, device="cuda").float()) * 1.19
        check_tree(c, *run_tree(c))


def test_tree_attention_reports_lengths_and_pages():
    """Pages outside the cache read as zero rows; lengths beyond what the call promises are cut and reported."""
    import paper_2410_03960_b200 as P
    for kind in (BF, FF):
        c = tree_case(41, [(300, 4)], 4, 2, 128, kind)
        c["table"][0, 1] = 10 ** 6
        c["rows"][0][128:256] = -1
        check_tree(c, *run_tree(c))
        c["table"][0, 1] = -5
        check_tree(c, *run_tree(c))
        P.op_status()
        run_tree(dict(c, max_new=3))
        with pytest.raises(P.SwiftKVError) as e:
            P.op_status()
        assert e.value.code == -6
        run_tree(dict(c, max_kv=200))
        with pytest.raises(P.SwiftKVError):
            P.op_status()


def rows_gone(c):
    """The same case for the reference, with the rows outside the cache (-1) as one more row of zeros."""
    one_more = lambda t: None if t is None else torch.cat([t, torch.zeros_like(t[:1])])  # noqa: E731
    end = c["k"].shape[0]
    return dict(c, rows=[np.where(r < 0, end, r) for r in c["rows"]], **{name: one_more(c[name]) for name in ("k", "v", "ks", "vs")})


def lose_pages(c, b, pages, entry=-1):
    for j in pages:
        c["table"][b, j] = entry
        c["rows"][b][j * 128: (j + 1) * 128] = -1


@pytest.mark.parametrize("kind", ["bf16 fp8", "f16 fp8", "f32 fp8", "bf16"])
@pytest.mark.parametrize("n", [1, 8, 12, 20])
@pytest.mark.parametrize("gone", [[0], [3], [5], [0, 5], [0, 1, 2, 3, 4, 5], []], ids=str)
def test_tree_attention_pages_that_are_missing(kind, n, gone):
    """Pages outside the cache read as zeros, first, in the middle, last, all of them; a second sequence has none at all.  4 rows per token
    and KV head: with an FP8 cache a query tile is laid out 4, 4, 2 and 1 times."""
    import paper_2410_03960_b200 as P
    c = tree_case(100 + n, [(700, n), (60, n)], 32, 8, 128, {"bf16": BF, "f16": HF, "f32": FF}[kind.split()[0]], fp8="fp8" in kind)
    lose_pages(c, 0, gone, -1 if n < 12 else 10 ** 6)
    lose_pages(c, 1, [0])
    check_tree(rows_gone(c), *run_tree(c))
    P.op_status()


@pytest.mark.parametrize("kind", ["bf16 fp8", "f16 fp8", "bf16"])
@pytest.mark.parametrize("n", [2, 20])
def test_tree_attention_pieces_of_missing_pages(kind, n):
    """Runs of missing pages as long as what a block of the grid works on, so that whole pieces of a sequence hold nothing else."""
    c = tree_case(130 + n, [(9000, n)], 32, 8, 128, HF if "f16" in kind.split() else BF, fp8="fp8" in kind)
    lose_pages(c, 0, list(range(0, 9)) + list(range(30, 44)) + [69, 70])
    check_tree(rows_gone(c), *run_tree(c))


@pytest.mark.parametrize("n", [1, 12, 20])
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -64 / 448, 1e-38])
def test_tree_attention_rows_of_zeros_in_v(n, scale):
    """FP8 pages whose V rows are zero: by a scale of 0 (or next to it), or quantized from zeros."""
    for dt in (BF, HF, FF):
        c = tree_case(140 + n, [(700, n), (60, n), (5000, n)], 16, 4, 128, dt, fp8=True)
        for b, pages in ((0, (0, 5)), (1, (0,)), (2, range(10, 20))):
            for j in pages:
                rows = torch.as_tensor(c["rows"][b][j * 128: (j + 1) * 128], device="cuda")
                c["vs"][rows] = scale
                if scale:
                    c["v"][rows] = 0
        check_tree(c, *run_tree(c))


@pytest.mark.parametrize("kind", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("past", [50, 2100])
def test_tree_attention_rows_cut_off_a_sequence(kind, past):
    """A sequence of more new tokens than max_new: the rest of its rows stay as they were, and the call is reported."""
    import paper_2410_03960_b200 as P
    c = tree_case(past, [(past, 9), (40, 3)], 8, 2, 128, FF if kind == "f32" else BF, fp8=kind == "fp8", mask=False)
    c["max_new"] = 5
    out = torch.full(c["q"].shape, 5.0, dtype=c["dt"], device="cuda")
    out, lse = run_tree(c, out=out)
    assert (out[5:9] == 5).all() and (lse[5:9] == 77).all()
    assert (out[:5] != 5).any(dim=-1).all() and (out[9:] != 5).any(dim=-1).all() and (lse[9:] != 77).all()
    with pytest.raises(P.SwiftKVError) as e:
        P.op_status()
    assert e.value.code == -6


def test_tree_attention_one_token_equals_tail_attention():
    """One new token per sequence is the single-query attention of the last-token path."""
    import paper_2410_03960_b200 as P
    lens = [(699, 1), (128, 1), (2999, 1)]
    c = tree_case(51, lens, 32, 8, 128, BF, paged=False)
    k = torch.cat([c["k"][torch.as_tensor(r, device="cuda")] for r in c["rows"]]).contiguous()
    v = torch.cat([c["v"][torch.as_tensor(r, device="cuda")] for r in c["rows"]]).contiguous()
    ref = P.tail_attention(c["q"].float().contiguous(), k, v, [p + 1 for p, _ in lens]).view(3, 32, 128)
    out, _ = run_tree(c)
    # both round probabilities: 2^-9 each at most, on outputs of sum p |v| <= max |v| (about 4.5)
    assert (out.float() - ref).abs().max() <= 2.0 ** -8 * float(v.float().abs().max())


def test_tree_attention_beyond_32_bit_offsets():
    """Cache planes of more than 2^32 bytes / 2^31 elements: rows at their far end."""
    import paper_2410_03960_b200 as P
    n_kv, hd = 8, 128
    rows = (1 << 31) // (n_kv * hd) + 4096                    # elements beyond 2^31, 4.3 GB per plane
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("needs 14 GB")
    k, v = (torch.zeros((rows, n_kv, hd), dtype=BF, device="cuda") for _ in range(2))
    c = tree_case(61, [(600, 5)], 16, n_kv, hd, BF, paged=False)
    first = rows - 700
    src = torch.as_tensor(c["rows"][0], device="cuda")
    k[first: first + 605], v[first: first + 605] = c["k"][src], c["v"][src]
    out, lse = run_tree(dict(c, k=k, v=v, row0=i32([first])))
    check_tree(c, out, lse)
    P.op_status()


# --------------------------------------------------------------------------------------------------- token_logprobs
def lp_case(rows, vocab, dt, seed, pad=0, std=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((rows, vocab + pad), dtype=dt, device="cuda").normal_(0, std, generator=g)[:, :vocab]
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    return g, x, t


def check_lp(x, t, temperature, k, got):
    """lse, logprob, entropy in fp32: exponents (z - m) carry 2 roundings of their own size, so p is good to 2^-22 (1 + range) with range
    the spread of the logits that matter (p > 2^-24: about 17 + 1); log2 is good to 2^-21 absolute, the sums to (vocab / 4096 + 32)
    2^-24 relative; adding m / T rounds once at its size."""
    xn = f64(x)
    with np.errstate(all="ignore"):
        want = R.token_logprobs(xn, np.maximum(t.cpu().numpy(), -1), temperature, k)
    rel = 20 * 2.0 ** -22 + (xn.shape[1] / 4096 + 32) * 2.0 ** -24 + 2.0 ** -21
    for name in ("lse", "logprob", "entropy") + (("top_logprobs",) if k else ()):
        a, b = f64(got[name]), want[name]
        fin = np.isfinite(b)
        assert np.array_equal(fin, np.isfinite(a)), name
        scale = np.where(np.isfinite(want["lse"]), np.abs(want["lse"]), 0) * 2.0 ** -22
        tol = rel * (1 + np.abs(np.where(fin, b, 0)) * 2.0 ** -1 * (name == "entropy")) + (scale if a.ndim == 1 else scale[:, None]) + 2.0 ** -21 * np.abs(np.where(fin, b, 0))
        assert (np.abs(np.where(fin, a - np.where(fin, b, 0), 0)) <= tol).all(), (name, np.nanmax(np.abs(a - b)))
    if k:
        assert np.array_equal(got["top_ids"].cpu().numpy(), want["top_ids"])


@pytest.mark.parametrize("rows,vocab,pad", [(1, 1, 0), (1, 5, 0), (3, 17, 2), (2, 1000, 1), (5, 4097, 0), (9, 32000, 0), (1, 128256, 0), (200, 50001, 0), (3, 160001, 63), (40, 8191, 1)])
@pytest.mark.parametrize("dt", [FF, BF, HF])
@pytest.mark.parametrize("k,temperature", [(0, 1.0), (1, 0.7), (5, 1.0), (20, 2.0), (32, 1.0)])
def test_token_logprobs(rows, vocab, pad, dt, k, temperature):
    import paper_2410_03960_b200 as P
    _, x, t = lp_case(rows, vocab, dt, rows + vocab, pad)
    t[rows // 2] = -1
    k = min(k, vocab)
    got = P.token_logprobs(x, t, top_k=k, temperature=temperature)
    P.op_status()
    check_lp(x, t, float(np.float32(temperature)), k, got)


@pytest.mark.parametrize("dt", [FF, BF])
@pytest.mark.parametrize("split", [True, False])
def test_token_logprobs_ties_and_orders(dt, split):
    """Equal logits keep the lowest index first; rising, falling and constant rows; zeros of both signs are equal."""
    import paper_2410_03960_b200 as P
    rows, vocab = (6, 40000) if split else (6 * 160, 9000)
    x = torch.zeros((rows, vocab), dtype=dt, device="cuda")
    i = torch.arange(vocab, device="cuda")
    x[1::6] = (i / 1000).to(dt)
    x[2::6] = (-i / 1000).to(dt)
    x[3::6] = torch.where(i % 2 == 0, 0.0, -0.0).to(dt)
    x[4::6] = ((i * 7919) % 13).to(dt)
    x[5::6] = torch.where(i >= vocab - 40, 3.0, 1.0).to(dt)
    t = torch.full((rows,), vocab - 1, dtype=torch.int32, device="cuda")
    for k in (1, 7, 32):
        check_lp(x, t, 1.0, k, P.token_logprobs(x, t, top_k=k))


def test_token_logprobs_masked_and_peaked():
    """Logits of -inf, of the type's lowest value, of some thousands; all mass on one token; rows without any finite logit."""
    import paper_2410_03960_b200 as P
    _, x, t = lp_case(12, 5000, FF, 4)
    x[0, 10:] = -math.inf
    x[1, :4990] = torch.finfo(FF).min
    x[2] *= 1000
    x[3, 77] = 60.0
    x[4, :] = -math.inf
    x[4, 4321] = -5.0
    x[5, :] = torch.finfo(FF).min
    x[6, 0] = -math.inf
    x[7, 1:] = -math.inf
    t[3], t[4], t[6], t[7] = 77, 4321, 0, 0
    got = P.token_logprobs(x[:4], t[:4], top_k=5)
    check_lp(x[:4], t[:4], 1.0, 5, {k: v for k, v in got.items()})
    got = P.token_logprobs(x[4:12].contiguous(), t[4:12], top_k=5)
    check_lp(x[4:12], t[4:12], 1.0, 5, got)
    y = x[8:11].clone()
    y[0] = -math.inf
    y[1, 9] = math.nan
    y[2, 8] = math.inf
    got = P.token_logprobs(y, t[:3], top_k=2)
    assert got["lse"][0] == -math.inf and torch.isnan(got["entropy"]).all() and torch.isnan(got["logprob"]).all()
    for i, at in ((0, 0), (1, 4999), (2, 2500)):             # a NaN among masked logits, wherever it is met
        z = torch.full((1, 5000), -math.inf if i else torch.finfo(FF).min, device="cuda")
        z[0, at] = math.nan
        z[0, 10:20] = 1.0
        assert all(torch.isnan(v).all() for v in P.token_logprobs(z, t[:1] * 0 + 12).values())
    assert torch.isnan(got["lse"][1:]).all() and got["top_ids"][1, 0] == 9 and got["top_ids"][2, 0] == 8 and got["top_ids"][0].tolist() == [0, 1]
    P.op_status()


@pytest.mark.parametrize("dt", [FF, BF, HF])
@pytest.mark.parametrize("vocab", [3, 4, 8, 9, 5000, 40000])
def test_token_logprobs_a_nan_in_every_vector(dt, vocab):
    """Rows of which no thread holds a whole vector without a NaN: finite logits beside it are not the row's maximum, and nothing of the
    row's results is a number but its top_ids."""
    import paper_2410_03960_b200 as P
    rows = 3
    x = torch.arange(rows * vocab, device="cuda").remainder(11).view(rows, vocab).to(dt)
    x[0, 2::4] = math.nan                        # one in every 16 bytes of fp32, two of the 16-bit types
    x[1, 1] = math.nan
    x[1, 2:] = -math.inf
    x[2, 0] = math.nan
    t = i32([0, 0, vocab - 1])
    k = min(3, vocab)
    got = P.token_logprobs(x, t, top_k=k)
    P.op_status()
    for name in ("lse", "entropy", "logprob", "top_logprobs"):
        assert torch.isnan(got[name]).all(), (name, got[name])
    assert got["top_ids"].tolist() == np.argsort(-np.nan_to_num(f64(x), nan=1e30), 1, kind="stable")[:, :k].tolist()


@pytest.mark.parametrize("dt", [FF, BF, HF])
@pytest.mark.parametrize("vocab", [18, 3001, 40000])
@pytest.mark.parametrize("temperature", [0.7, 1.0, 1.5, 3.0, 50.0])
def test_token_logprobs_masked_by_low_values(dt, vocab, temperature):
    """Logits masked by the type's lowest value, or by others near it: ahead of the rest, behind them, in between, all but one, all.  (As
    a probability every one of them is 0 where anything else is there.)"""
    import paper_2410_03960_b200 as P
    g, x, t = lp_case(10, vocab, dt, vocab)
    low = torch.finfo(dt).min
    for i, value in enumerate((low, low / 2, low / 1.7, low / 1.4, low)):
        x[i, : vocab - 7] = value
        x[5 + i] = value
        x[5 + i, (vocab - 1) * i // 4] = 0.5
    x[0, 9] = -math.inf
    x[9] = low
    x[4, : vocab // 2], x[4, vocab // 2:] = 1.0, low
    t[:5], t[5:] = (torch.tensor([vocab - 1, vocab - 2, vocab - 3, vocab - 4, 0]), torch.tensor([(vocab - 1) * i // 4 for i in range(5)]))
    got = P.token_logprobs(x, t, temperature=temperature)
    P.op_status()
    n = 10
    if low / temperature < -3.41e38:             # the last row's lse, low / T + log(vocab), is beyond fp32
        n = 9
        assert got["lse"][9] == -math.inf and abs(got["entropy"][9] - math.log(vocab)) < 1e-4 and abs(got["logprob"][9] + math.log(vocab)) < 1e-4
    check_lp(x[:n], t[:n], float(np.float32(temperature)), 0, {k: v[:n] for k, v in got.items()})
    d = P.token_logprobs_bwd(x, t, got["lse"], got["entropy"], torch.ones(10, device="cuda"), torch.ones(10, device="cuda"), temperature=temperature)
    assert torch.isfinite(d[:9].float()).all()


@pytest.mark.parametrize("dt", [FF, BF, HF])
@pytest.mark.parametrize("value", [-6e4, -1e6, -1e9, -3e9, -1e10, -1e20, -1e30])
def test_token_logprobs_masked_by_large_values(dt, value):
    """The usual constants of masks, over whole chunks ahead of what counts, over a row, and large logits of the other sign."""
    import paper_2410_03960_b200 as P
    if dt == HF and value < -65504:
        value = -65504.0
    for vocab in (40, 9000, 70000):
        g, x, t = lp_case(6, vocab, dt, vocab)
        x[0, : vocab - 9] = value
        x[1, 3:] = value
        x[2] = value
        x[3, vocab // 2] = -value
        x[4, ::2] = value
        x[4, 1::2] = -math.inf
        x[5] = -value
        t[:] = torch.tensor([vocab - 1, 0, 5, vocab // 2, 4, 7])
        for temperature in (1.0, 0.6):
            got = P.token_logprobs(x, t, top_k=3, temperature=temperature)
            check_lp(x, t, float(np.float32(temperature)), 3, got)
    P.op_status()


def test_token_logprobs_reports_bad_targets():
    import paper_2410_03960_b200 as P
    _, x, t = lp_case(3, 100, BF, 5)
    t[1] = 100
    got = P.token_logprobs(x, t)
    assert got["logprob"][1] == 0
    with pytest.raises(P.SwiftKVError) as e:
        P.op_status()
    assert e.value.code == -6
    none = P.token_logprobs(x)
    assert (none["logprob"] == 0).all() and torch.equal(none["lse"], got["lse"])


@pytest.mark.parametrize("rows,vocab,pad,out_pad", [(1, 1, 0, 0), (3, 17, 2, 0), (2, 1000, 1, 3), (5, 4097, 0, 0), (4, 32000, 8, 0), (7, 9001, 0, 4), (300, 1009, 2, 0)])
@pytest.mark.parametrize("dt", [FF, BF, HF])
@pytest.mark.parametrize("entropy", [True, False])
def test_token_logprobs_gradient(rows, vocab, pad, out_pad, dt, entropy):
    """|d - want| <= u |want| + e (|g_lp| p + |g_H| p (|log p| + H)) / T, e the relative error of p: the exponent's, which is its size (z and lse
    up to about 20: 2^-20) plus exp2's 2^-22, and lse's and H's own rounding to fp32."""
    import paper_2410_03960_b200 as P
    g, x, t = lp_case(rows, vocab, dt, rows * 3 + vocab, pad)
    t[0] = -1
    T = 0.7
    fwd = P.token_logprobs(x, t, temperature=T)
    g_lp, g_h = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))
    g_h = g_h if entropy else None
    out = torch.full((rows, vocab + out_pad), 3.0, dtype=dt, device="cuda")
    got = P.token_logprobs_bwd(x, t, fwd["lse"], fwd["entropy"] if entropy else None, g_lp, g_h, temperature=T, out=out[:, :vocab])
    P.op_status()
    assert (out[:, vocab:] == 3).all()
    xn, tn, Tn = f64(x), t.cpu().numpy(), float(np.float32(T))
    want = R.token_logprobs_bwd(xn, tn, Tn, f64(g_lp), None if g_h is None else f64(g_h))
    w = R.token_logprobs(xn, tn, Tn, 0)
    logp = xn / Tn - w["lse"][:, None]
    p = np.exp(logp)
    mag = np.abs(f64(g_lp))[:, None] * (p + (np.arange(vocab) == tn[:, None]))
    if g_h is not None:
        mag = mag + np.abs(f64(g_h))[:, None] * p * (1 + np.abs(logp) + w["entropy"][:, None])
    assert (np.abs(f64(got) - want) <= u_of(dt) * np.abs(want) + 2.0 ** -18 * mag / Tn + tiny_of(dt)).all()
    if pad == 0 and out_pad == 0:
        y = x.clone()
        again = P.token_logprobs_bwd(y, t, fwd["lse"], fwd["entropy"], g_lp, g_h, temperature=T, out=y)
        assert again.data_ptr() == y.data_ptr() and torch.equal(again, got)


def test_token_logprobs_gradient_against_differences():
    """Directional derivatives of the 64-bit forward formula (h = 1e-4: error about 1e-7 of the terms)."""
    import paper_2410_03960_b200 as P
    g, x, t = lp_case(4, 300, FF, 8)
    t[2] = -1
    fwd = P.token_logprobs(x, t, temperature=2.0)
    g_lp, g_h = (torch.randn(4, generator=g, device="cuda") for _ in range(2))
    d = f64(P.token_logprobs_bwd(x, t, fwd["lse"], fwd["entropy"], g_lp, g_h, temperature=2.0))
    xn, tn = f64(x), t.cpu().numpy()

    def f(y):
        w = R.token_logprobs(y, tn, 2.0, 0)
        return float((w["logprob"] * f64(g_lp)).sum() + (w["entropy"] * f64(g_h)).sum())

    rng = np.random.default_rng(1)
    for _ in range(4):
        e = rng.standard_normal(xn.shape)
        num = (f(xn + 1e-4 * e) - f(xn - 1e-4 * e)) / 2e-4
        assert abs(num - (d * e).sum()) <= (2.0 ** -17 + 1e-6) * np.abs(d * e).sum() + 1e-9


def test_token_logprobs_gradient_of_masked_logits():
    import paper_2410_03960_b200 as P
    g, x, t = lp_case(2, 600, BF, 9)
    x[:, 100:300] = -math.inf
    x[:, 300:400] = torch.finfo(BF).min
    t[:] = 5
    fwd = P.token_logprobs(x, t)
    big = torch.full((2,), 1e9, device="cuda")
    d = P.token_logprobs_bwd(x, t, fwd["lse"], fwd["entropy"], big, big)
    assert torch.isfinite(d.float()).all() and (d[:, 100:400] == 0).all()


# -------------------------------------------------------------------------------------------------------- together
class Step:
    """One layer's verification step over a paged cache, as a server would run it: plan, norm + rotate + store, attend, score."""

    def __init__(self, seed, lens, fp8=False, n_q=8, n_kv=2, hd=128, vocab=5000):
        import paper_2410_03960_b200 as P
        self.P, self.fp8, self.n_q, self.n_kv, self.hd = P, fp8, n_q, n_kv, hd
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.past, self.new = [p for p, _ in lens], [n for _, n in lens]
        T = self.T = sum(self.new)
        owned = [-(-p // 128) for p in self.past]
        pages = rng.permutation(sum(owned) + 20)
        blocks = max(-(-(p + n) // 128) for p, n in lens) + 1
        table, at = np.full((len(lens), blocks), -1), 0
        for b, o in enumerate(owned):
            table[b, :o] = pages[at: at + o]
            at += o
        self.host = (owned, table, pages[at:], len(pages) - at, blocks)
        self.d = dict(past=i32(self.past), new=i32(self.new), owned=i32(owned), table=i32(table), free=i32(pages[at:]), n_free=i32([len(pages) - at]))
        rows = len(pages) * 128
        make = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        if fp8:
            self.k, self.v = (make(rows, n_kv, hd).mul(100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2))
            self.ks, self.vs = (torch.rand(rows, generator=g, device="cuda") / 100 + 0.005 for _ in range(2))
        else:
            self.k, self.v, self.ks, self.vs = make(rows, n_kv, hd).to(BF), make(rows, n_kv, hd).to(BF), None, None
        self.qkv = make(T, (n_q + 2 * n_kv) * hd).to(BF)
        self.qg, self.kg = (1 + 0.2 * make(hd)).to(BF), (1 + 0.2 * make(hd)).to(BF)
        self.cos, self.sin = P.rope_table(4096, hd, THETA)
        words = -(-max(self.new) // 32)
        trees = [random_tree(rng, n, words) for n in self.new]
        self.mask, self.sees = i32(np.concatenate([m for m, _ in trees])), [s for _, s in trees]
        self.logits = make(T, vocab).to(BF)
        self.targets = torch.randint(0, vocab, (T,), generator=g, device="cuda", dtype=torch.int32)
        self.before = (self.k.clone(), self.v.clone(), None if not fp8 else self.ks.clone(), None if not fp8 else self.vs.clone())

    def run(self, stream=None):
        P, d, n_q, n_kv, hd = self.P, self.d, self.n_q, self.n_kv, self.hd
        plan = P.plan_pages(d["past"], d["new"], d["owned"], d["table"], d["free"], d["n_free"], max_tokens=self.T, stream=stream)
        q, k, v = (self.qkv[:, a * hd: (a + n) * hd].view(self.T, n, hd) for a, n in ((0, n_q), (n_q, n_kv), (n_q + n_kv, n_kv)))
        q = P.qk_norm_rope(q, k, v, plan["positions"], self.cos, self.sin, q_gain=self.qg, k_gain=self.kg, k_cache=self.k, v_cache=self.v, k_scale=self.ks,
                           v_scale=self.vs, slot_map=plan["slot_map"], stream=stream)
        lse = torch.empty((self.T, n_q), device="cuda")
        o = P.tree_attention(q, self.k, self.v, d["past"], plan["cu_new"], max(self.new), max(a + b for a, b in zip(self.past, self.new)),
                             block_table=plan["block_table"], tree_mask=self.mask, k_scale=self.ks, v_scale=self.vs, lse=lse, stream=stream)
        return plan, q, o, lse, P.token_logprobs(self.logits, self.targets, top_k=4, stream=stream)

    def check(self, got):
        """The plan exactly; each later operator against its reference on what the ones before it gave."""
        plan, q, o, lse, lp = got
        owned, table, free, n_free, blocks = self.host
        want = R.plan(self.past, self.new, owned, table, free, n_free, blocks)
        for name, x in want.items():
            assert np.array_equal(plan[name].cpu().numpy(), x), name
        n_q, n_kv, hd, T = self.n_q, self.n_kv, self.hd, self.T
        x = f64(self.qkv).reshape(T, n_q + 2 * n_kv, hd)
        p = want["positions"]
        wq = R.rotate(R.head_norm(x[:, :n_q], f64(self.qg), EPS), p, THETA)
        assert (np.abs(f64(q) - wq) <= rope_bound(x[:, :n_q], f64(self.qg), p, 2.0 ** -8, hd, wq)).all()
        slots = want["slot_map"]
        wk = R.rotate(R.head_norm(x[:, n_q: n_q + n_kv], f64(self.kg), EPS), p, THETA)
        if not self.fp8:
            assert (np.abs(f64(self.k)[slots] - wk) <= rope_bound(x[:, n_q: n_q + n_kv], f64(self.kg), p, 2.0 ** -8, hd, wk)).all()
            assert np.array_equal(f64(self.v)[slots], x[:, n_q + n_kv:])
        left = np.setdiff1d(np.arange(self.k.shape[0]), slots)
        assert torch.equal(self.k[left], self.before[0][left]) and torch.equal(self.v[left], self.before[1][left])
        rows = [want["block_table"][b][np.arange(a + n) // 128] * 128 + np.arange(a + n) % 128 for b, (a, n) in enumerate(zip(self.past, self.new))]
        c = dict(q=q, k=self.k, v=self.v, ks=self.ks, vs=self.vs, past=self.past, cu=want["cu_new"].astype(int), rows=rows, sees=self.sees, dt=BF, fp8=self.fp8, hd=hd,
                 max_kv=max(a + b for a, b in zip(self.past, self.new)))
        check_tree(c, o, lse)
        check_lp(self.logits, self.targets, 1.0, 4, lp)


LENS_STEP = [(300, 9), (0, 5), (127, 1), (128, 33), (1000, 12)]


@pytest.mark.parametrize("fp8", [False, True])
def test_a_verification_step(fp8):
    s = Step(71, LENS_STEP, fp8)
    s.check(s.run())
    s.P.op_status()


@pytest.mark.parametrize("fp8", [False, True])
def test_a_verification_step_on_another_stream_and_two_at_once(fp8):
    a, b = Step(72, LENS_STEP, fp8), Step(73, LENS_STEP[::-1], fp8)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        for s in (s1, s2):
            s.wait_stream(torch.cuda.current_stream())
        ga, gb = a.run(s1), b.run(s2)
        s1.synchronize()
        s2.synchronize()
    a.check(ga)
    b.check(gb)


@pytest.mark.parametrize("fp8", [False, True])
def test_a_verification_step_captured_and_replayed(fp8):
    """Two graphs over the same kernels, replayed in turn and side by side, with inputs changed in between."""
    a, b = Step(74, LENS_STEP, fp8), Step(75, LENS_STEP[::-1], fp8)
    a.run(), b.run()
    torch.cuda.synchronize()
    graphs, got = [], []
    for s in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(s.run())
        graphs.append(g)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for k in range(3):
        for s in (a, b):
            s.qkv.mul_(-1.25 if k else 1.0)
            s.logits.add_(0.5)
        torch.cuda.synchronize()
        with torch.cuda.stream(s1):
            graphs[0].replay()
        with torch.cuda.stream(s2):
            graphs[1].replay()
        torch.cuda.synchronize()
        a.check(got[0])
        b.check(got[1])


def test_the_gradients_captured_and_replayed():
    import paper_2410_03960_b200 as P
    g, q, k, v, pos, (qg, kg) = rope_inputs(60, 8, 2, 128, BF, 81)
    dq, dk = (torch.randn((60, n, 128), generator=g, device="cuda").to(BF) for n in (8, 2))
    cos, sin = P.rope_table(131072, 128, THETA)
    _, x, t = lp_case(5, 3001, BF, 82)
    gl = torch.randn(5, generator=g, device="cuda")

    def both():
        f = P.token_logprobs(x, t)
        return P.qk_norm_rope_bwd(dq, dk, q, k, pos, cos, sin, q_gain=qg, k_gain=kg) + (P.token_logprobs_bwd(x, t, f["lse"], f["entropy"], gl, gl),)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(2):
        dq.mul_(0.5)
        x.add_(1.0)
        graph.replay()
        for a, b in zip(got, both()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dt", [BF, FF])
def test_no_tokens_and_no_rows(dt):
    """A step in which nothing is drafted: empty results of the right shapes, caches as they were; bad arguments are refused all the same."""
    import paper_2410_03960_b200 as P
    e = lambda *shape: torch.empty(shape, dtype=dt, device="cuda")  # noqa: E731
    q, k, cos, sin = e(0, 4, 64), e(0, 2, 64), *P.rope_table(16, 64, THETA)
    kc, vc, gain = e(256, 2, 64).fill_(3), e(256, 2, 64).fill_(3), e(64).fill_(1)
    plan = P.plan_pages(i32([100]), i32([0]), i32([1]), i32([[0]]), i32([1]), i32([1]), max_tokens=0)
    assert plan["info"].tolist() == [0, 0, 0, 100]
    out = P.qk_norm_rope(q, k, k, plan["positions"], cos, sin, q_gain=gain, k_gain=gain, k_cache=kc, v_cache=vc, slot_map=plan["slot_map"])
    assert out.shape == (0, 4, 64) and out.dtype == dt and (kc == 3).all() and (vc == 3).all()
    dq, dk, gq, gk = P.qk_norm_rope_bwd(q, k, q, k, plan["positions"], cos, sin, q_gain=gain)
    assert dq.shape == (0, 4, 64) and dk.shape == (0, 2, 64) and (gq == 0).all() and gq.shape == (64,) and gk is None
    lse = torch.empty((0, 4), device="cuda")
    assert P.tree_attention(q, kc, vc, i32([100]), plan["cu_new"], 8, 1000, block_table=plan["block_table"], lse=lse).shape == (0, 4, 64)
    x, none = e(0, 300), torch.empty(0, device="cuda")
    got = P.token_logprobs(x, i32([]), top_k=3)
    assert got["lse"].shape == (0,) and got["top_ids"].shape == (0, 3)
    assert P.token_logprobs_bwd(x, i32([]), none, None, none).shape == (0, 300)
    with pytest.raises(ValueError):
        P.qk_norm_rope(q, k, k, i32([1]), cos, sin, k_cache=kc, v_cache=vc)
    with pytest.raises(ValueError):
        P.tree_attention(q, kc, vc, i32([100]), i32([0]), 8, 1000, block_table=plan["block_table"])
    with pytest.raises(ValueError):
        P.token_logprobs(x, i32([1]))
    P.op_status()
