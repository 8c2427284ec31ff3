"""What the verification-step operators refuse, on the host and without a GPU: every bad call returns its code before
anything reaches a device.  Addresses here are never followed."""
import ctypes as C

import pytest
import torch

INVALID, SMALL, UNSUPPORTED = -1, -2, -7
A = 0x10000000          # a 256-byte aligned address in steps that keep the arguments apart


@pytest.fixture(scope="module")
def lib():
    from paper_2410_03960_b200 import binding, build
    build.build()
    return binding.load_library()


def at(i):
    return A + i * 0x1000000


PLAN = dict(n_past=at(0), n_new=at(1), n_owned=at(2), n_seqs=4, block_table=at(3), max_blocks=16, free_pages=at(4), free_capacity=64, n_free=at(5),
            block_table_out=at(6), n_owned_out=at(7), n_free_out=at(8), cu_new=at(9), slot_map=at(10), positions=at(11), max_tokens=100, info=at(12), stream=None)


@pytest.mark.parametrize("bad", [dict(n_past=None), dict(info=None), dict(n_seqs=0), dict(n_seqs=8193), dict(max_blocks=0), dict(free_capacity=-1),
                                 dict(max_tokens=-1), dict(slot_map=None), dict(free_pages=None),
                                 dict(n_owned_out=at(2)), dict(n_free_out=at(5)), dict(cu_new=at(0) + 8), dict(block_table_out=at(3) + 64), dict(positions=at(10) + 4),
                                 dict(info=at(4) + 4 * 63)])
def test_plan_pages(lib, bad):
    assert lib.swiftkv_plan_pages(*{**PLAN, **bad}.values()) == INVALID
    assert lib.swiftkv_last_error()


ROPE = dict(q=at(0), q_stride=1024, k=at(1), k_stride=256, v=at(2), v_stride=256, dtype=1, n_tokens=5, n_q=8, n_kv=2, hd=128, q_gain=None, k_gain=None, eps=1e-5,
            positions=at(3), cos=at(4), sin=at(5), max_pos=100, q_out=at(6), q_out_stride=1024, k_cache=at(7), v_cache=at(8), k_scale=None, v_scale=None,
            cache_rows=64, slot_map=at(9), stream=None)


@pytest.mark.parametrize("bad,code", [(dict(q=None), INVALID), (dict(positions=None), INVALID), (dict(v_cache=None), INVALID), (dict(q_stride=1023), INVALID),
                                      (dict(k_stride=255), INVALID), (dict(q_out_stride=1000), INVALID), (dict(dtype=3), INVALID), (dict(dtype=9), INVALID),
                                      (dict(n_tokens=0), INVALID), (dict(hd=127), INVALID), (dict(hd=258), INVALID), (dict(hd=0), INVALID), (dict(max_pos=0), INVALID),
                                      (dict(cache_rows=0), INVALID), (dict(k_scale=at(10)), INVALID), (dict(v_scale=at(10)), INVALID), (dict(eps=-1.0), INVALID),
                                      (dict(eps=float("nan")), INVALID), (dict(q=at(0) + 1), INVALID), (dict(k_cache=at(7) + 1), INVALID),
                                      (dict(slot_map=None, cache_rows=4), INVALID), (dict(n_kv=2000, k_stride=1 << 20, v_stride=1 << 20), INVALID),
                                      (dict(n_kv=65, k_stride=65 * 128, v_stride=65 * 128, k_scale=at(10), v_scale=at(11)), UNSUPPORTED)])
def test_qk_norm_rope(lib, bad, code):
    assert lib.swiftkv_qk_norm_rope(*{**ROPE, **bad}.values()) == code


BWD = dict(dq=at(0), dk=at(1), q=at(2), q_stride=1024, k=at(3), k_stride=256, dtype=1, n_tokens=5, n_q=8, n_kv=2, hd=128, q_gain=at(4), k_gain=at(5), eps=1e-5,
           positions=at(6), cos=at(7), sin=at(8), max_pos=100, dq_in=at(9), dk_in=at(10), dq_gain=at(11), dk_gain=at(12), scratch=at(13), scratch_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("bad,code", [(dict(dq=None), INVALID), (dict(dq_gain=None), INVALID), (dict(q_gain=None), INVALID), (dict(scratch=None), INVALID),
                                      (dict(hd=3), INVALID), (dict(q_stride=8), INVALID), (dict(dtype=7), INVALID), (dict(n_tokens=-2), INVALID),
                                      (dict(scratch=at(13) + 4), INVALID), (dict(dk_in=at(10) + 1), INVALID), (dict(scratch_bytes=64), SMALL)])
def test_qk_norm_rope_bwd(lib, bad, code):
    assert lib.swiftkv_qk_norm_rope_bwd(*{**BWD, **bad}.values()) == code


def test_rope_table(lib):
    assert lib.swiftkv_rope_table(None, at(1), 8, 128, 1e4, None) == INVALID
    for bad in [(0, 128, 1e4), (8, 127, 1e4), (8, 300, 1e4), (8, 128, 0.0), (8, 128, float("nan"))]:
        assert lib.swiftkv_rope_table(at(0), at(1), *bad, None) == INVALID


TREE = dict(q=at(0), q_stride=1024, q_dtype=1, k=at(1), v=at(2), kv_dtype=1, k_scale=None, v_scale=None, cache_rows=256, block_table=at(3), max_blocks=4, row0=None,
            n_past=at(4), cu_new=at(5), mask=at(6), mask_words=2, out=at(7), lse=None, n_seqs=2, total_new=8, max_new=5, max_kv=300, n_q=8, n_kv=2, hd=128,
            scale=0.0, scratch=at(8), scratch_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("bad,code", [(dict(q=None), INVALID), (dict(n_past=None), INVALID), (dict(out=None), INVALID), (dict(block_table=None), INVALID),
                                      (dict(row0=at(9)), INVALID), (dict(n_seqs=0), INVALID), (dict(total_new=0), INVALID), (dict(max_new=0), INVALID),
                                      (dict(max_kv=0), INVALID), (dict(n_kv=3), INVALID), (dict(hd=1), INVALID), (dict(hd=257), INVALID), (dict(cache_rows=0), INVALID),
                                      (dict(max_blocks=0), INVALID), (dict(mask_words=0), INVALID), (dict(q_stride=1000), INVALID), (dict(kv_dtype=2), INVALID),
                                      (dict(q_dtype=3, kv_dtype=3), INVALID), (dict(kv_dtype=3), INVALID), (dict(k_scale=at(9), v_scale=at(10)), INVALID),
                                      (dict(scale=float("inf")), INVALID), (dict(scale=-1.0), INVALID), (dict(q=at(0) + 1), INVALID), (dict(k=at(1) + 1), INVALID),
                                      (dict(scratch=at(8) + 8), INVALID), (dict(scratch=None, max_kv=100000), SMALL), (dict(scratch_bytes=16, max_kv=100000), SMALL)])
def test_tree_attention(lib, bad, code):
    assert lib.swiftkv_tree_attention(*{**TREE, **bad}.values()) == code


def test_tree_attention_scratch_grows_with_its_arguments(lib):
    f = lib.swiftkv_tree_attention_scratch_bytes
    for bad in [(0, 10, 8, 128), (4, 0, 8, 128), (4, 10, 0, 128), (4, 10, 8, 0), (4, 10, 8, 257)]:
        assert f(*bad) == 0
    for hd in (32, 64, 128, 256):
        last = 0
        for kv in (1, 100, 1024, 1025, 5000, 33000, 131072, 1 << 20):
            now = f(64, kv, 32, hd)
            assert now >= last and f(32, kv, 32, hd) <= now
            last = now


def test_tree_attention_scratch_is_bounded(lib):
    """A long prompt chunk over a large promised length: partial results of 131072 rows at most, whatever the form, and never less than a
    smaller call needs."""
    f = lib.swiftkv_tree_attention_scratch_bytes
    assert f(16384, 131072, 32, 128) <= 128 << 20 and f(65536, 1 << 20, 64, 256) <= 160 << 20
    for hd in (32, 128, 256):
        sizes = [[f(t, kv, 32, hd) for kv in (1, 1024, 1025, 9000, 33000, 1 << 20, 1 << 30)] for t in (1, 2, 60, 128, 129, 300, 4095, 4096, 4097, 50000)]
        for t, row in enumerate(sizes):
            assert row == sorted(row) and (t == 0 or all(a <= b for a, b in zip(sizes[t - 1], row)))


LP = dict(logits=at(0), stride=1000, dtype=0, targets=at(1), rows=4, vocab=1000, temperature=1.0, top_k=3, logprob=at(2), entropy=at(3), lse=at(4), ids=at(5), top=at(6),
          stream=None)


@pytest.mark.parametrize("bad", [dict(logits=None), dict(stride=999), dict(dtype=3), dict(rows=0), dict(vocab=0), dict(temperature=0.0), dict(temperature=-1.0),
                                 dict(temperature=float("inf")), dict(temperature=float("nan")), dict(top_k=-1), dict(top_k=33), dict(vocab=2, top_k=3), dict(lse=None),
                                 dict(ids=None), dict(top=None), dict(logits=at(0) + 2)])
def test_token_logprobs(lib, bad):
    assert lib.swiftkv_token_logprobs(*{**LP, **bad}.values()) == INVALID


LPB = dict(logits=at(0), stride=1000, dtype=1, targets=at(1), rows=4, vocab=1000, temperature=1.0, lse=at(2), entropy=at(3), g=at(4), gh=at(5), out=at(6), out_stride=1000,
           stream=None)


@pytest.mark.parametrize("bad", [dict(targets=None), dict(lse=None), dict(g=None), dict(out=None), dict(entropy=None), dict(out_stride=10), dict(out=at(6) + 1),
                                 dict(out=at(0) + 2), dict(out=at(0), out_stride=1024), dict(temperature=0.0)])
def test_token_logprobs_bwd(lib, bad):
    assert lib.swiftkv_token_logprobs_bwd(*{**LPB, **bad}.values()) == INVALID


@pytest.mark.parametrize("bad", [dict(vocab=(1 << 30) + 1, stride=1 << 31), dict(vocab=(1 << 31) - 1, stride=1 << 31), dict(rows=(1 << 26) + 1)])
def test_token_logprobs_of_more_than_32_bits_count(lib, bad):
    """Rows whose last elements a block's step would carry past 2^31."""
    assert lib.swiftkv_token_logprobs(*{**LP, **bad}.values()) == INVALID
    assert lib.swiftkv_token_logprobs_bwd(*{**LPB, **bad, "out_stride": 1 << 31}.values()) == INVALID


# 5 tokens of 8 + 2 + 2 heads of 128 as slices of one projection's rows (12 heads and 8 elements of padding) that start at at(0)
WIDE = 12 * 128 + 8
ROW = 2 * WIDE
FUSED = dict(q=at(0), q_stride=WIDE, k=at(0) + 2048, k_stride=WIDE, v=at(0) + 2560, v_stride=WIDE)


@pytest.mark.parametrize("bad", [dict(q_out=at(0) + 256), dict(q_out=at(0)), dict(q_out=at(0), q_out_stride=1024), dict(q_out=at(0) - 2, q_out_stride=WIDE),
                                 dict(q_out=at(0) + 512, q_out_stride=WIDE), dict(q_out=at(0) + ROW, q_out_stride=2048), dict(k_cache=at(0) + 2048), dict(v_cache=at(0) + 9000),
                                 dict(v_cache=at(7) + 512), dict(q_out=at(8) + 64 * 512 - 2), dict(k_cache=at(0) + 2048, slot_map=None)])
def test_qk_norm_rope_refuses_overlaps(lib, bad):
    assert lib.swiftkv_qk_norm_rope(*{**ROPE, **FUSED, **bad}.values()) == INVALID
    assert b"overlap" in lib.swiftkv_last_error()


@pytest.mark.parametrize("good", [dict(FUSED, q_out=at(0), q_out_stride=WIDE), dict(FUSED, q_out=at(0) + 5 * ROW), dict(FUSED, k_cache=at(0) + 5 * ROW),
                                  dict(q_out=at(0)), dict(k_cache=at(1), v_cache=at(2), slot_map=None), dict(n_tokens=1, q_out=at(0), q_out_stride=4096)])
def test_qk_norm_rope_takes_what_shares_no_byte(lib, good):
    """Slices of one projection's rows, results behind their last row, a head on itself: nothing here is refused as an overlap."""
    if not torch.cuda.is_available():
        assert lib.swiftkv_qk_norm_rope(*{**ROPE, **good}.values()) not in (0, INVALID)      # (no device: it fails behind the checks)


@pytest.mark.parametrize("bad", [dict(dq_in=at(0) + 2), dict(dk_in=at(1) + 256), dict(dq_in=at(1)), dict(dk_in=at(0)), dict(dk_in=at(9) + 64), dict(dq_in=at(2), q_stride=1100),
                                 dict(dk_in=at(2) + 2048), dict(dk_in=at(3), k_stride=300)])
def test_qk_norm_rope_bwd_refuses_overlaps(lib, bad):
    assert lib.swiftkv_qk_norm_rope_bwd(*{**BWD, **bad}.values()) == INVALID
    assert b"overlap" in lib.swiftkv_last_error()


@pytest.mark.parametrize("good", [dict(dq_in=at(0), dk_in=at(1)), dict(dq_in=at(2), dk_in=at(3)), dict(dq_in=at(0) + 5 * 2048), dict(q=at(2), q_stride=WIDE, dk_in=at(2) + 5 * ROW)])
def test_qk_norm_rope_bwd_takes_what_shares_no_byte(lib, good):
    if not torch.cuda.is_available():
        assert lib.swiftkv_qk_norm_rope_bwd(*{**BWD, **good}.values()) not in (0, INVALID)


@pytest.mark.parametrize("bad", [dict(out=at(0)), dict(out=at(0) + 7 * 2048 + 2046), dict(out=at(1) + 256 * 512 - 2), dict(out=at(2)), dict(lse=at(7)), dict(lse=at(0) + 64),
                                 dict(q_stride=WIDE, out=at(0) + 1024), dict(scratch=at(0) - 256), dict(scratch=at(7) - 256), dict(lse=at(8) + 4)])
def test_tree_attention_refuses_overlaps(lib, bad):
    assert lib.swiftkv_tree_attention(*{**TREE, **bad}.values()) == INVALID
    assert b"overlap" in lib.swiftkv_last_error()


@pytest.mark.parametrize("good", [dict(out=at(0) + 8 * 2048), dict(q_stride=WIDE, out=at(0) + 8 * ROW), dict(total_new=1, q_stride=WIDE, out=at(0) + 2048), dict(lse=at(7) + 8 * 2048)])
def test_tree_attention_takes_what_shares_no_byte(lib, good):
    if not torch.cuda.is_available():
        assert lib.swiftkv_tree_attention(*{**TREE, **good}.values()) not in (0, INVALID)


def test_token_logprobs_refuses_temperatures_without_a_reciprocal(lib):
    for t in (1e-45, 1e-40, 2.0 ** -126):
        assert lib.swiftkv_token_logprobs(*{**LP, "temperature": t}.values()) == INVALID
        assert lib.swiftkv_token_logprobs_bwd(*{**LPB, "temperature": t}.values()) == INVALID


def test_wrappers_refuse_host_tensors(lib):
    import paper_2410_03960_b200 as P
    x, i = torch.zeros(2, 4), torch.zeros(2, dtype=torch.int32)
    h = torch.zeros(2, 2, 8)
    for call in (lambda: P.token_logprobs(x, i), lambda: P.token_logprobs_bwd(x, i, x[:, 0], None, x[:, 0]), lambda: P.plan_pages(i, i, i, i[None], i, i[:1]),
                 lambda: P.qk_norm_rope(h, h, h, i, x, x, k_cache=h, v_cache=h), lambda: P.qk_norm_rope_bwd(h, h, h, h, i, x, x),
                 lambda: P.tree_attention(h, h, h, i, i, 1, 1, row0=i)):
        with pytest.raises(ValueError):
            call()


def test_wrappers_refuse_what_is_no_tensor(lib):
    import paper_2410_03960_b200 as P
    with pytest.raises(ValueError):
        P.token_logprobs_bwd("logits", None, None, None, None)
    with pytest.raises(ValueError):
        P.tree_attention(None, None, None, None, None, 1, 1)


def test_the_extension_checks_its_own_arguments(lib):
    from paper_2410_03960_b200 import verify
    ext = verify._load()
    for name in ("plan_pages", "qk_norm_rope", "qk_norm_rope_bwd", "tree_attention", "token_logprobs", "token_logprobs_bwd", "bind"):
        with pytest.raises(TypeError):
            getattr(ext, name)()
    with pytest.raises(ValueError):
        ext.bind(RuntimeError, {})
