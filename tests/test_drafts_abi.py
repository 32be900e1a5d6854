"""Refusals of the calls of a step of drafted tokens, found on the host before anything is launched, and the tree's bits."""
import ctypes as C
import random

import pytest

from paper_2302_01382_amd import mpq
from test_abi_host import FAKE, FAKE16, needs_no_gpu
from test_serving_abi import BIG, ODD, kv

INF, NAN = float("inf"), float("nan")


def caller(f, ok):
    """f with the arguments `ok` but for those named _i."""
    def but(**kw):
        a = list(ok)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return f(*a)
    return but


@needs_no_gpu
def test_linear_groups_refuses():
    # x, type, M, N, K, stride, w, group, steps, their type, act, y type, y, stream
    but = caller(mpq.lib().mpq_linear_groups, [FAKE16, 1, 4, 8, 256, 256, FAKE16, 64, FAKE16, 0, 0, 1, FAKE16, None])
    for i in (0, 6, 8, 12):
        assert but(**{"_%d" % i: None}) == mpq.ERR_NULL
    for i in (1, 9, 10, 11):
        for v in (-1, 3):
            assert but(**{"_%d" % i: v}) == mpq.ERR_SHAPE
    for i in (3, 4):
        for v in (0, -64):
            assert but(**{"_%d" % i: v}) == mpq.ERR_SHAPE
    assert but(_2=-1) == mpq.ERR_SHAPE
    assert but(_5=255) == mpq.ERR_SHAPE                                    # rows overlap
    for group in (0, 16, 48, 256, -64):
        assert but(_7=group) == mpq.ERR_SHAPE
    assert but(_4=96, _5=96) == mpq.ERR_SHAPE                              # a group and a half
    assert but(_4=2 ** 31, _5=2 ** 31) == mpq.ERR_SHAPE
    assert but(_2=2 ** 40, _5=2 ** 40) == mpq.ERR_SHAPE
    assert but(_3=2 ** 27) == mpq.ERR_SHAPE and but(_2=64 * 65535 + 1) == mpq.ERR_SHAPE  # grids that a launch cannot count
    assert but(_1=0, _2=32 * 65535 + 1) == mpq.ERR_SHAPE and but(_1=0, _2=32 * 65535, _0=None) == mpq.ERR_NULL           # blocks of 32 rows
    assert but(_2=64 * 65535, _0=None) == mpq.ERR_NULL
    assert but(_0=ODD) == mpq.ERR_ALIGN and but(_8=C.c_void_p(0x10002)) == mpq.ERR_ALIGN
    assert but(_8=ODD, _9=2) == mpq.ERR_ALIGN and but(_12=ODD) == mpq.ERR_ALIGN and but(_11=0, _12=C.c_void_p(0x10002)) == mpq.ERR_ALIGN
    assert but(_2=0, _0=None, _6=None, _8=None, _12=None) == mpq.OK        # no rows


@needs_no_gpu
def test_rotate_heads_refuses():
    # type, rows, dim, q, ts, hs, heads, k, ts, hs, heads, positions, frequencies, pairs, layout, weights, eps, q_out, ts, hs, k_out, ts, hs
    other = C.c_void_p(0x20000)
    but = caller(mpq.lib().mpq_rotate_heads, [1, 5, 64, FAKE16, 256, 64, 4, FAKE16, 128, 64, 2, FAKE, FAKE, 32, 0, FAKE, FAKE, 1e-6,
                                              other, 256, 64, other, 128, 64, None])
    for i in (3, 7, 11, 12, 18, 21):
        assert but(**{"_%d" % i: None}) == mpq.ERR_NULL
    for v in (-1, 3):
        assert but(_0=v) == mpq.ERR_SHAPE
    for dim in (0, -16, 8, 40, 272):
        assert but(_2=dim) == mpq.ERR_SHAPE
    assert but(_1=-1) == mpq.ERR_SHAPE and but(_6=-1) == mpq.ERR_SHAPE and but(_10=-2) == mpq.ERR_SHAPE
    for pairs in (-4, 2, 30, 36):
        assert but(_13=pairs) == mpq.ERR_SHAPE
    for layout in (-1, 2):
        assert but(_14=layout) == mpq.ERR_SHAPE
    for eps in (0.0, -1.0, INF, NAN, 1e-40):
        assert but(_17=eps) == mpq.ERR_SHAPE
    for i in (4, 5, 8, 9, 19, 20, 22, 23):
        for v in (-1, 1 << 62):
            assert but(**{"_%d" % i: v}) == mpq.ERR_SHAPE
    assert but(_19=255) == mpq.ERR_SHAPE and but(_20=63) == mpq.ERR_SHAPE and but(_22=64) == mpq.ERR_SHAPE   # outputs that overlap
    assert but(_18=FAKE16, _19=512) == mpq.ERR_SHAPE and but(_21=FAKE16, _23=80, _22=256) == mpq.ERR_SHAPE   # in place, other strides
    assert but(_3=ODD) == mpq.ERR_ALIGN and but(_0=0, _21=C.c_void_p(0x20002)) == mpq.ERR_ALIGN
    for i in (11, 12, 15, 16):
        assert but(**{"_%d" % i: C.c_void_p(0x1002)}) == mpq.ERR_ALIGN
    assert but(_6=2 ** 30, _5=0, _20=64) == mpq.ERR_SHAPE
    assert but(_1=0, _3=None, _7=None, _18=None, _21=None, _11=None) == mpq.OK                               # no rows
    assert but(_6=0, _10=0, _3=None, _7=None, _18=None, _21=None, _4=-1) == mpq.OK                           # no heads


@needs_no_gpu
def test_kv_attention_tree_refuses():
    L = mpq.lib()
    ok = [1, FAKE16, 256, 64, 4, 0.125, FAKE16, 1, FAKE16, 256, 64, FAKE16, BIG, None]

    def but(cache=None, batch=None, **kw):
        return caller(L.mpq_kv_attention_tree, list(kv(cache, batch)) + ok)(**{"_%d" % (int(i[1:]) + 2): v for i, v in kw.items()})

    assert L.mpq_kv_attention_tree(None, kv()[1], *ok) == mpq.ERR_NULL and L.mpq_kv_attention_tree(kv()[0], None, *ok) == mpq.ERR_NULL
    for n in ("k_codes", "v_codes", "k_absmax", "v_absmax"):
        assert but({n: None}) == mpq.ERR_NULL and but({n: 0x10002}) == mpq.ERR_ALIGN
    assert but({"dim": 24}) == mpq.ERR_SHAPE and but({"page": 48}) == mpq.ERR_SHAPE and but({"bits": 9}) == mpq.ERR_BITS
    for n in ("rows", "seqs", "max_new", "max_len", "table_pages"):
        assert but(batch={n: -1}) == mpq.ERR_SHAPE
    for i in (1, 6, 8):
        assert but(**{"_%d" % i: None}) == mpq.ERR_NULL
    assert but(_0=3) == mpq.ERR_SHAPE
    for heads in (0, -2, 3):
        assert but(_4=heads) == mpq.ERR_SHAPE
    for scale in (NAN, INF, -INF):
        assert but(_5=scale) == mpq.ERR_SHAPE
    for words in (-1, 0):
        assert but(_7=words) == mpq.ERR_SHAPE
    assert but(batch={"rows": 2 ** 31 - 1, "max_new": 1}, _7=2 ** 31 - 1) == mpq.ERR_SHAPE
    for i in (2, 3, 9, 10):
        for v in (-1, 1 << 62):
            assert but(**{"_%d" % i: v}) == mpq.ERR_SHAPE
    assert but(_9=255) == mpq.ERR_SHAPE and but(_10=48) == mpq.ERR_SHAPE     # outputs that overlap
    assert but(_1=ODD) == mpq.ERR_ALIGN and but(_8=ODD) == mpq.ERR_ALIGN and but(_6=C.c_void_p(0x10004)) == mpq.ERR_ALIGN
    long = {"max_len": 100000, "table_pages": 7000}
    need = L.mpq_kv_attention_tree_workspace_bytes(*kv(batch=long), 1, 4)
    assert need > 0 and but(batch=long, _12=need - 1) == mpq.ERR_WORKSPACE and but(batch=long, _11=None) == mpq.ERR_WORKSPACE
    assert but(batch=long, _11=C.c_void_p(0x10008)) == mpq.ERR_ALIGN
    assert L.mpq_kv_attention_tree_workspace_bytes(*kv({"dim": 24}), 1, 4) == 0
    assert L.mpq_kv_attention_tree_workspace_bytes(*kv(batch={"max_len": 50}), 1, 4) == 0
    assert but(batch={"rows": 2 ** 31 - 1, "max_new": 1}, _7=2 ** 17) == mpq.ERR_SHAPE   # the bits' bytes overflow
    assert but(batch={"rows": 0}, _1=None, _6=None, _8=None) == mpq.OK
    assert but(batch={"seqs": 2 ** 31 - 1, "rows": 2 ** 31 - 1, "max_new": 2 ** 31 - 1, "table_pages": 2 ** 31 - 1}, _7=2 ** 26) == mpq.ERR_SHAPE


@needs_no_gpu
def test_token_logprobs_refuses():
    L = mpq.lib()
    # logits, type, rows, vocab, stride, scale, tokens, logprob, entropy, top, top_logprob, top_index, ws, ws_bytes
    but = caller(L.mpq_token_logprobs, [FAKE16, 1, 3, 90000, 90000, 1.0, FAKE, FAKE, FAKE, 5, FAKE, FAKE, FAKE16, BIG, None])
    for i in (0, 6, 10, 11):
        assert but(**{"_%d" % i: None}) == mpq.ERR_NULL
    assert but(_7=None, _8=None, _9=0) == mpq.ERR_NULL                      # no output
    for t in (-1, 3):
        assert but(_1=t) == mpq.ERR_SHAPE
    assert but(_2=-1) == mpq.ERR_SHAPE and but(_2=2 ** 45) == mpq.ERR_SHAPE
    for vocab in (0, -5, 2 ** 22 + 1):
        assert but(_3=vocab, _4=2 ** 23) == mpq.ERR_SHAPE
    assert but(_4=89999) == mpq.ERR_SHAPE
    for scale in (0.0, -1.0, INF, NAN):
        assert but(_5=scale) == mpq.ERR_SHAPE
    assert L.mpq_token_logprobs_workspace_bytes(2 ** 62, 50000, 1, 5) == 0 and but(_2=2 ** 62) == mpq.ERR_SHAPE
    for top in (-1, 33):
        assert but(_9=top) == mpq.ERR_SHAPE
    assert but(_0=ODD) == mpq.ERR_ALIGN
    for i in (6, 7, 8, 10, 11):
        assert but(**{"_%d" % i: C.c_void_p(0x1002)}) == mpq.ERR_ALIGN
    need = L.mpq_token_logprobs_workspace_bytes(3, 90000, 1, 5)
    assert need > 0 and but(_13=need - 1) == mpq.ERR_WORKSPACE and but(_12=None) == mpq.ERR_WORKSPACE
    assert but(_12=C.c_void_p(0x10008)) == mpq.ERR_ALIGN
    assert L.mpq_token_logprobs_workspace_bytes(3, 1000, 1, 5) == 0 and L.mpq_token_logprobs_workspace_bytes(3, 90000, 7, 5) == 0
    assert but(_2=0, _0=None, _6=None, _10=None) == mpq.OK


@needs_no_gpu
def test_an_output_of_the_layer_in_a_place_that_is_read_is_refused():
    """Workgroups would read what others have written: found on the host (nothing here reaches a launch)."""
    L = mpq.lib()
    P = lambda a: C.c_void_p(0x1000000 + 2 * a)  # noqa: E731  (element a of one buffer of 2-byte values)
    # x, type, M, N, K, stride, w, group, steps, their type, act, y type, y, stream
    far = C.c_void_p(0x8000000)
    but = caller(L.mpq_linear_groups, [P(0), 1, 4, 8, 256, 512, far, 64, C.c_void_p(0x9000000), 0, 0, 1, P(256), None])
    assert but(_12=P(0)) == mpq.ERR_SHAPE and but(_12=P(255)) == mpq.ERR_SHAPE and but(_12=P(3 * 512 + 255)) == mpq.ERR_SHAPE
    assert but(_12=P(512 - 31)) == mpq.ERR_SHAPE                                          # the last of 32 elements
    assert but(_12=far) == mpq.ERR_SHAPE and but(_12=C.c_void_p(0x8000000 + 8 * 128 - 2)) == mpq.ERR_SHAPE   # the codes
    assert but(_12=C.c_void_p(0x9000000 + 8 * 4 * 4 - 4)) == mpq.ERR_SHAPE                 # the steps


@needs_no_gpu
def test_rotated_heads_in_a_place_that_is_read_or_written_are_refused():
    L = mpq.lib()
    P = lambda a: C.c_void_p(0x1000000 + 2 * a)  # noqa: E731
    # type, rows, dim, q, ts, hs, heads, k, ts, hs, heads, positions, frequencies, pairs, layout, weights, eps, q_out, ts, hs, k_out, ts, hs
    R = 8 * 64                                                                             # a row of eight heads
    q, k, out = 0, 4 * 64, 100000
    but = caller(L.mpq_rotate_heads, [1, 5, 64, P(q), R, 64, 4, P(k), R, 64, 2, FAKE, FAKE, 32, 0, FAKE, FAKE, 1e-6,
                                      P(out), R, 64, P(out + k), R, 64, None])
    assert but(_21=P(out)) == mpq.ERR_SHAPE and but(_21=P(out + k - 1)) == mpq.ERR_SHAPE    # both outputs in one place, or one element too near
    assert but(_21=P(out + R - 2 * 64 + 1)) == mpq.ERR_SHAPE                               # into the next row's
    assert but(_21=P(out + 4 * R + 3 * 64 + 63)) == mpq.ERR_SHAPE                          # q's last element
    assert but(_21=P(out - 5 * R + 7 * 64 + 1)) == mpq.ERR_SHAPE
    assert but(_19=R, _20=128, _21=P(out + 63), _22=R, _23=128) == mpq.ERR_SHAPE           # heads in turn
    assert but(_21=P(out + 1024), _22=R + 64) == mpq.ERR_SHAPE                             # rows of another length among them
    assert but(_18=P(q + 16)) == mpq.ERR_SHAPE and but(_18=P(k), _21=P(out)) == mpq.ERR_SHAPE and but(_21=P(q)) == mpq.ERR_SHAPE
    assert but(_18=P(q), _21=P(k - 1)) == mpq.ERR_SHAPE and but(_18=P(q + R), _19=R) == mpq.ERR_SHAPE


@needs_no_gpu
def test_places_of_queries_and_keys():
    """Patterns of few rows and heads of two outputs in one buffer against the elements that they cover, and of an output and the other's input.  A
    call that is taken ends at its launch, without a GPU.  (Rows of two lengths among one another count as one place.)"""
    r = random.Random(5)
    L, dim, seen = mpq.lib(), 16, {}
    far = [C.c_void_p(0x8000000 * i) for i in range(1, 5)]
    for trial in range(30000):
        rows, qh, kh = r.choice((1, 2, 3, 4)), r.choice((1, 2, 3, 5)), r.choice((1, 2, 4))
        strides = (16, 17, 24, 32, 33, 48, 64, 80, 96, 112, 128, 160, 200)
        q_ts, q_hs, k_hs = r.choice(strides), r.choice(strides), r.choice(strides)
        k_ts = q_ts if r.random() < 0.8 else r.choice(strides)
        at = r.choice((0, 1, 15, 16, 17, 32, 48, 64, 80, -16, -15, -40, -64, 100, 200, 300, 500, -200, -300))
        cells = lambda at, heads, ts, hs: [at + i * ts + h * hs + d for i in range(rows) for h in range(heads) for d in range(dim)]  # noqa: E731
        a, b = cells(0, qh, q_ts, q_hs), cells(at, kh, k_ts, k_hs)
        if len(set(a)) < len(a) or len(set(b)) < len(b):
            continue   # (each alone is looked at elsewhere)
        place = C.c_void_p(0x1000000), C.c_void_p(0x1000000 + 2 * at)
        if trial % 2:
            ins, outs = (far[0], far[1]), place
        else:
            ins, outs = (far[0], place[1]), (place[0], far[2])
        rc = L.mpq_rotate_heads(1, rows, dim, ins[0], 0, 16, qh, ins[1], k_ts, k_hs, kh, None, None, 0, 0, None, None, 1e-6,
                                outs[0], q_ts, q_hs, outs[1], k_ts, k_hs, None)
        meet = bool(set(a) & set(b))
        among = min(b) <= max(a) and min(a) <= max(b)
        if meet or not among or rows == 1 or q_ts == k_ts:
            assert rc == (mpq.ERR_SHAPE if meet else mpq.ERR_HIP), (rows, qh, kh, q_ts, q_hs, k_ts, k_hs, at, rc)
            seen[meet, among] = seen.get((meet, among), 0) + 1
        else:
            assert rc == mpq.ERR_SHAPE
    assert min(seen.get(x, 0) for x in ((True, True), (False, True), (False, False))) > 200, seen


def test_tree_bits():
    # 0 and 1 continue the sequence, 2 and 3 continue 0, 4 continues 3
    assert mpq.tree_bits([-1, -1, 0, 0, 3]).tolist() == [[0b1], [0b10], [0b101], [0b1001], [0b11001]]
    chain = mpq.tree_bits(range(-1, 129))
    assert chain.shape == (130, 3) and chain[63].tolist() == [-1, 0, 0] and chain[129].tolist() == [-1, -1, 3]
    assert chain[62].tolist() == [2 ** 63 - 1, 0, 0]
    assert mpq.tree_bits([]).shape == (0, 1)
    for parents in ([0], [-1, 1], [-2]):
        with pytest.raises(ValueError):
            mpq.tree_bits(parents)
