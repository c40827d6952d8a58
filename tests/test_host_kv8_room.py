"""CPU-only checks of how long slices on the 8-bit cache go where the workspace is smaller than what they ask for: a call whose blocks of rows do not fill the
chip keeps the key ranges that there is room for."""
import ctypes
import random

import pytest

NULL, SHAPE, WORKSPACE = -1, -2, -6


@pytest.fixture(scope="module")
def sp():
    import paper_2504_14519_amd as sp_
    return sp_


def params(sp, B, s, Hq, Hkv, D, off, begin=0):
    N, row, kv = off + s, Hq * D, Hkv * D
    return sp.AttnParams(B, s, Hq, Hkv, D, 1, N, off, begin, N, 0.1, sp.BF16, s * row, row, D, N * kv, kv, D, s * row, row, D)


def asked(sp, p):
    n = ctypes.c_size_t(0)
    assert sp.lib.slimpipe_attn_kv8_workspace_bytes(ctypes.byref(p), 64, ctypes.byref(n)) == 0
    return n.value


def path(sp, p, room):
    x = sp.slimpipe_attn_kv8_call_path(p, 64, room)
    return x.copy, x.ranges, x.workgroup_rows


def range_bytes(p):
    return p.batch * p.n_q_heads * p.s_q * (p.head_dim + 1) * 4


def copy_bytes(p):
    return 4 * p.head_dim * p.batch * p.n_kv_heads * (p.kv_end - p.kv_begin)


def test_few_blocks_of_rows_keep_their_ranges(sp):
    """256 rows of 8 heads on one (8 blocks of 256) behind 32512 keys; 256 compute units, as where no device can be asked."""
    p = params(sp, 1, 256, 8, 1, 128, 32512)
    need, copy, each = asked(sp, p), copy_bytes(p), range_bytes(p)
    assert path(sp, p, need)[0] == 1 and path(sp, p, 1 << 40) == path(sp, p, need)
    # room for the copy and nothing beside it: undivided it would be 8 workgroups
    got = path(sp, p, copy + 512)
    assert got == (0, (copy + 512) // each, 128)
    for n in (2, 3, 5, 8, 12):
        assert path(sp, p, n * each + 1024) == (0, n, 128)
    # a range alone: blocks of 128 rows, twice as many workgroups
    for room in (0, each, 2 * each - 256):
        assert path(sp, p, room) == (0, 1, 128)


def test_calls_that_fill_the_chip_and_calls_without_a_range_copy(sp):
    # 640 blocks of rows: the copy undivided costs nothing; tiles would be 1.22 times as long
    p = params(sp, 1, 4096, 40, 40, 128, 14592)
    assert path(sp, p, copy_bytes(p) + 512)[:2] == (1, 1) and path(sp, p, copy_bytes(p) - 512)[0] == 0 and path(sp, p, 0) == (0, 1, 256)
    # 64 blocks, room for the copy or for one range, not for two
    p = params(sp, 1, 2048, 8, 1, 128, 30700)
    assert 2 * range_bytes(p) > copy_bytes(p) + 512
    assert path(sp, p, copy_bytes(p) + 512)[:2] == (1, 1) and path(sp, p, 2 * range_bytes(p) + 1024) == (0, 2, 128)
    # three ranges of 64 blocks: more than half of the chip with eight waves
    p = params(sp, 1, 4096, 4, 4, 128, 12000)
    assert path(sp, p, 2 * range_bytes(p) + 1024) == (0, 2, 128) and path(sp, p, 3 * range_bytes(p) + 1024) == (0, 3, 256)


def test_paths_fit_their_room(sp):
    """Whatever the room: what the path needs fits; a tile call never has fewer ranges than with less room; the copy is taken with room for it alone; all that is
    asked for gives what any more gives; calls of fewer rows than have a copy are refused below what they ask for."""
    rng = random.Random(12)
    copies = tiles = 0
    for _ in range(1500):
        Hq, Hkv = rng.choice([(8, 1), (4, 4), (8, 2), (12, 4), (16, 16), (40, 40)])
        s, off = int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 16))
        p = params(sp, rng.choice([1, 1, 2, 3]), s, Hq, Hkv, rng.choice([64, 128]), off, rng.choice([0, 0, off // 2]))
        need, each, copy, long_ = asked(sp, p), range_bytes(p), copy_bytes(p), Hq // Hkv * s >= 2048
        assert path(sp, p, need) == path(sp, p, 1 << 50)
        last = 0
        for room in sorted([0, need // 7, need // 3, need // 2, copy - 1, copy + 512, copy + each, need - 1]):
            if not 0 <= room < need:
                continue
            if not long_:
                with pytest.raises(sp.SlimpipeError):
                    sp.slimpipe_attn_kv8_call_path(p, 64, room)
                continue
            got = path(sp, p, room)
            assert got[2] in ((0,) if got[0] else (128, 256)), (s, off, room)
            assert (copy if got[0] else 0) + (each * got[1] if got[1] > 1 else 0) <= room, (s, off, room)
            if got[0]:
                copies += 1
                continue
            assert got[1] >= last
            last = got[1]
            tiles += 1
    assert copies > 100 and tiles > 500


def test_refusals(sp):
    p = params(sp, 1, 256, 8, 1, 128, 32512)
    out = (ctypes.c_int32 * 3)()
    call = lambda p, block, room: sp.lib.slimpipe_attn_kv8_call_path(p, block, room, ctypes.cast(out, ctypes.POINTER(sp.binding.Kv8CallPath)))
    assert call(ctypes.byref(p), 48, 0) == SHAPE and call(None, 64, 0) == NULL
    assert sp.lib.slimpipe_attn_kv8_call_path(ctypes.byref(p), 64, 0, None) == NULL
    token = params(sp, 1, 1, 8, 1, 128, 32767)
    assert call(ctypes.byref(token), 64, 0) == WORKSPACE and call(ctypes.byref(token), 64, asked(sp, token)) == 0 and tuple(out)[::2] == (0, 32)
    token.s_q = 0
    assert call(ctypes.byref(token), 64, 1 << 20) == SHAPE
