"""Long lists of slots, checked on the host; no GPU: the last entry is refused after all others have been looked at."""
import ctypes
import time

import card_inputs as ci
import paper_2508_04462_amd as card


def test_lists_of_pages_far_apart_take_no_longer():
    """Pages of a sequence lie far apart where many sequences grow side by side: at any distance the slots are told apart as quickly."""
    cfg, n = card.make_cfg(ci.SHAPES["tiny"], 256), 100000
    kv = card.CardKV(0x10000, 0x10000, None, 1 << 26, -1)

    def seconds(stride):
        slots = [(p // 16) * stride * 16 + p % 16 for p in range(n)]
        dst, src = (ctypes.c_int32 * (n + 1))(*slots, 5), (ctypes.c_int32 * (n + 1))(*[1000000007] * n, -1)
        best = 1e9
        for _ in range(3):
            t = time.perf_counter()
            assert card.lib.card_kv_move_slots(cfg, kv, n + 1, src, dst, None) == card.CARD_ERANGE
            best = min(best, time.perf_counter() - t)
        return best

    near = seconds(1)
    for stride in (64, 256, 4096):
        assert seconds(stride) <= 25 * near + 0.002, stride
