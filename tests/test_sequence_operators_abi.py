"""What of the sequence model's operators runs without a GPU: sizes, refusals before anything is enqueued, the generator."""

import pytest
import torch

from paper_2205_13104_b200 import twa
from philox import philox4x32
from test_operators_abi import on_device


def test_generator_gives_its_published_numbers():
    """The known answers that its authors publish for ten rounds."""
    known = [((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
             ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
             ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]
    for counter, key, want in known:
        assert tuple(int(v) for v in philox4x32(counter, key)) == want


def test_state_sizes():
    twa.build_library()
    size = twa.twa_gated_scan_states_bytes
    assert size(0, 0, 8) == 0
    assert size(1, 1, 8) >= 4 * 8
    assert size(65536, 3, 100) >= 4 * 100 * (65536 // 8)
    # every sequence's states have a place of their own, wherever sequences begin
    for rows in (8, 16):                        # from one kept state to the next, of float32 and bfloat16
        for lengths in ([1] * 9, [63, 65, 64, 1], [0, 0, 200, 0], [64] * 5, [5, 500], [7, 9, 8, 15, 17], [16] * 4):
            at, end = 0, 0
            for s, n in enumerate(lengths):
                first = at // rows + s
                assert first >= end
                end, at = first + -(-n // rows), at + n
            assert end * 4 * 8 <= size(at, len(lengths), 8)
    assert size(-1, 1, 8) == 0 and size(8, -1, 8) == 0 and size(8, 1, 0) == 0 and size(8, 1, twa.TWA_SCAN_MAX_CHANNELS + 1) == 0


def test_calls_without_a_context_are_refused():
    twa.build_library()
    lib, d, bad = twa.load(), 4096, twa.TWA_ERR_INVALID_ARG            # addresses that are never looked at
    assert lib.twa_dropout(None, d, 8, 0, 4, 8, 0.1, d, 0, None, 0, d, 8) == bad
    assert lib.twa_dropout_backward(None, d, 8, 0, 4, 8, 0.1, d, 0, d, 8) == bad
    assert lib.twa_gated_scan(None, d, 8, d, 8, 0, 4, 8, None, 0, 1, None, d, 8, None, None, 0) == bad
    assert lib.twa_gated_scan_backward(None, d, 8, d, 8, d, 8, 0, 4, 8, None, 0, 1, d, 1 << 20, None, d, 8, d, 8, None) == bad
    assert lib.twa_expert_dispatch(None, d, 8, 0, 4, 8, d, 0, 2, 4, d, d, None, d, 8) == bad
    assert lib.twa_expert_combine(None, d, 8, 0, 8, d, d, 4, 2, 8, d, 8) == bad
    assert lib.twa_expert_combine_backward(None, d, 8, d, 8, 0, 8, d, d, 4, 2, 8, d, 8, d) == bad


def test_wrong_tensors_are_refused():
    twa.build_library()
    ctx = twa.Context()                        # no handle: a call that gets through the binding's checks is refused as without a context
    ctx.device = 0
    t = on_device(0)
    i32, i64 = dict(dtype=torch.int32), dict(dtype=torch.int64)
    rng = t(2, **i64)

    def refused(call, *args, **kw):
        with pytest.raises((ValueError, TypeError)):
            call(ctx, *args, **kw)

    refused(twa.twa_dropout, t(4, 8), 0.1, t(2, **i32), 0, t(4, 8))
    refused(twa.twa_dropout, t(4, 8), 0.1, t(3, **i64), 0, t(4, 8))
    refused(twa.twa_dropout, t(4, 8, dtype=torch.float16), 0.1, rng, 0, t(4, 8, dtype=torch.float16))
    refused(twa.twa_dropout, t(4, 8), 0.1, rng, 0, t(4, 9))
    refused(twa.twa_dropout, t(4, 8), 0.1, rng, 0, t(4, 8), t(4, 8, dtype=torch.bfloat16))
    refused(twa.twa_dropout, t(8, 4).T, 0.1, rng, 0, t(4, 8))
    refused(twa.twa_gated_scan, t(4, 8), t(4, 9), t(4, 8))
    refused(twa.twa_gated_scan, t(4, 8), t(4, 8), t(4, 8, dtype=torch.bfloat16))
    refused(twa.twa_gated_scan, t(4, 8), t(4, 8), t(4, 8), t(2, **i64), 2)
    refused(twa.twa_gated_scan, t(4, 8), t(4, 8), t(4, 8), t(3), 2)
    refused(twa.twa_gated_scan, t(4, 8), t(4, 8), t(4, 8), None, 2, t(1, 8))
    refused(twa.twa_gated_scan_backward, t(4, 8), t(4, 8), t(4, 8), t(8), t(4, 8), t(4, 8), None, 2, t(2, 7))
    refused(twa.twa_expert_dispatch, t(4, 8), t(4, 2, **i64), 3, t(4, 2, **i32), t(3, **i32), t(8, 8))
    refused(twa.twa_expert_dispatch, t(4, 8), t(4, 2, **i64), 3, t(4, 2, **i32), t(4, **i32), t(7, 8))
    refused(twa.twa_expert_dispatch, t(4, 8), t(4, 2, **i64), 3, t(4, 2, **i32), t(4, **i32), None)
    refused(twa.twa_expert_dispatch, t(4, 8), t(2, 4, **i64), 3, t(4, 2, **i32), t(4, **i32), t(8, 8))
    refused(twa.twa_expert_dispatch, t(4, 8), t(4, 2), 3, t(4, 2, **i32), t(4, **i32), t(8, 8))
    refused(twa.twa_expert_dispatch, t(4, 8), t(4, 2, **i64), 3, t(4, 2, **i64), t(4, **i32), t(8, 8))
    refused(twa.twa_expert_combine, t(8, 8), t(4, 2, **i32), t(4, 3), t(4, 8))
    refused(twa.twa_expert_combine, t(8, 8), t(4, 2, **i32), None, t(4, 9))
    refused(twa.twa_expert_combine_backward, t(4, 8), t(8, 8), t(4, 2, **i32), t(4, 2), t(7, 8))


def test_tensors_of_another_device_than_the_contexts_are_refused():
    twa.build_library()
    ctx = twa.Context()
    ctx.device = 0
    here, there = on_device(0), on_device(1)

    def calls(n):
        """Every call with its n-th tensor on the other device."""
        def t(i, *shape, dtype=torch.float32):
            return (there if i == n else here)(*shape, dtype=dtype)

        i32, i64, u8 = (dict(dtype=d) for d in (torch.int32, torch.int64, torch.uint8))
        yield 4, lambda: twa.twa_dropout(ctx, t(0, 4, 8), 0.1, t(1, 2, **i64), 0, t(2, 4, 8), t(3, 4, 8))
        yield 3, lambda: twa.twa_dropout_backward(ctx, t(0, 4, 8), 0.1, t(1, 2, **i64), 0, t(2, 4, 8))
        yield 7, lambda: twa.twa_gated_scan(ctx, t(0, 4, 8), t(1, 4, 8), t(2, 4, 8), t(3, 3, **i64), 2, t(4, 2, 8), t(5, 2, 8), t(6, 64, **u8))
        yield 9, lambda: twa.twa_gated_scan_backward(ctx, t(0, 4, 8), t(1, 4, 8), t(2, 4, 8), t(3, 64, **u8), t(4, 4, 8), t(5, 4, 8),
                                                     t(6, 3, **i64), 2, t(7, 2, 8), t(8, 2, 8))
        yield 6, lambda: twa.twa_expert_dispatch(ctx, t(0, 4, 8), t(1, 4, 2, **i64), 3, t(2, 4, 2, **i32), t(3, 4, **i32), t(4, 8, 8), t(5, 8, **i32))
        yield 4, lambda: twa.twa_expert_combine(ctx, t(0, 8, 8), t(1, 4, 2, **i32), t(2, 4, 2), t(3, 4, 8))
        yield 6, lambda: twa.twa_expert_combine_backward(ctx, t(0, 4, 8), t(1, 8, 8), t(2, 4, 2, **i32), t(3, 4, 2), t(4, 8, 8), t(5, 4, 2))

    for n in range(9):
        for count, call in calls(n):
            if n < count:
                with pytest.raises(ValueError, match="device"):
                    call()
    for count, call in calls(-1):              # and with all on the context's device the checks let them through
        with pytest.raises(twa.TwaError):
            call()
