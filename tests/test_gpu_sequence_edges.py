"""What calls of the sequence model's operators do at their edges: waits that run out, states in place where several blocks share a
sequence, values at the ends of float32's range, calls without tokens, launches in parts."""

import pytest
import torch

from paper_2205_13104_b200 import twa
from philox import dropout_numbers
from test_gpu_sequence_operators import BF16, DEV, F32, FILL, ROUND, clean, close, ctx, gen, ok, randn, scan_64  # noqa: F401 (two fixtures among them)

pytestmark = pytest.mark.gpu


def scan_case(g, lengths, channels, dtype, equal=False):
    """Inputs and a function that runs both directions into outputs of FILL."""
    q, n = len(lengths), sum(lengths)
    starts = None if equal else torch.tensor([sum(lengths[:i]) for i in range(q + 1)], device=DEV)
    x, f, dh = randn(g, n, channels).to(dtype), (2 * randn(g, n, channels) + 2).to(dtype), randn(g, n, channels).to(dtype)
    h0, d_last = randn(g, q, channels), randn(g, q, channels)
    states = torch.empty(twa.twa_gated_scan_states_bytes(n, q, channels), dtype=torch.uint8, device=DEV)

    def forward(ctx):
        h, last = torch.full_like(x, FILL), torch.full_like(h0, FILL)
        twa.twa_gated_scan(ctx, x, f, h, starts, q, h0, last, states)
        return h, last

    def backward(ctx):
        dx, df, dh0 = torch.full_like(x, FILL), torch.full_like(x, FILL), torch.full_like(h0, FILL)
        twa.twa_gated_scan_backward(ctx, dh, x, f, states, dx, df, starts, q, d_last, dh0)
        return dx, df, dh0

    return forward, backward


@pytest.mark.parametrize("cluster,rank,warp", [(2, 0, 0), (2, 1, 3), (2, 0, 7), (8, 0, 2), (8, 0, 7), (8, 7, 0), (8, 3, 5)])
@pytest.mark.parametrize("lengths,channels,dtype", [([4200], 64, F32), ([4200, 4200], 40, BF16), ([900, 0, 5000, 1, 2100], 24, F32), ([3000, 17, 4100], 71, BF16)])
def test_gated_scan_reports_a_wait_that_ran_out_in_any_warp(ctx, lengths, channels, dtype, cluster, rank, warp):
    """One warp of one block takes its first wait for one that ran out; the others of its block have had the maps.  It has to be
    reported, and nothing wrong may be stored: an output is right, or was not written."""
    forward, backward = scan_case(gen(sum(lengths) + channels), lengths, channels, dtype, len(set(lengths)) == 1)
    twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CLUSTER, cluster)
    twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CHANNELS, 64)
    try:
        for call in (forward, backward):
            want = call(ctx)
            ok(ctx)
            twa.twa_set_tuning(ctx, twa.TWA_TUNE_WAIT_LIMIT_MS, 5)
            twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_GIVE_UP, 1 + 8 * rank + warp)
            got = call(ctx)
            code, detail = twa.twa_get_status(ctx)
            assert code == twa.TWA_ERR_TIMEOUT and lengths[detail] > 0
            for a, b in zip(got, want):
                assert bool(((a == b) | (a == FILL)).all())
            assert not torch.equal(got[0], want[0])                # the warp's own rows at least
            twa.twa_clear_status(ctx)
            twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_GIVE_UP, 0)
            twa.twa_set_tuning(ctx, twa.TWA_TUNE_WAIT_LIMIT_MS, 0)
            assert all(torch.equal(a, b) for a, b in zip(call(ctx), want))
            ok(ctx)
    finally:
        for key in (twa.TWA_TUNE_SCAN_GIVE_UP, twa.TWA_TUNE_WAIT_LIMIT_MS, twa.TWA_TUNE_SCAN_CLUSTER, twa.TWA_TUNE_SCAN_CHANNELS):
            twa.twa_set_tuning(ctx, key, 0)


def test_the_scan_knob_for_waits_takes_what_it_means(ctx):
    for value in (1, 64, 0):
        twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_GIVE_UP, value)
    for value in (65, -1):
        with pytest.raises(twa.TwaError):
            twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_GIVE_UP, value)


@pytest.mark.parametrize("cluster", [2, 4, 8])
@pytest.mark.parametrize("lengths", [[300], [90, 0, 255, 1], [70] * 6, [2500, 40], [64, 128]])
@pytest.mark.parametrize("channels,dtype", [(64, F32), (48, BF16), (33, F32)])
def test_gated_scan_states_in_place_where_blocks_share_a_sequence(ctx, lengths, channels, dtype, cluster):
    """Every block of a cluster reads the state that enters, one writes the state that leaves: behind a barrier of all of them, in
    sequences of a single round too."""
    g = gen(sum(lengths) * cluster)
    q, n = len(lengths), sum(lengths)
    starts = None if len(set(lengths)) == 1 else torch.tensor([sum(lengths[:i]) for i in range(q + 1)], device=DEV)
    x, f, dh = randn(g, n, channels).to(dtype), (2 * randn(g, n, channels) + 2).to(dtype), randn(g, n, channels).to(dtype)
    h, dx, df = (torch.empty_like(x) for _ in range(3))
    states = torch.empty(twa.twa_gated_scan_states_bytes(n, q, channels), dtype=torch.uint8, device=DEV)
    twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CLUSTER, cluster)
    try:
        for _ in range(20):
            h0, d_last = randn(g, q, channels), randn(g, q, channels)
            last, dh0 = torch.empty_like(h0), torch.empty_like(h0)
            twa.twa_gated_scan(ctx, x, f, h, starts, q, h0, last, states)
            twa.twa_gated_scan_backward(ctx, dh, x, f, states, dx, df, starts, q, d_last, dh0)
            want = [t.clone() for t in (h, dx, df)]
            twa.twa_gated_scan(ctx, x, f, h, starts, q, h0, h0, states)
            twa.twa_gated_scan_backward(ctx, dh, x, f, states, dx, df, starts, q, d_last, d_last)
            assert torch.equal(h0, last) and torch.equal(d_last, dh0)
            assert all(torch.equal(a, b) for a, b in zip((h, dx, df), want))
    finally:
        twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CLUSTER, 0)
    ok(ctx)


@pytest.mark.parametrize("cluster", [0, 2, 8])
@pytest.mark.parametrize("lengths", [[1], [3, 1, 20, 0, 2], [2] * 9, [700], [129, 400], [1, 2, 1, 1, 3, 1, 1, 1, 1, 40, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1]])
@pytest.mark.parametrize("channels,dtype", [(64, F32), (71, F32), (64, BF16), (37, BF16), (70, BF16)])
def test_gated_scan_of_values_further_apart_than_the_largest_float(ctx, lengths, channels, dtype, cluster):
    """A state lies between its tokens, whatever their difference: 3e38 and -3e38 included."""
    g = gen(sum(lengths) + channels)
    q, n = len(lengths), sum(lengths)
    first = [sum(lengths[:i]) for i in range(q)]
    starts = None if len(set(lengths)) == 1 else torch.tensor(first + [n], device=DEV)
    x = ((0.5 + 0.5 * torch.rand((n, channels), generator=g, device=DEV)) * 3e38 * torch.sign(randn(g, n, channels))).to(dtype)
    f, dh = (3 * randn(g, n, channels)).to(dtype), (0.01 * randn(g, n, channels)).to(dtype)
    h0, d_last = 3e38 * torch.sign(randn(g, q, channels)), 0.01 * randn(g, q, channels)
    h, dx, df = (torch.empty_like(x) for _ in range(3))
    last, dh0 = torch.empty_like(h0), torch.empty_like(h0)
    states = torch.empty(twa.twa_gated_scan_states_bytes(n, q, channels), dtype=torch.uint8, device=DEV)
    twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CLUSTER, cluster)
    try:
        twa.twa_gated_scan(ctx, x, f, h, starts, q, h0, last, states)
        twa.twa_gated_scan_backward(ctx, dh, x, f, states, dx, df, starts, q, d_last, dh0)
    finally:
        twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CLUSTER, 0)
    scan_64.dtype = dtype
    want = scan_64(x, f, lengths, first, h0, dh, d_last)
    for name, got in (("h", h), ("dx", dx), ("df", df)):
        v, e = want[name]
        close(got, v, e + ROUND[dtype] * (v.abs() + e) + 1e-37)
    for name, got in (("h_last", last), ("dh0", dh0)):
        v, e = want[name]
        close(got, v, e + 1e-37)
    ok(ctx)


@pytest.mark.parametrize("experts", [1, 4, 1000])
def test_dispatch_of_no_tokens_with_room_for_some(ctx, experts):
    """A program's buffers stay as large as they are where a batch has no token: an empty tensor has no address, its buffers have one."""
    none, x = torch.empty((0, 2), dtype=torch.int64, device=DEV), torch.empty((0, 8), device=DEV)
    place, starts = torch.empty((0, 2), dtype=torch.int32, device=DEV), torch.full((experts + 1,), 9, dtype=torch.int32, device=DEV)
    out = torch.full((6, 8), FILL, device=DEV)
    twa.twa_expert_dispatch(ctx, x, none, experts, place, starts, out)
    assert bool((starts == 0).all()) and bool((out == FILL).all())
    back, h = torch.empty_like(x), torch.empty_like(x)
    twa.twa_expert_combine(ctx, out, place, None, back)
    twa.twa_expert_combine_backward(ctx, x, out, place, torch.empty((0, 2), device=DEV), out)
    twa.twa_dropout(ctx, x, 0.5, torch.tensor([1, 2], device=DEV), 0, h)
    h0, last = torch.ones(3, 8, device=DEV), torch.zeros(3, 8, device=DEV)
    states = torch.empty(1024, dtype=torch.uint8, device=DEV)
    for starts in (None, torch.zeros(4, dtype=torch.int64, device=DEV)):
        twa.twa_gated_scan(ctx, x, x, h, starts, 3, h0, last, states)
        assert torch.equal(last, h0)
        twa.twa_gated_scan_backward(ctx, x, x, x, states, h, back, starts, 3, h0, last.zero_())
        assert torch.equal(last, h0)
        last.zero_()
    assert bool((out == FILL).all())
    ok(ctx)


@pytest.mark.parametrize("shared", [("one block", 1, 64), ("clusters", 2, 64), ("clusters", 8, 16), ("by length", 0, 2560)], ids=lambda v: f"{v[0]}-{v[1]}")
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("wrong", [(0, -1), (3, 2000), (10, 1 << 40), (9, 1001)])
def test_gated_scan_leaves_wrong_sequences_alone_however_they_are_shared(ctx, shared, dtype, wrong):
    """Offsets outside the tokens where one block's opinion of them goes to others, or they are ranked by their length: sequences on
    both sides of a wrong offset are reported and left alone, the others give the bits that they give among right ones."""
    way, cluster, channels = shared
    n, edges = 1000, [0, 37, 300, 301, 301, 450, 600, 700, 790, 800, 1000]
    if way == "by length":                                        # more blocks than begin at once, fewer than twice as many
        blocks = (len(edges) - 1) * channels // 64
        sms = torch.cuda.get_device_properties(0).multi_processor_count
        assert 2 * sms < blocks <= 4 * sms
    at, value = wrong
    bad = [s for s in (at - 1, at) if 0 <= s < len(edges) - 1]
    q, g = len(edges) - 1, gen(channels + at)
    x, f, dh = randn(g, n, channels).to(dtype), (2 * randn(g, n, channels) + 2).to(dtype), randn(g, n, channels).to(dtype)
    h0, d_last = randn(g, q, channels), randn(g, q, channels)
    twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CLUSTER, cluster)
    twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CHANNELS, channels if cluster else 0)
    states = torch.empty(twa.twa_gated_scan_states_bytes(n, q, channels), dtype=torch.uint8, device=DEV)

    def run(edges, back):
        starts = torch.tensor(edges, device=DEV)
        out = [torch.full_like(x, FILL) for _ in range(2)] + [torch.full_like(h0, FILL)]
        if back:
            twa.twa_gated_scan_backward(ctx, dh, x, f, states, out[0], out[1], starts, q, d_last, out[2])
        else:
            twa.twa_gated_scan(ctx, x, f, out[0], starts, q, h0, out[2], states)
        return out

    try:
        for back in (False, True):
            want = run(edges, back)
            ok(ctx)
            got = run(edges[:at] + [value] + edges[at + 1:], back)
            code, detail = twa.twa_get_status(ctx)
            assert code == twa.TWA_ERR_INVALID_ARG and detail in bad
            twa.twa_clear_status(ctx)
            for s in bad:
                for t in want[:2]:
                    t[edges[s]: edges[s + 1]] = FILL
                want[2][s] = FILL
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            if not back:
                run(edges, back)                                   # the states of all sequences, for the way back
    finally:
        twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CLUSTER, 0)
        twa.twa_set_tuning(ctx, twa.TWA_TUNE_SCAN_CHANNELS, 0)


def test_dropout_in_more_than_one_launch(ctx):
    """A launch counts its work in 31 bits; rows beyond that go in another, with the numbers of their own places."""
    rows, cols = twa.TWA_DROPOUT_MAX_ROWS, 16
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB of device memory")
    x = torch.ones((rows, cols), dtype=BF16, device=DEV)
    twa.twa_dropout(ctx, x, 0.5, torch.tensor([5, 6], device=DEV), 7, x)
    for first, count in ((0, 8), (rows // 2 - 4, 8), (rows - 1000, 1000)):        # the second launch begins some hundred rows before the end
        kept = torch.from_numpy(dropout_numbers(5, 6, 7, count, cols, first) >= 32768).to(DEV)
        assert torch.equal(x[first: first + count], torch.where(kept, 2.0, 0.0).to(BF16))
    ok(ctx)
