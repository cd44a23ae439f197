"""it_experts_forward against its formula in 64 bits."""
import pytest
import torch

from paper_2307_00228_b200 import binding as B
from block_util import BF16, F32, check_experts, experts_case, experts_desc, run_experts

pytestmark = pytest.mark.gpu

SHAPES = [  # n, experts, top_k, in, hidden, out
    (1, 4, 2, 64, 128, 64), (1, 16, 2, 256, 1024, 256), (3, 8, 3, 48, 80, 112), (7, 3, 1, 128, 0, 128), (130, 4, 2, 64, 256, 64), (257, 5, 2, 96, 192, 32),
    (1000, 16, 4, 128, 512, 128), (640, 1, 1, 16, 16, 16), (513, 7, 2, 272, 0, 528), (300, 40, 3, 512, 144, 256), (2000, 2, 2, 64, 64, 768)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("kind", ["f32", "bf16", "eight"])
@pytest.mark.parametrize("gated,act", [(False, "relu"), (True, "silu"), (False, "elu")])
def test_against_formula(shape, kind, gated, act):
    n, E, k, a, h, o = shape
    c = experts_case(n + a, n, E, k, a, h, o, F32 if kind == "f32" else BF16, gated=gated and h > 0, act=act, eight=kind == "eight", masked=0.1 if n > 100 else 0.0)
    check_experts(c, run_experts(c))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n", [2, 5, 16, 31, 64, 100, 129, 500])
def test_few_and_more_places(kind, n):
    c = experts_case(n, n, 8, 2, 72, 136, 40, F32 if kind == "f32" else BF16, biased=False, act="none")
    check_experts(c, run_experts(c))


@pytest.mark.parametrize("n", [4, 900])
@pytest.mark.parametrize("h", [0, 96])
def test_places_without_an_expert(n, h):
    c = experts_case(n, n, 6, 3, 64, h, 64, BF16, masked=0.5)
    c["ids"][0] = -1
    c["ids"][1] = torch.tensor([6, -2147483648, 2147483647], dtype=torch.int32)   # outside the experts: none
    c["weights"][1] = float("nan")
    got = run_experts(c)
    assert (got[:2] == 0).all()
    c["weights"][1] = 0
    c["ids"][1] = -1
    check_experts(c, got)
    c["ids"][:] = -1
    assert (run_experts(c) == 0).all()


@pytest.mark.parametrize("n", [3, 700])
def test_an_expert_named_twice(n):
    c = experts_case(n, n, 3, 4, 64, 64, 64, BF16, repeat=True)
    check_experts(c, run_experts(c))


@pytest.mark.parametrize("skew", [0.9, 1.0])
def test_one_expert_takes_nearly_all(skew):
    c = experts_case(11, 3000, 32, 2, 64, 128, 64, BF16, skew=skew)
    check_experts(c, run_experts(c))


@pytest.mark.parametrize("kind", ["f32", "bf16", "eight"])
def test_many_vertices(kind):
    c = experts_case(12, 60_001, 16, 2, 128, 256, 128, F32 if kind == "f32" else BF16, eight=kind == "eight")
    check_experts(c, run_experts(c), device="cuda")


@pytest.mark.parametrize("kind,a,h,o,k,gated", [("bf16", 320, 384, 320, 2, False), ("bf16", 272, 136, 264, 3, True), ("bf16", 64, 0, 96, 1, False), ("bf16", 136, 0, 520, 2, False),
                                                ("eight", 256, 0, 256, 1, False), ("eight", 528, 400, 48, 2, False), ("eight", 144, 272, 512, 1, True),
                                                ("f32", 40, 0, 72, 1, False), ("f32", 104, 200, 64, 2, True), ("f32", 64, 320, 136, 1, False), ("bf16", 768, 1024, 768, 2, True)])
@pytest.mark.parametrize("E,n", [(2, 4001), (5, 9000)])
def test_many_places_an_expert(kind, a, h, o, k, gated, E, n):
    """Rows of two tiles side by side: odd numbers of tiles, experts of few places, widths that leave a half of the columns empty."""
    c = experts_case(a + o + E, n, E, k, a, h, o, F32 if kind == "f32" else BF16, eight=kind == "eight", gated=gated, act="silu", masked=0.05, repeat=k > E, skew=0.7 if E == 5 else None)
    c["ids"][(c["ids"] == 3)] = 0   # an expert without a place
    check_experts(c, run_experts(c), device="cuda")


@pytest.mark.parametrize("E", [1, 300, 1500])
def test_numbers_of_experts(E):
    c = experts_case(13, 4000, E, 2, 32, 48, 32, BF16, repeat=True)
    check_experts(c, run_experts(c))


@pytest.mark.parametrize("n", [2, 800])
def test_a_bad_row_stays_in_its_vertex(n):
    c = experts_case(14, n, 4, 2, 64, 64, 64, BF16, act="silu")
    want = run_experts(c)
    c["x"][1, 3] = float("nan")
    got = run_experts(c)
    assert got[1].isnan().all()
    keep = [i for i in range(n) if i != 1]
    assert torch.equal(got[keep], want[keep])


@pytest.mark.parametrize("kind", ["f32", "bf16", "eight"])
@pytest.mark.parametrize("n", [2, 5000])
def test_results_are_the_same_every_time(kind, n):
    c = experts_case(15, n, 8, 3, 64, 128, 64, F32 if kind == "f32" else BF16, eight=kind == "eight")
    d = experts_desc(c)
    want = run_experts(c, desc=d)
    for _ in range(3):
        assert torch.equal(run_experts(c, desc=d), want)


@pytest.mark.parametrize("n", [3, 2000])
def test_captured_replays_take_new_inputs(n):
    c = experts_case(16, n, 8, 2, 64, 128, 64, BF16)
    other = experts_case(17, n, 8, 2, 64, 128, 64, BF16)
    d = experts_desc(c)
    x, ids, w = c["x"].cuda(), c["ids"].cuda(), c["weights"].cuda()
    out = torch.zeros(n, 64, dtype=BF16, device="cuda")
    ws = torch.empty(B.it_experts_workspace_bytes(d, n), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.it_experts_forward(d, x, ids, w, out, ws)
    for src in (c, other):
        x.copy_(src["x"]); ids.copy_(src["ids"]); w.copy_(src["weights"])
        graph.replay()
        B.it_experts_check(ws)
        assert torch.equal(out, run_experts({**c, "x": src["x"], "ids": src["ids"], "weights": src["weights"]}, desc=d))


def test_two_streams_with_a_workspace_each():
    cs = [experts_case(s, 3000, 8, 2, 64, 256, 64, BF16) for s in (18, 19)]
    want = [run_experts(c) for c in cs]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ds = [experts_desc(c) for c in cs]
    args = [[c["x"].cuda(), c["ids"].cuda(), c["weights"].cuda(), torch.zeros(3000, 64, dtype=BF16, device="cuda"),
             torch.empty(B.it_experts_workspace_bytes(d, 3000), dtype=torch.uint8, device="cuda")] for c, d in zip(cs, ds)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, d, a in zip(streams, ds, args):
            B.it_experts_forward(d, *a, stream=s)
    torch.cuda.synchronize()
    for a, w in zip(args, want):
        assert torch.equal(a[3], w)


def test_rows_and_bytes_behind_the_last_are_left():
    c = experts_case(20, 1000, 8, 2, 64, 128, 64, BF16)
    d = experts_desc(c)
    need = B.it_experts_workspace_bytes(d, 1000)
    ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    out = torch.full((1003, 64), 7.0, dtype=BF16, device="cuda")
    B.it_experts_forward(d, c["x"].cuda(), c["ids"].cuda(), c["weights"].cuda(), out[:1000], ws[:need])
    B.it_experts_check(ws)
    assert (out[1000:] == 7).all() and (ws[need:] == 0x5a).all()


def test_no_vertices():
    c = experts_case(21, 0, 4, 2, 64, 64, 64, BF16)
    assert run_experts(c).shape == (0, 64)


@pytest.mark.parametrize("kind", ["f32", "bf16", "eight"])
@pytest.mark.parametrize("h,k", [(128, 2), (0, 1)])
def test_waits_that_run_out_are_reported_and_over(kind, h, k):
    c = experts_case(22, 700, 4, k, 64, h, 64, F32 if kind == "f32" else BF16, eight=kind == "eight")
    d = experts_desc(c)
    dev = lambda t: None if t is None else t.cuda()   # noqa: E731
    out = torch.empty(700, 64, dtype=c["dtype"], device="cuda")
    ws = torch.empty(B.it_experts_workspace_bytes(d, 700), dtype=torch.uint8, device="cuda")
    B.it_debug_expire_wait_experts(d, dev(c["x"]), dev(c["ids"]), dev(c["weights"]), out, ws, x_scale=dev(c["x_scale"]))
    with pytest.raises(B.ItError, match="IT_ERR_TIMEOUT"):
        B.it_experts_check(ws)
    check_experts(c, run_experts(c, desc=d, workspace=ws))


def test_offsets_past_32_bits():
    """Typed vertices whose rows lie beyond 2^31 elements, in and out."""
    n, a, o = (1 << 31) // 128 + 1500, 128, 128
    c = experts_case(23, 1000, 2, 1, a, 0, o, BF16)
    x = torch.zeros(n, a, dtype=BF16, device="cuda")
    ids, w = torch.zeros(n, 1, dtype=torch.int32, device="cuda"), torch.ones(n, 1, device="cuda")
    x[-1000:], ids[-1000:], w[-1000:] = c["x"].cuda(), c["ids"].cuda(), c["weights"].cuda()
    d = experts_desc(c)
    out = torch.full((n, o), float("nan"), dtype=BF16, device="cuda")
    ws = torch.empty(B.it_experts_workspace_bytes(d, n), dtype=torch.uint8, device="cuda")
    B.it_experts_forward(d, x, ids, w, out, ws)
    B.it_experts_check(ws)
    check_experts(c, out[-1000:])
    first = run_experts({**c, "n": 8, "x": c["x"][:8] * 0, "ids": c["ids"][:8] * 0, "weights": c["weights"][:8] * 0 + 1}, desc=d)
    assert torch.equal(out[:8], first[:8])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_one_workspace_for_calls_in_turn(kind):
    """Different sizes and forms one after the other in the same scratch, large enough for each."""
    cs = [experts_case(30 + n, n, 4, 2, 64, 128, 64, F32 if kind == "f32" else BF16) for n in (3, 900, 40, 5000, 3)]
    ds = [experts_desc(c) for c in cs]
    ws = torch.full((max(B.it_experts_workspace_bytes(d, c["n"]) for c, d in zip(cs, ds)),), 0xff, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        for c, d in zip(cs, ds):
            check_experts(c, run_experts(c, desc=d, workspace=ws))


@pytest.mark.parametrize("kind,a,h,o,gated", [("bf16", 136, 200, 136, False), ("bf16", 200, 96, 192, True), ("bf16", 256, 512, 256, False), ("bf16", 248, 136, 72, True),
                                              ("bf16", 64, 1000, 256, True), ("bf16", 256, 64, 16, False), ("eight", 272, 208, 136, False), ("eight", 400, 144, 64, False),
                                              ("eight", 512, 272, 256, False), ("eight", 112, 528, 200, False)])
@pytest.mark.parametrize("n,k", [(700, 1), (2501, 2), (30_003, 2)])
def test_wide_rows_of_both_products_at_once(kind, a, h, o, gated, n, k):
    """Rows that fill several panels, results of more than 128 columns, widths that end inside a panel."""
    c = experts_case(a + h + o + n, n, 6, k, a, h, o, BF16, eight=kind == "eight", gated=gated, act="silu" if gated else "relu", masked=0.1)
    check_experts(c, run_experts(c), device="cuda")


@pytest.mark.parametrize("a,h,o,k,gated", [(256, 1024, 256, 2, False), (544, 0, 72, 1, False), (1024, 520, 136, 2, True), (512, 512, 128, 1, True), (520, 528, 64, 2, False),
                                           (8, 504, 8, 3, False), (2048, 0, 264, 1, False)])
@pytest.mark.parametrize("n", [500, 6001])
def test_long_sums_in_fp32(a, h, o, k, gated, n):
    """Sums of up to 512 terms and of more take accumulators of different kinds."""
    c = experts_case(a + h + o + n, n, 5, k, a, h, o, F32, gated=gated, act="elu", masked=0.1)
    check_experts(c, run_experts(c), device="cuda")


@pytest.mark.parametrize("kind,a,h,o,gated", [("f32", 576, 640, 64, True), ("bf16", 256, 192, 256, False), ("bf16", 320, 128, 320, False), ("eight", 512, 64, 136, False)])
def test_waits_that_run_out_in_wide_rows(kind, a, h, o, gated):
    c = experts_case(24, 40_000, 4, 2, a, h, o, F32 if kind == "f32" else BF16, eight=kind == "eight", gated=gated)
    d = experts_desc(c)
    dev = lambda t: None if t is None else t.cuda()   # noqa: E731
    out = torch.empty(40_000, o, dtype=c["dtype"], device="cuda")
    ws = torch.empty(B.it_experts_workspace_bytes(d, 40_000), dtype=torch.uint8, device="cuda")
    B.it_debug_expire_wait_experts(d, dev(c["x"]), dev(c["ids"]), dev(c["weights"]), out, ws, x_scale=dev(c["x_scale"]))
    with pytest.raises(B.ItError, match="IT_ERR_TIMEOUT"):
        B.it_experts_check(ws)
    check_experts(c, run_experts(c, desc=d, workspace=ws), device="cuda")


@pytest.mark.parametrize("kind,a,h,o,gated", [("bf16", 64, 128, 64, False), ("bf16", 128, 72, 40, True), ("eight", 64, 64, 200, False)])
@pytest.mark.parametrize("n,E,masked,repeat", [(60, 2, 0.0, False), (700, 4, 0.3, False), (700, 3, 0.0, True), (5000, 1, 0.2, True), (9001, 7, 0.5, True), (150_001, 8, 0.1, False)])
def test_two_places_a_vertex(kind, a, h, o, gated, n, E, masked, repeat):
    """The two rows of a vertex in the same tile, in tiles of the same time and of different times; one of them or both masked; the same result every time."""
    c = experts_case(n + a + h, n, E, 2, a, h, o, BF16, eight=kind == "eight", gated=gated, act="silu" if gated else "relu", masked=masked, repeat=repeat)
    d = experts_desc(c)
    want = run_experts(c, desc=d)
    check_experts(c, want, device="cuda")
    ws = torch.full((B.it_experts_workspace_bytes(d, n),), 0xff, dtype=torch.uint8, device="cuda")
    for _ in range(4):
        assert torch.equal(run_experts(c, desc=d, workspace=ws), want)


@pytest.mark.parametrize("n,E,k", [(1200, 8, 2), (3100, 32, 2), (3100, 33, 2), (700, 300, 3), (25_003, 20, 2), (25_800, 20, 2), (40_500, 256, 2), (41_100, 700, 2), (9000, 1024, 1),
                                   (16_384, 1025, 1), (16_385, 1025, 1), (3000, 4096, 2), (20_000, 1, 1)])
def test_sorting_of_places(n, E, k):
    """Sizes on either side of those where the places are sorted otherwise; experts without a place, one of most of them, masked places."""
    c = experts_case(n + E, n, E, k, 16, 0, 16, BF16, masked=0.2, repeat=True, skew=0.6 if n % 2 else None)
    c["ids"][c["ids"] % 5 == 3] = E - 1
    check_experts(c, run_experts(c), device="cuda")


@pytest.mark.parametrize("kind,gated", [("bf16", False), ("bf16", True), ("eight", False)])
@pytest.mark.parametrize("a,h,o", [(64, 2048, 64), (256, 1536, 256), (16, 1024, 8)])
def test_many_chunks_take_turns_in_two_buffers(kind, gated, a, h, o):
    """A chunk of the hidden row is written where the one before the last was read: long hidden rows, short products between them, the same result every time."""
    c = experts_case(a + h + o, 20_000, 4, 1, a, h, o, BF16, eight=kind == "eight", gated=gated, act="relu")
    d = experts_desc(c)
    ws = torch.full((B.it_experts_workspace_bytes(d, c["n"]),), 0xff, dtype=torch.uint8, device="cuda")
    want = run_experts(c, desc=d, workspace=ws)
    check_experts(c, want, device="cuda")
    for _ in range(4):
        assert torch.equal(run_experts(c, desc=d, workspace=ws), want)


@pytest.mark.parametrize("kind", ["bf16", "eight"])
@pytest.mark.parametrize("a,h", [(64, 16), (64, 80), (64, 128), (64, 208), (520, 80)])
@pytest.mark.parametrize("n", [20, 700])
def test_an_infinite_state_whose_hidden_row_is_finite(kind, a, h, n):
    """A state of plus infinity before negative weights: ReLU leaves a hidden row of zeros, and the result is the second bias, whatever fills up a tile of hidden columns."""
    a = a // 16 * 16
    c = experts_case(h + n, n, 3, 2, a, h, 64, BF16, act="relu", eight=kind == "eight")
    c["W1"] = (-(c["W1"].float().abs() + 2.0 ** -6).clamp_max(448)).to(c["W1"].dtype)
    if kind == "eight":   # (e4m3 has no infinity: the scale of a vertex has)
        c["x"][1] = torch.full((a,), 2.0).to(c["x"].dtype)
        c["x_scale"][1] = float("inf")
    else:
        c["x"][1] = float("inf")
    got = run_experts(c)
    assert torch.isfinite(got).all()
    want = (c["weights"][1][:, None].double() * c["b2"][c["ids"][1].long()].double()).sum(0)
    # (a rounding of the result, and two products and two sums in fp32, which may cancel)
    off = c["weights"][1].double() @ c["b2"][c["ids"][1].long()].double().abs()
    assert ((got[1].double().cpu() - want).abs() <= want.abs() * 2.0 ** -8 + off * 4 * 2.0 ** -24).all()
