"""The projection with low-rank adapters of many requests on the GPU, bit for bit against the plain definition."""
import numpy as np
import pytest
import torch

from oracle import layers as P

pytestmark = pytest.mark.gpu

NP = {torch.int8: np.int8, torch.uint8: np.uint8, torch.int32: np.int32}


@pytest.fixture(scope="module")
def G():
    import paper_2206_08869_b200 as g
    g.load_library()
    return g


def make_layer(rng, K, N, y_dtype, relu=False, s=None):
    clamp = {torch.int8: (-128, 127), torch.uint8: (0, 255), torch.int32: None}[y_dtype]
    s = np.full(N, max(1, int(np.log2(32 * np.sqrt(K))))) if s is None else s
    return {"k": 1, "c_in": K, "c_out": N, "w": rng.integers(-127, 128, (N, K)).astype(np.int8),
            "bias": rng.integers(-30000, 30000, N).astype(np.int32), "m0": rng.integers(2 ** 30, 2 ** 31, N).astype(np.int32),
            "s": s.astype(np.int32), "relu": relu or y_dtype == torch.uint8, "clamp": clamp}


def make_adapter(rng, K, N, R):
    return {"rank": R, "down": rng.integers(-127, 128, (R, K)).astype(np.int8),
            "m0": rng.integers(2 ** 30, 2 ** 31, R).astype(np.int32),
            "s": rng.integers(0, max(2, int(np.log2(64 * np.sqrt(K)))), R).astype(np.int32),
            "up": rng.integers(-127, 128, (N, R)).astype(np.int8)}


def make_x(rng, rows, K, dtype, ld=None):
    ld = ld or (K + 15) // 16 * 16
    lo, hi = (0, 256) if dtype == torch.uint8 else (-128, 128)
    buf = rng.integers(lo, hi, (rows, ld)).astype(NP[dtype])           # what lies behind a row is not zero
    return buf[:, :K], torch.from_numpy(buf).cuda()[:, :K]


def run(G, rng, rows, K, N, ranks, starts, which, x_dtype=torch.int8, y_dtype=torch.int8, max_rank=None, ldx=None, ldy=None,
        max_rows=None, **kw):
    layer = make_layer(rng, K, N, y_dtype, **kw)
    ads = [make_adapter(rng, K, N, R) if R else None for R in ranks]
    h = G.iodf_proj_create(layer, max_rows or rows, len(ads), max_rank or max([1] + list(ranks)), x_dtype=x_dtype, y_dtype=y_dtype)
    for i, ad in enumerate(ads):
        if ad:
            G.iodf_proj_set_adapter(h, i, ad)
    xh, x = make_x(rng, rows, K, x_dtype, ldx)
    ldy = ldy or N
    ybuf = torch.full((rows + 2, ldy), 77, dtype=y_dtype, device="cuda")
    y = ybuf[1:rows + 1, :N]
    st = torch.tensor(starts, dtype=torch.int32, device="cuda") if starts is not None else None
    wh = torch.tensor(which, dtype=torch.int32, device="cuda") if starts is not None else None
    G.iodf_proj_forward(h, x, st, wh, y=y)
    G.iodf_proj_check(h)
    want = P.projection(layer, xh, ads, starts, which, np.full((rows, N), 77))
    np.testing.assert_array_equal(y.cpu().numpy().astype(np.int64), want)
    full = ybuf.cpu().numpy()
    assert (full[0] == 77).all() and (full[-1] == 77).all() and (full[:, N:] == 77).all()      # nothing beside the rows
    return h, layer, ads


@pytest.mark.parametrize("x_dtype", [torch.int8, torch.uint8])
@pytest.mark.parametrize("y_dtype", [torch.int8, torch.uint8, torch.int32])
@pytest.mark.parametrize("rows,K,N", [(1, 1, 1), (1, 16, 8), (2, 173, 109), (7, 33, 257), (31, 128, 128), (65, 300, 130),
                                      (129, 64, 17), (200, 513, 255), (300, 96, 384)])
def test_plain_projection(G, rows, K, N, x_dtype, y_dtype):
    run(G, np.random.default_rng(rows * K + N), rows, K, N, [], None, None, x_dtype, y_dtype)


@pytest.mark.parametrize("x_dtype", [torch.int8, torch.uint8])
@pytest.mark.parametrize("rows,K,N,R", [(1, 64, 64, 16), (3, 173, 109, 13), (40, 256, 200, 32), (130, 96, 140, 64),
                                        (260, 512, 256, 128), (513, 160, 128, 1)])
def test_one_adapter_for_all_rows(G, rows, K, N, R, x_dtype):
    run(G, np.random.default_rng(rows + R), rows, K, N, [R, R], [0, rows], [1], x_dtype)


@pytest.mark.parametrize("rows", [1, 5, 16, 17, 33, 64, 100, 128, 200])
def test_a_request_per_row(G, rows):
    rng = np.random.default_rng(rows)
    which = rng.integers(-1, 9, rows)
    run(G, rng, rows, 208, 144, [16] * 9, list(range(rows + 1)), which.tolist())


@pytest.mark.parametrize("ranks", [[4, 16, 7, 1], [33, 2, 64, 0], [128, 1, 31, 32]])
def test_ragged_requests_of_mixed_ranks(G, ranks):
    """Empty requests, ones of one row, ones without adapter or with an empty slot, rows in front and behind."""
    rng = np.random.default_rng(sum(ranks))
    starts = [3, 3, 4, 60, 60, 200, 201, 459, 700]
    which = [0, 1, 2, 3, -1, 3, 0, 2]
    for y_dtype in (torch.int8, torch.int32):
        run(G, rng, 777, 173, 131, ranks, starts, which, torch.uint8, y_dtype, ldx=192, ldy=140)


def test_many_adapters_in_one_tile(G):
    """More adapters among neighbouring rows than fit next to each other on the chip."""
    rng = np.random.default_rng(8)
    rows, n = 600, 150
    which = (np.arange(rows) * 7 % n).tolist()
    run(G, rng, rows, 128, 128, [24] * n, list(range(rows + 1)), which)
    run(G, rng, rows, 128, 136, [128] * n, list(range(rows + 1)), which)


def test_alternating_adapters_and_none(G):
    rng = np.random.default_rng(9)
    starts = list(range(0, 514, 2))
    run(G, rng, 514, 64, 64, [16, 16], starts, [(-1, 0, 1, 0)[i % 4] for i in range(len(starts) - 1)])


def test_no_row_in_any_request(G):
    run(G, np.random.default_rng(1), 40, 64, 64, [8], [10, 10], [0])
    run(G, np.random.default_rng(1), 300, 64, 64, [8], [300, 300], [0])


def test_extreme_values_keep_every_bit(G):
    """All operands at their ends: the largest accumulators, both signs of the rounding, clips at both ends."""
    for x_dtype, xv in ((torch.int8, (-128, 127)), (torch.uint8, (0, 255))):
        K, N, R, rows = 1000, 64, 64, 70
        rng = np.random.default_rng(K)
        layer = {"k": 1, "c_in": K, "c_out": N, "w": rng.choice([-127, 127, -128], (N, K)).astype(np.int8),
                 "bias": rng.choice([-2 ** 30, 2 ** 30], N).astype(np.int32), "m0": rng.choice([2 ** 30, 2 ** 31 - 1], N).astype(np.int32),
                 "s": rng.choice([0, 31, 1, 18], N).astype(np.int32), "relu": False, "clamp": None}
        layer["w"][0], layer["w"][1] = 127, -128
        ad = make_adapter(rng, K, N, R)
        ad["down"][:] = rng.choice([-128, 127], (R, K))
        ad["up"][:] = rng.choice([-128, 127], (N, R))
        h = G.iodf_proj_create(layer, rows, 1, R, x_dtype=x_dtype)
        G.iodf_proj_set_adapter(h, 0, ad)
        xh, x = make_x(rng, rows, K, x_dtype)
        xh[:] = rng.choice(xv, xh.shape)
        xh[0], xh[1] = xv[0], xv[1]
        x.copy_(torch.from_numpy(np.ascontiguousarray(xh)))
        st = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
        y = G.iodf_proj_forward(h, x, st, torch.zeros(1, dtype=torch.int32, device="cuda"))
        np.testing.assert_array_equal(y.cpu().numpy(), P.projection(layer, xh, [ad], [0, rows], [0]))


@pytest.mark.parametrize("rows,K,N,R", [(1, 4096, 520, 16), (20, 2049, 300, 32), (700, 1500, 640, 48), (3000, 256, 256, 8)])
def test_larger_sizes(G, rows, K, N, R):
    rng = np.random.default_rng(rows)
    cut = sorted(rng.integers(0, rows + 1, 5).tolist())
    run(G, rng, rows, K, N, [R] * 3, [0] + cut + [rows], [0, 1, 2, -1, 1, 0])


@pytest.mark.parametrize("rows,K,N,R", [(3000, 1300, 300, 0), (3000, 1300, 900, 33), (2500, 2050, 260, 128), (4099, 1025, 128, 40),
                                        (2111, 700, 384, 100), (9000, 1100, 130, 16)])
def test_many_rows_of_many_channels(G, rows, K, N, R):
    """Sizes whose x tile does not stay in shared memory; odd numbers of output tiles, rows that end inside a tile."""
    rng = np.random.default_rng(rows + K)
    cut = sorted(rng.integers(5, rows - 7, 11).tolist())
    cut[4] = cut[3]
    which = [0, 1, 2, -1, 1, 0, 4, 3, 2, 2, 3, 4]
    for x_dtype, y_dtype in ((torch.int8, torch.int8), (torch.uint8, torch.int32)):
        if R:
            run(G, rng, rows, K, N, [R, 1, R // 2 + 1, 0, R], [5] + cut + [rows - 7], which, x_dtype, y_dtype)
        else:
            run(G, rng, rows, K, N, [], None, None, x_dtype, y_dtype)


def test_many_requests_of_many_channels(G):
    rng = np.random.default_rng(61)
    rows, n = 1100, 70
    starts = list(range(0, rows + 1, 4))
    run(G, rng, rows, 1200, 300, [64] * n, starts, [(i * 11) % n - 1 for i in range(len(starts) - 1)])


def test_adapters_are_replaced_and_emptied(G):
    rng = np.random.default_rng(4)
    h, layer, ads = run(G, rng, 50, 80, 72, [8, 16], [0, 20, 50], [0, 1], max_rows=64)
    xh, x = make_x(rng, 50, 80, torch.int8)
    st = torch.tensor([0, 20, 50], dtype=torch.int32, device="cuda")
    wh = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    ads = [None, make_adapter(rng, 80, 72, 3)]
    G.iodf_proj_set_adapter(h, 0, None)
    G.iodf_proj_set_adapter(h, 1, ads[1])
    y = G.iodf_proj_forward(h, x, st, wh)
    np.testing.assert_array_equal(y.cpu().numpy(), P.projection(layer, xh, ads, [0, 20, 50], [0, 1]))


def test_fewer_rows_than_the_handle_holds_and_none(G):
    rng = np.random.default_rng(6)
    h, layer, ads = run(G, rng, 100, 64, 48, [8], [0, 90], [0], max_rows=100)
    for rows in (99, 1, 17):
        xh, x = make_x(rng, rows, 64, torch.int8)
        y = G.iodf_proj_forward(h, x)
        np.testing.assert_array_equal(y.cpu().numpy(), P.projection(layer, xh))
    assert G.iodf_proj_forward(h, x[:0]).shape == (0, 48)


def test_bad_requests_are_reported_and_touch_nothing_else(G):
    rng = np.random.default_rng(12)
    rows, K, N = 200, 64, 48
    layer = make_layer(rng, K, N, torch.int8)
    ad = make_adapter(rng, K, N, 8)
    h = G.iodf_proj_create(layer, rows, 2, 8, y_dtype=torch.int8)
    G.iodf_proj_set_adapter(h, 0, ad)
    xh, x = make_x(rng, rows, K, torch.int8)
    for rows_used in (200, 20):
        ybuf = torch.full((rows + 2, N), 55, dtype=torch.int8, device="cuda")
        for starts, which, bad in (([0, 10, 20], [2, -2], 2), ([0, 50, 20], [0, 0], None), ([-7, 10, 9999], [0, 0], 2),
                                   ([2 ** 31 - 1, -2 ** 31, 5], [2 ** 31 - 1, -2 ** 31], 2)):
            st = torch.tensor(starts, dtype=torch.int64).to(torch.int32).cuda()
            wh = torch.tensor(which, dtype=torch.int64).to(torch.int32).cuda()
            G.iodf_proj_forward(h, x[:rows_used], st, wh, y=ybuf[1:rows_used + 1])
            with pytest.raises(G.IodfError) as e:
                G.iodf_proj_check(h)
            assert e.value.status == -9
            if bad:
                assert "(%d requests)" % bad in str(e.value)
        assert (ybuf[0] == 55).all() and (ybuf[rows_used + 1:] == 55).all()
    # a slot outside the handle counts as none, and the handle works on
    st, wh = torch.tensor([0, 200], dtype=torch.int32, device="cuda"), torch.tensor([5], dtype=torch.int32, device="cuda")
    y = G.iodf_proj_forward(h, x, st, wh)
    with pytest.raises(G.IodfError):
        G.iodf_proj_check(h)
    np.testing.assert_array_equal(y.cpu().numpy(), P.projection(layer, xh))
    G.iodf_proj_check(h)


def test_refusals(G):
    rng = np.random.default_rng(2)
    layer = make_layer(rng, 20, 12, torch.int8)
    h = G.iodf_proj_create(layer, 8, 1, 4, y_dtype=torch.int8)
    _, x = make_x(rng, 8, 20, torch.int8)

    def status(f, *a, **k):
        with pytest.raises(G.IodfError) as e:
            f(*a, **k)
        return e.value.status

    ad = make_adapter(rng, 20, 12, 4)
    assert status(G.iodf_proj_set_adapter, h, 1, ad) == -1                        # no such slot
    assert status(G.iodf_proj_set_adapter, h, 0, make_adapter(rng, 20, 12, 5)) == -1   # rank above the handle's
    assert status(G.iodf_proj_set_adapter, h, 0, dict(ad, m0=ad["m0"] // 4)) == -1
    assert status(G.iodf_proj_set_adapter, h, 0, dict(ad, s=ad["s"] * 0 + 32)) == -1
    over = G.iodf_proj_create(dict(layer, w=layer["w"] * 0, bias=np.full(12, 2 ** 31 - 1 - 100, np.int32)), 8, 1, 4, y_dtype=torch.int8)
    assert status(G.iodf_proj_set_adapter, over, 0, dict(ad, up=np.full((12, 4), 1, np.int8))) == -7
    big = torch.zeros((9, 32), dtype=torch.int8, device="cuda")[:, :20]
    assert status(G.iodf_proj_forward, h, big) == -1                              # more rows than the handle holds
    assert status(G.iodf_proj_forward, h, torch.zeros((8, 20), dtype=torch.int8, device="cuda")) == -1   # row stride 20
    odd = torch.zeros(8 * 32 + 16, dtype=torch.int8, device="cuda")
    assert status(G.iodf_proj_forward, h, odd[8:8 + 256].view(8, 32)[:, :20]) == -1                      # base not aligned
    with pytest.raises(ValueError):
        G.iodf_proj_forward(h, x.to(torch.uint8))
    with pytest.raises(ValueError):
        G.iodf_proj_forward(h, x[:, :19])
    with pytest.raises(ValueError):
        G.iodf_proj_forward(h, x.cpu())
    with pytest.raises(ValueError):
        G.iodf_proj_forward(h, x, y=torch.zeros((8, 12), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        G.iodf_proj_forward(h, x, torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("rows", [5, 48, 400])
def test_captured_replayed_and_on_another_stream(G, rows):
    rng = np.random.default_rng(rows)
    K, N = 160, 96
    layer = make_layer(rng, K, N, torch.int8)
    ads = [make_adapter(rng, K, N, 12) for _ in range(3)]
    h = G.iodf_proj_create(layer, rows, 3, 16, y_dtype=torch.int8)
    for i, ad in enumerate(ads):
        G.iodf_proj_set_adapter(h, i, ad)
    xh, x = make_x(rng, rows, K, torch.int8)
    st = torch.tensor([0, rows // 2, rows], dtype=torch.int32, device="cuda")
    wh = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    y = torch.zeros((rows, N), dtype=torch.int8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    G.iodf_proj_forward(h, x, st, wh, y=y, stream=side)
    side.synchronize()
    np.testing.assert_array_equal(y.cpu().numpy(), P.projection(layer, xh, ads, [0, rows // 2, rows], [0, 1]))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        G.iodf_proj_forward(h, x, st, wh, y=y)
        with pytest.raises(G.IodfError):
            G.iodf_proj_set_adapter(h, 0, ads[0])
    for cut, w in ((rows, [2, 0]), (0, [0, 2]), (rows // 3, [-1, 1])):        # what the graph reads changes between replays
        xh2, x2 = make_x(rng, rows, K, torch.int8)
        x.copy_(x2)
        st.copy_(torch.tensor([0, cut, rows], dtype=torch.int32))
        wh.copy_(torch.tensor(w, dtype=torch.int32))
        g.replay()
        g.replay()
        np.testing.assert_array_equal(y.cpu().numpy(), P.projection(layer, xh2, ads, [0, cut, rows], w))
    G.iodf_proj_check(h)


def test_two_handles_at_once(G):
    rng = np.random.default_rng(77)
    lanes = []
    for i in range(3):
        rows, K, N = 300 + 41 * i, 128, 96
        layer, ad = make_layer(rng, K, N, torch.int32), make_adapter(rng, K, N, 16)
        h = G.iodf_proj_create(layer, rows, 1, 16)
        G.iodf_proj_set_adapter(h, 0, ad)
        xh, x = make_x(rng, rows, K, torch.int8)
        lanes.append((h, layer, ad, xh, x, torch.tensor([0, rows], dtype=torch.int32, device="cuda"),
                      torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty((rows, N), dtype=torch.int32, device="cuda"),
                      torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for h, _, _, _, x, st, wh, y, stream in lanes:
            G.iodf_proj_forward(h, x, st, wh, y=y, stream=stream)
    torch.cuda.synchronize()
    for h, layer, ad, xh, x, st, wh, y, _ in lanes:
        np.testing.assert_array_equal(y.cpu().numpy(), P.projection(layer, xh, [ad], [0, len(xh)], [0]))


@pytest.mark.parametrize("rows,K,N", [(5000, 160, 200), (20000, 40, 50), (3000, 1300, 400)])
def test_many_rows_captured_and_replayed(G, rows, K, N):
    rng = np.random.default_rng(rows)
    layer = make_layer(rng, K, N, torch.int8)
    ads = [make_adapter(rng, K, N, 30) for _ in range(3)]
    h = G.iodf_proj_create(layer, rows, 3, 30, y_dtype=torch.int8)
    for i, ad in enumerate(ads):
        G.iodf_proj_set_adapter(h, i, ad)
    xh, x = make_x(rng, rows, K, torch.int8)
    st = torch.tensor([0, rows // 2, rows], dtype=torch.int32, device="cuda")
    wh = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    y = torch.zeros((rows, N), dtype=torch.int8, device="cuda")
    G.iodf_proj_forward(h, x, st, wh, y=y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        G.iodf_proj_forward(h, x, st, wh, y=y)
        G.iodf_proj_forward(h, x, st, wh, y=y)
    for cut, w in ((rows, [2, 0]), (0, [0, 2]), (rows // 3, [-1, 1])):
        xh2, x2 = make_x(rng, rows, K, torch.int8)
        x.copy_(x2)
        st.copy_(torch.tensor([0, cut, rows], dtype=torch.int32))
        wh.copy_(torch.tensor(w, dtype=torch.int32))
        g.replay()
        g.replay()
        np.testing.assert_array_equal(y.cpu().numpy(), P.projection(layer, xh2, ads, [0, cut, rows], w))
    G.iodf_proj_check(h)


@pytest.mark.parametrize("rows,K,N,R", [(3001, 70, 60, 20), (5003, 33, 140, 16), (2600, 1400, 140, 64)])
def test_more_requests_than_are_read_at_once(G, rows, K, N, R):
    rng = np.random.default_rng(rows)
    which = (np.arange(rows) * 13 % 9 - 1).tolist()
    run(G, rng, rows, K, N, [R] * 8, list(range(rows + 1)), which)
    empty = sorted(rng.integers(0, rows + 1, 2500).tolist())
    run(G, rng, rows, K, N, [R] * 8, [0] + empty + [rows], [i % 9 - 1 for i in range(2501)])


def test_requests_as_short_as_the_deepest_levels_images(G):
    """Sixteen rows each: sixteen adapters among the rows of a tile, in every one of its output tiles."""
    rng = np.random.default_rng(44)
    n = 500
    run(G, rng, 16 * n, 64, 300, [8] * 40, list(range(0, 16 * n + 1, 16)), (rng.integers(0, 40, n)).tolist(), torch.uint8, torch.uint8)


@pytest.mark.parametrize("rows,K,N", [(700, 96, 72), (9000, 96, 72), (2500, 1100, 260)])
def test_calls_of_one_handle_in_a_row_with_other_rows(G, rows, K, N):
    """The workspace of one call is the next one's: nothing of it may be taken for the next one's."""
    rng = np.random.default_rng(rows)
    layer = make_layer(rng, K, N, torch.int8)
    ads = [make_adapter(rng, K, N, 17) for _ in range(4)]
    h = G.iodf_proj_create(layer, rows, 4, 17, y_dtype=torch.int8)
    for i, ad in enumerate(ads):
        G.iodf_proj_set_adapter(h, i, ad)
    todo = []
    for i in range(6):
        m = max(1, rows // (i + 1) - i)
        xh, x = make_x(rng, m, K, torch.int8)
        st = [0, m // 3, m // 3, m - i // 2]
        w = [(i + j) % 5 - 1 for j in range(3)]
        todo.append((xh, x, st, w, torch.tensor(st, dtype=torch.int32, device="cuda"), torch.tensor(w, dtype=torch.int32, device="cuda")))
    torch.cuda.synchronize()
    ys = [G.iodf_proj_forward(h, x, st_d, w_d) for _, x, _, _, st_d, w_d in todo]
    G.iodf_proj_check(h)
    for (xh, _, st, w, _, _), y in zip(todo, ys):
        np.testing.assert_array_equal(y.cpu().numpy(), P.projection(layer, xh, ads, st, w, np.zeros((len(xh), N))))


def test_narrow_clips(G):
    rng = np.random.default_rng(3)
    for rows, K, N in ((9, 64, 40), (700, 200, 150), (3000, 1200, 150)):
        for y_dtype, clamp, relu in ((torch.int8, (-7, 5), False), (torch.uint8, (3, 200), True), (torch.int32, (-1000, 900), False),
                                     (torch.int32, (-5, -2), True)):
            layer = dict(make_layer(rng, K, N, y_dtype), clamp=clamp, relu=relu, s=np.full(N, 4, np.int32))
            h = G.iodf_proj_create(layer, rows, y_dtype=y_dtype)
            xh, x = make_x(rng, rows, K, torch.int8)
            np.testing.assert_array_equal(G.iodf_proj_forward(h, x).cpu().numpy(), P.projection(layer, xh))


@pytest.mark.parametrize("ldy_pad,skip", [(0, 0), (1, 0), (4, 4), (3, 1), (16, 2)])
@pytest.mark.parametrize("rows,K,N", [(20, 64, 132), (900, 64, 132), (3000, 1100, 260)])
def test_outputs_at_any_alignment(G, rows, K, N, ldy_pad, skip):
    rng = np.random.default_rng(rows + ldy_pad)
    for y_dtype in (torch.int8, torch.int32):
        layer = make_layer(rng, K, N, y_dtype)
        h = G.iodf_proj_create(layer, rows, y_dtype=y_dtype)
        xh, x = make_x(rng, rows, K, torch.int8)
        buf = torch.full((skip + rows * (N + ldy_pad) + 5,), 9, dtype=y_dtype, device="cuda")
        y = buf[skip:skip + rows * (N + ldy_pad)].view(rows, N + ldy_pad)
        G.iodf_proj_forward(h, x, y=y[:, :N])
        np.testing.assert_array_equal(y[:, :N].cpu().numpy(), P.projection(layer, xh))
        assert (y[:, N:] == 9).all() and (buf[:skip] == 9).all() and (buf[-5:] == 9).all()


@pytest.mark.parametrize("x_dtype", [torch.int8, torch.uint8])
@pytest.mark.parametrize("rows,K,N,R", [(1, 1024, 300, 16), (1, 4096, 130, 32), (1, 1000, 4100, 100), (2, 500, 64, 64), (3, 17, 9, 5),
                                        (4, 1024, 260, 31), (4, 1025, 260, 31), (5, 64, 64, 8), (1, 130, 20000, 8)])
def test_one_to_five_rows(G, rows, K, N, R, x_dtype):
    rng = np.random.default_rng(rows + K)
    for starts, which in (([0, rows], [1]), ([0, rows], [-1]), (list(range(rows + 1)), [(i * 3 + 2) % 5 - 1 for i in range(rows)]),
                          ([0, 0, 1, 1], [0, 2, 1]), ([rows, rows], [0])):
        run(G, rng, rows, K, N, [R, 1, R // 2 + 1, R], starts, which, x_dtype)
    many = sorted(rng.integers(0, rows + 1, 3000).tolist())
    run(G, rng, rows, K, N, [R, 1, R // 2 + 1, R], [0] + many + [rows], [i % 5 - 1 for i in range(3001)], x_dtype)
    some = sorted(rng.integers(0, rows + 1, 300).tolist())
    run(G, rng, rows, K, N, [R, 1, R // 2 + 1, R], [0] + some + [rows], [i % 5 - 1 for i in range(301)], x_dtype)


@pytest.mark.parametrize("rows,K,N", [(33, 250, 60), (97, 1030, 300), (130, 1024, 520), (130, 2100, 130), (257, 173, 300), (257, 1030, 60),
                                      (512, 2100, 260), (700, 1024, 300), (1030, 1152, 130)])
def test_a_few_hundred_rows(G, rows, K, N):
    """Around the sizes where the kernel for few rows gives way, with one adapter, a few, one per row and none."""
    rng = np.random.default_rng(rows * K)
    for R in (16, 70):
        ranks = [R, 1, R // 2 + 1, R, R, R - 1, 3]
        for starts, which in ((None, None), ([0, rows], [0]), ([0, rows // 3, rows // 3, rows - 1], [3, 4, -1]),
                              (list(range(rows + 1)), [(i * 5 + 3) % 8 - 1 for i in range(rows)])):
            run(G, rng, rows, K, N, ranks, starts, which, torch.uint8 if rows % 2 else torch.int8)
