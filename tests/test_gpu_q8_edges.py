"""The operators beside the layer where numbers are at the edge of their types and tensors at the edge of others, and the forms of the
products by name."""
import numpy as np
import pytest
import torch

import oracle.ops as ops
from ops_tolerance import U, route_weights
from paper_2510_26730_amd import binding as ef
from test_gpu_ops import TYPES, check_product, check_quant, f64, near, product_tolerance, run_route, stream, weights

pytestmark = pytest.mark.gpu


# ---- routing ------------------------------------------------------------------------------------

def check_weights(z, bias, k, dtype=torch.float32, **kw):
    got, zd = run_route(z, bias, k, dtype, **kw)
    want = ops.route_scores(zd, None if bias is None else f64(bias), k, **kw)
    assert np.array_equal(got["ids"], want["ids"].reshape(-1))
    tol = route_weights(zd, want["ids"], want["w"], kw.get("sigmoid", False))
    near(torch.from_numpy(got["w"]).view(-1, k), want["w"], tol, f"weights {tuple(z.shape)} k={k} {kw}")


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("groups", [dict(), dict(n_groups=4, groups_kept=2, group_best=2)])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("low", [-60, -86, -90, -120, -200, -600])
def test_weights_of_very_low_sigmoid_scores(low, with_bias, groups, renorm):
    """Scores that 32 bits cannot hold still have the right quotients; rows whose chosen ones straddle the border of 32 bits."""
    gen = torch.Generator().manual_seed(-low)
    z = low + 4 * torch.rand(60, 64, generator=gen)
    z[:20] = low + 4 * torch.randint(0, 200, (20, 64), generator=gen).float() / 100
    z[20:40, 5] = torch.linspace(low, 3, 20)
    bias = torch.linspace(0, 1, 64)[torch.randperm(64, generator=gen)] if with_bias else None
    check_weights(z, bias, 4, sigmoid=True, renorm=renorm, scale=2.5, **groups)


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("depth", [20, 90, 105, 130, 600])
def test_weights_of_experts_far_below_the_top(depth, best, renorm):
    """A softmax whose bias chooses experts `depth` below the largest logit."""
    gen = torch.Generator().manual_seed(depth)
    z = 3 * torch.rand(50, 32, generator=gen)
    z[:, 8:24] -= depth
    bias = torch.zeros(32)
    bias[8:24] = 3 + torch.linspace(0, 1, 16)[torch.randperm(16, generator=gen)]
    check_weights(z, bias, 4, renorm=renorm)
    check_weights(z, bias, 4, renorm=renorm, n_groups=4, groups_kept=2, group_best=best)


def test_chosen_scores_that_are_all_0():
    """Behind a logit of +inf a softmax leaves nothing for the others, whatever the bias chooses."""
    z = torch.randn(8, 16, generator=torch.Generator().manual_seed(2))
    z[:, 3] = float("inf")
    bias = torch.linspace(2, 3, 16)
    bias[3] = 0
    check_weights(z, bias, 4, renorm=True)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("groups", [dict(), dict(n_groups=4, groups_kept=2, group_best=2), dict(n_groups=4, groups_kept=2)])
def test_weights_beside_masked_logits(sigmoid, dtype, with_bias, groups):
    """-inf, NaN, +inf and the type's lowest value in some rows say nothing about how far the weights of others may be off."""
    gen = torch.Generator().manual_seed(11)
    z = torch.randn(60, 48, generator=gen)
    inf, nan, low = float("inf"), float("nan"), torch.finfo(TYPES[dtype]).min
    z[0], z[1], z[2] = -inf, nan, low
    z[3, ::2], z[4, :46], z[5, 7], z[6, 3:9] = nan, -inf, inf, inf
    z[7, ::3] = low
    z[8, 1:] = low
    z[10:30][torch.rand(20, 48, generator=gen) < 0.9] = -inf
    z[30:40][torch.rand(10, 48, generator=gen) < 0.9] = low
    bias = 0.3 * torch.randn(48, generator=gen) if with_bias else None
    check_weights(z, bias, 4, TYPES[dtype], sigmoid=sigmoid, renorm=True, **groups)


def test_sums_of_two_best_beyond_32_bits():
    z = torch.randn(40, 16, generator=torch.Generator().manual_seed(9))
    bias = torch.tensor([3.0e38, 3.0e38, 0, 0, 3.1e38, 3.1e38, 0, 0, 3.3e38, 2.7e38, 0, 0, 3.2e38, 3.2e38, 0, 0])
    for kept in (1, 2, 3):
        check_weights(z, bias, 2, sigmoid=True, n_groups=4, groups_kept=kept, group_best=2)
        check_weights(z, -bias, 2, n_groups=4, groups_kept=kept, group_best=2)
        check_weights(z[:, :8], bias[[0, 1, 4, 5, 8, 9, 12, 13]], 2, sigmoid=True, n_groups=4, groups_kept=kept, group_best=2)
        check_weights(z[:, :8], -bias[[0, 1, 4, 5, 8, 9, 12, 13]], 2, sigmoid=True, n_groups=4, groups_kept=kept, group_best=2)
        check_weights(z[:, :8], -bias[[12, 13, 4, 5, 8, 9, 0, 1]], 2, n_groups=4, groups_kept=kept, group_best=2)


# ---- rows to 8 bits ------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,first,last,pitch", [(4, 100, 100, 200, 200), (7, 100, 0, 110, 200), (1, 65, 16, 90, 90), (5, 96, 16, 112, 128),
                                                     (1200, 96, 32, 144, 144), (3, 1000, 16, 1020, 1040), (6, 64, 16, 80, 80), (9, 2056, 0, 2100, 2112)])
def test_codes_in_columns_of_a_wider_matrix(rows, K, first, last, pitch, dtype):
    """Codes and zeros go into the columns given, and nowhere else: not into the next row, not behind the last."""
    gen = torch.Generator().manual_seed(rows + K)
    x = torch.randn(rows, K, generator=gen).to(TYPES[dtype])
    room = torch.full((rows * pitch + 512,), 99, dtype=torch.int8, device="cuda")
    wide = room[:rows * pitch].view(rows, pitch)
    scales = torch.empty(rows, device="cuda")
    ef.ef_quant_rows(x.cuda(), wide[:, first:last], scales, stream=stream())
    torch.cuda.synchronize()
    q, s = ops.quant_rows(f64(x))
    padded = min((K + 63) // 64 * 64, last - first)
    assert np.array_equal(wide[:, first:first + K].cpu().numpy(), q) and np.array_equal(f64(scales), s)
    assert (wide[:, first + K:first + padded] == 0).all()
    assert (wide[:, :first] == 99).all() and (wide[:, first + padded:] == 99).all() and (room[rows * pitch:] == 99).all()


def test_quant_rows_at_halves_of_the_smallest_scales():
    """Scales between 2^-126 and 2^-125, whose halves are no 32-bit numbers: the values on both sides of them."""
    rng = np.random.default_rng(4)
    most = (127 * 2.0 ** -126 * (1 + rng.random(400))).astype(np.float32)
    scale = np.maximum((most.astype(np.float64) / 127).astype(np.float32), np.float32(2.0 ** -126)).astype(np.float64)
    x = np.zeros((400, 64), np.float32)
    x[:, 0] = most
    for c in range(1, 64):
        half = (c // 4 + 0.5) * scale * (1 if c % 2 else -1)
        x[:, c] = half.astype(np.float32)
        x[:, c] = np.nextafter(x[:, c], np.float32(np.inf if c % 4 < 2 else -np.inf))
    check_quant(torch.from_numpy(x))
    check_quant(torch.from_numpy(x[:, :63].copy()))


def test_more_rows_than_a_launch_has_workgroups():
    """2^24 workgroups of 256 lanes are more than one launch takes."""
    n, K = (1 << 24) + 3, 3
    base = torch.randn(1000, K, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    at = torch.arange(n, device="cuda") % 1000
    x, codes, scales = base[at], torch.full((n, K), 99, dtype=torch.int8, device="cuda"), torch.full((n,), -1.0, device="cuda")
    ef.ef_quant_rows(x, codes, scales, stream=stream())
    q, s = ops.quant_rows(f64(base))
    q, s = torch.from_numpy(q).to(torch.int8).cuda(), torch.from_numpy(s).float().cuda()
    assert torch.equal(codes, q[at]) and torch.equal(scales, s[at])
    w, ws = weights(torch.Generator().manual_seed(2), 1, 5, K)
    rows = torch.tensor([0, n - 1, n, 1 << 24, 1234567], dtype=torch.int32, device="cuda")
    want = ops.matmul_q8(q[at[rows.long().clamp(max=n - 1)]].cpu().numpy(), f64(s[at[rows.long().clamp(max=n - 1)]]), w.cpu().numpy(), f64(ws))
    want[2] = np.nan
    for a, kw in ((x, {}), (codes, dict(a_scale=scales))):
        out = torch.empty(5, 5, device="cuda")
        work = torch.empty(ef.ef_matmul_q8_work(a, w[0], ws, out, rows=rows, **kw), dtype=torch.uint8, device="cuda")
        ef.ef_matmul_q8(a, w[0], ws, out, work, rows=rows, stream=stream(), **kw)
        near(out, want, product_tolerance(want, torch.float32), f"a row of {n}")


# ---- products ------------------------------------------------------------------------------------

# every form: rows, K, N (swiglu: twice the columns), rows of each group
SHAPES = [(2, 512, 256, None), (12, 512, 256, None), (30, 320, 512, None), (200, 192, 2048, None), (100, 1300, 8300, None), (520, 192, 2300, None),
          (520, 1152, 14000, None), (0, 1088, 1408, [30, 0, 1, 64, 65, 7] * 9), (0, 320, 512, [90, 0, 129, 33])]
IDS = [f"{s[0]}-{s[1]}-{s[2]}" for s in SHAPES]


@pytest.mark.parametrize("M,K,N,counts", SHAPES, ids=IDS)
def test_swiglu_of_gates_whose_exponential_passes_32_bits(M, K, N, counts):
    """silu(g) is a 32-bit number down to g = -91, and its product with a large u farther down.  Gates from -102 to -60 and from 60 to 102."""
    gen = torch.Generator().manual_seed(M + N)
    M, G = sum(counts) if counts else M, len(counts) if counts else 1
    x = torch.linspace(0.6, 1.02, M)[torch.randperm(M, generator=gen)][:, None].expand(M, K).contiguous()
    w, ws = weights(gen, G, N, K)
    F = N // 2
    w[:, :F], w[:, F:] = -100, 90
    w[:, 1:F:5] = 100
    ws[:, :F] = 1 / K
    ws[:, F:] = torch.logspace(8, 12, F, device="cuda") / K
    off = None if counts is None else np.concatenate([[0], np.cumsum(counts)])
    out = torch.empty(M, F, device="cuda")
    a, xc, kw = w if counts else w[0], x.cuda(), dict(swiglu=True, offsets=None if off is None else torch.tensor(off, dtype=torch.int32, device="cuda"))
    work = torch.empty(ef.ef_matmul_q8_work(xc, a, ws, out, **kw), dtype=torch.uint8, device="cuda")
    ef.ef_matmul_q8(xc, a, ws, out, work, stream=stream(), **kw)
    q, s = ops.quant_rows(f64(x))
    y = ops.matmul_q8(q, s, w.cpu().numpy(), f64(ws), offsets=off)
    want = ops.matmul_q8(q, s, w.cpu().numpy(), f64(ws), offsets=off, swiglu=True)
    # three roundings in front of each factor, which silu multiplies by up to 1 + |g|; the exponential's argument and itself; subnormal results
    tol = np.abs(want) * (8 * np.abs(y[:, :F]) + 24) * U + 2.0 ** -126
    near(out, want, tol, f"swiglu M={M} N={N} K={K} G={G}")
    assert (np.abs(want) > 1e-34).all()


@pytest.mark.parametrize("swiglu", [False, True])
@pytest.mark.parametrize("M,K,N,counts", SHAPES, ids=IDS)
def test_products_whose_sum_and_scale_pass_32_bits(M, K, N, counts, swiglu):
    """Rows near the type's largest value beside ordinary ones: a sum times the row's scale is beyond 32 bits, their result is not."""
    gen = torch.Generator().manual_seed(K + N)
    M = sum(counts) if counts else M
    x = torch.rand(M, K, generator=gen)
    x[::3] *= 1e38
    check_product(gen, x, len(counts) if counts else 1, N, counts, swiglu=swiglu, out="f32", magnitude=1e-37 if swiglu else 1e-6)


@pytest.mark.parametrize("M,K,N,counts", SHAPES, ids=IDS)
def test_large_scales_of_sums_that_are_0(M, K, N, counts):
    """0 times two scales whose product is beyond 32 bits is 0, a sum of more is infinite, and neither touches the rows beside."""
    gen = torch.Generator().manual_seed(K)
    M = sum(counts) if counts else M
    G = len(counts) if counts else 1
    x = torch.rand(M, K, generator=gen) + 0.5
    x[::2] *= 2.0 ** 110
    w, ws = weights(gen, G, N, K)
    w[:, ::2] = 0
    w[:, 1::2] = 1
    w[:, 1::4] = -1
    ws[:] = 2.0 ** 110
    off = None if counts is None else torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    out = torch.empty(M, N, device="cuda")
    a, xc = w if counts else w[0], x.cuda()
    work = torch.empty(ef.ef_matmul_q8_work(xc, a, ws, out, offsets=off), dtype=torch.uint8, device="cuda")
    ef.ef_matmul_q8(xc, a, ws, out, work, offsets=off, stream=stream())
    assert (out[:, ::2] == 0).all()
    assert (out[::2, 1::4] == -float("inf")).all() and (out[::2, 3::4] == float("inf")).all()
    assert out[1::2, 1::2].isfinite().all() and (out[1::2, 1::2] != 0).all()


FORMS = [
    # kernel, M, K, N, counts, swiglu, pitch: two teams with several steps each, in even and odd numbers; rows quantised in the product's launch
    ("q8_panel_kernel<false, 2>", 100, 2304, 8300, None, False, None), ("q8_panel_kernel<false, 2>", 100, 1300, 8300, None, False, None),
    ("q8_panel_kernel<false, 2>", 300, 5640, 5000, None, False, 5648), ("q8_panel_kernel<true, 2>", 70, 2304, 9000, None, True, None),
    ("q8_panel_kernel<true, 2>", 70, 1300, 9000, None, True, None), ("q8_panel_kernel<true, 2>", 70, 1793, 9000, None, True, 1808),
    ("q8_panel_kernel<false, 2>", 0, 3100, 1024, [10, 0, 15, 9, 10, 70, 0, 2], False, None), ("q8_panel_kernel<false, 1>", 0, 2560, 1024, [10] * 64 + [0, 130], False, None),
    ("q8_panel_kernel<true, 1>", 0, 1088, 1408, [30, 0, 1, 64, 65, 7] * 9, True, None),
    ("q8_stream_kernel<1, false, 1, 8, 2, true>", 2, 520, 256, None, False, None), ("q8_stream_kernel<1, false, 2, 4, 1, true>", 3, 136, 20000, None, False, None),
    ("q8_stream_kernel<1, false, 2, 1, 1, true>", 4, 72, 66000, None, False, None), ("q8_stream_kernel<1, true, 2, 4, 1, true>", 1, 1000, 512, None, True, None),
    ("q8_stream_kernel<1, true, 2, 1, 1, true>", 2, 320, 66000, None, True, None),
]


@pytest.mark.parametrize("form,M,K,N,counts,swiglu,pitch", FORMS, ids=[f"{i}-{f[0][3:].replace(' ', '')}" for i, f in enumerate(FORMS)])
def test_forms_of_the_product(form, M, K, N, counts, swiglu, pitch):
    gen = torch.Generator().manual_seed(K + N)
    M = sum(counts) if counts else M
    x = torch.randn(M, K, generator=gen).bfloat16()
    for _ in range(3):      # the profiler loses a session's events now and then
        with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
            check_product(gen, x, len(counts) if counts else 1, N, counts, None, 1, swiglu, "bf16", pad_o=2, pitch=pitch, magnitude=4 / K ** 0.5)
        ran = [e.name for e in prof.events() if "q8_" in e.name and "kernel" in e.name]
        if ran:
            break
    assert len(ran) == 1 and form in ran[0], ran


def test_a_prompt_of_codes_that_cannot_be_read_in_place():
    gen = torch.Generator().manual_seed(12)
    check_product(gen, torch.randn(2100, 1001, generator=gen), 1, 300, out="f32", codes=True)
    check_product(gen, torch.randn(1200, 196, generator=gen), 4, 130, [500, 0, 1, 690], out="bf16", codes=True, swiglu=True, magnitude=0.3)


# ---- weighted sum --------------------------------------------------------------------------------

@pytest.mark.parametrize("d,pad", [(8, 0), (33, 3)])
@pytest.mark.parametrize("y_type", ["bf16", "f32"])
def test_combine_without_any_row(y_type, d, pad):
    """No row of y exists: every number of a row is out of range, the sums are NaN, and nothing of y is read."""
    y = torch.ones(4, d + pad, dtype=TYPES[y_type], device="cuda")
    inv = torch.tensor([0, 1, -1, 3, 0, 2], dtype=torch.int32, device="cuda")
    out = torch.full((4, d + pad), 5.0, device="cuda")
    w = torch.ones(3, 2, device="cuda")
    for address in (None, y.data_ptr()):
        out[:] = 5
        assert ef.lib().ef_combine(address, ef._rows(y)[1], d + pad, 0, w.data_ptr(), inv.data_ptr(), 3, 2, d, out.data_ptr(), ef.EF_F32, d + pad,
                                   stream().cuda_stream) == ef.EF_OK
        got = out.cpu()
        assert got[:3, :d].isnan().all() and (got[3] == 5).all() and (got[:, d:] == 5).all()
    out[:] = 5
    ef.ef_combine(y[:0, :d], w, inv, out[:3, :d], stream=stream())
    assert out[:3, :d].isnan().all() and (out[:, d:] == 5).all()


def test_combine_of_more_tokens_than_a_launch_has_workgroups():
    n = (1 << 24) + 3
    y, w, out = torch.randn(n, 1, device="cuda"), torch.randn(n, 1, device="cuda"), torch.full((n, 1), 7.0, device="cuda")
    ef.ef_combine(y, w, None, out, stream=stream())
    assert torch.equal(out, y * w)
    inv = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda")
    ef.ef_combine(y, w, inv, out, stream=stream())
    assert torch.equal(out, y.flip(0) * w)


# ---- the layer -----------------------------------------------------------------------------------

@pytest.mark.parametrize("handle", [False, True])
def test_layer_on_a_stream(handle):
    """The output's memory is of the stream that writes it, and holds what the current stream gives."""
    from paper_2510_26730_amd.q8_layer import Q8Layer
    gen = torch.Generator().manual_seed(8)
    E, d, F, T = 8, 4096, 128, 700
    layer = Q8Layer(torch.randn(E, 2 * F, d, generator=gen).cuda(), torch.randn(E, d, F, generator=gen).cuda(), 2, T, renorm=True)
    x, z = torch.randn(T, d, generator=gen).cuda(), torch.randn(T, E, generator=gen).cuda()
    want = layer(x, z).clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = layer(x, z, stream=side.cuda_stream if handle else side)
    side.synchronize()
    assert torch.equal(out, want)
    owner = [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= out.data_ptr() < s["address"] + s["total_size"]]
    assert owner == [side.cuda_stream]
