"""Group-scaled 4-bit layers and expert operators on the GPU against plain definitions in 64 bits.

Tolerances.  A stored value is rounded once to its type: half a step, eps / 2 of the value.  In front of that stand fp32 sums.  A term of a
product passes at most 16 additions inside a matrix instruction, 8 instructions of a sum over 128 inputs, one addition for every 128
inputs, and 24 where warps, cluster and parts join, each off by at most 2^-23 (matrix instructions cut off) of the sum of the terms' magnitudes S:
D * 2^-23 * S with D = 48 + K / 128.  (The scale's multiplication and the zero point are exact or one of these.)  A weighted sum back of k rows
passes k additions, 2^-24 each; a dot product of H values by threads at most H / 16 + 24."""
import numpy as np
import pytest

from oracle import gs4_oracle as G
from paper_2111_00153_b200 import binding as R

pytestmark = pytest.mark.gpu

TYPES = {"f32": R.F32, "f16": R.F16, "bf16": R.BF16}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}


def td(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def half_step(name):
    import torch
    return torch.finfo(td(name)).eps / 2


def dev(a, name=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if name is None else t.to(td(name))


def host(t):
    return t.detach().double().cpu().numpy()


class Packed:
    """A layer of random weights, packed from codes; `w`: [E][M][K] in 64 bits."""

    def __init__(self, seed, E, M, K, group, mode, scale_type="bf16", spread=0.02):
        import torch
        rng = np.random.default_rng(seed)
        Gn = -(-K // group)
        self.codes = rng.integers(0, 16, (E, M, K)).astype(np.uint8)
        scale = G.round_to((spread * (0.5 + rng.random((E, M, Gn)))).astype(np.float32), scale_type)
        self.zero = rng.integers(0, 16, (E, M, Gn)).astype(np.uint8) if mode == R.GS4_ZERO else np.full((E, M, Gn), 8, np.uint8)
        self.scale = scale
        self.w = G.weights(self.codes, scale, self.zero, group)
        self.layer = R.rmsmp_gs4_layer_init(E, M, K, group, mode, TYPES[scale_type])
        self.buf = torch.full((self.layer.packed_bytes + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        self.packed = self.buf[256:-256]
        R.rmsmp_gs4_pack_codes(self.layer, dev(self.codes), dev(scale, scale_type), dev(self.zero) if mode == R.GS4_ZERO else None, self.packed)


def framed(rows, cols, ld, name, fill=float("nan")):
    """A [rows][ld] output with spare rows and columns around it, all `fill`."""
    import torch
    buf = torch.full(((rows + 2) * ld + 64,), fill, dtype=td(name), device="cuda")
    return buf, buf[ld + 32:ld + 32 + rows * ld].view(rows, ld)


def check_close(y, ref, absum, name, depth, eps=2.0 ** -23):
    fin = np.isfinite(ref)
    err = np.abs(y - ref)
    tol = half_step(name) * np.abs(ref) * (1 + 2.0 ** -10) + depth * eps * absum + TINY[name]
    bad = fin & ~(err <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], y[bad][:5], ref[bad][:5], tol[bad][:5])


def run_linear(p, x, x_name, y_name, pad_x=0, pad_y=0):
    """x: [N][K] numpy, rounded to the type here.  Returns (y, reference, sums of magnitudes); checks that nothing else was written."""
    import torch
    N, K, M = x.shape[0], p.layer.K, p.layer.M
    xb, xv = framed(N, K, K + pad_x, x_name)          # NaN around and between the rows
    xv[:, :K] = dev(x.astype(np.float32)).to(td(x_name))
    yb, yv = framed(N, M, M + pad_y, y_name)
    R.rmsmp_gs4_gemm(p.layer, p.packed, xv, TYPES[x_name], N, K + pad_x, yv, TYPES[y_name], M + pad_y)
    torch.cuda.synchronize()
    assert R.rmsmp_last_device_status(p.packed) == R.OK
    out = host(yv[:, :M])
    yv[:, :M] = float("nan")
    assert torch.isnan(yb).all()
    ref, absum = G.product(p.w[0], host(xv[:, :K]))
    return out, ref, absum


# ------------------------------------------------------------------ packing

@pytest.mark.parametrize("E, M, K, group", [(1, 1, 1, 32), (1, 16, 128, 128), (2, 17, 129, 32), (1, 33, 300, 64), (3, 5, 100, 96), (1, 40, 700, 256), (2, 8, 70, 4096)])
@pytest.mark.parametrize("mode", [R.GS4_SYM, R.GS4_ZERO])
@pytest.mark.parametrize("scale_type", ["f16", "bf16"])
def test_pack_and_unpack(E, M, K, group, mode, scale_type):
    import torch
    p = Packed(E + M + K, E, M, K, group, mode, scale_type)
    codes = torch.empty((E, M, K), dtype=torch.uint8, device="cuda")
    scale = torch.empty(p.scale.shape, dtype=td(scale_type), device="cuda")
    zero = torch.empty(p.zero.shape, dtype=torch.uint8, device="cuda")
    R.rmsmp_gs4_unpack(p.layer, p.packed, codes, scale, zero)
    assert np.array_equal(codes.cpu().numpy(), p.codes) and np.array_equal(zero.cpu().numpy(), p.zero)
    assert np.array_equal(host(scale), p.scale.astype(np.float64))
    assert (p.buf[:256] == 0xA5).all() and (p.buf[-256:] == 0xA5).all()


@pytest.mark.parametrize("M, K, group", [(1, 1, 32), (20, 200, 32), (33, 300, 64), (16, 257, 128), (5, 333, 512)])
@pytest.mark.parametrize("mode", [R.GS4_SYM, R.GS4_ZERO])
@pytest.mark.parametrize("scale_type", ["f16", "bf16"])
@pytest.mark.parametrize("w_type", ["f32", "f16", "bf16"])
def test_quantizer_bit_for_bit(M, K, group, mode, scale_type, w_type):
    import torch
    rng = np.random.default_rng(M + K)
    W = rng.standard_normal((2, M, K)).astype(np.float32) * np.float32(0.02)
    W[0, 0, :min(K, 40)] = 0                            # a group of zeros
    W[1, 0] = np.abs(W[1, 0])                           # one-sided rows
    W[1, M - 1] = -np.abs(W[1, M - 1])
    if scale_type == "f16" and w_type == "f32":
        W[0, M - 1, :32] *= np.float32(1e-9)            # a step that fp16 rounds to zero
        W[1, M // 2, :32] *= np.float32(1e8)            # and one beyond its range
    dW = dev(W, w_type)
    L = R.rmsmp_gs4_layer_init(2, M, K, group, mode, TYPES[scale_type])
    packed = torch.empty(L.packed_bytes, dtype=torch.uint8, device="cuda")
    R.rmsmp_gs4_quantize_pack(L, dW, TYPES[w_type], packed)
    want = G.quantize(dW.float().cpu().numpy(), group, mode, scale_type)
    codes = torch.empty((2, M, K), dtype=torch.uint8, device="cuda")
    scale = torch.empty(want[1].shape, dtype=td(scale_type), device="cuda")
    zero = torch.empty(want[2].shape, dtype=torch.uint8, device="cuda")
    R.rmsmp_gs4_unpack(L, packed, codes, scale, zero)
    assert np.array_equal(scale.float().cpu().numpy(), want[1])
    assert np.array_equal(zero.cpu().numpy(), want[2])
    assert np.array_equal(codes.cpu().numpy(), want[0])


# ------------------------------------------------------------------ linear

@pytest.mark.parametrize("N", [1, 2, 3, 5, 8, 9, 16, 17, 33, 70])
@pytest.mark.parametrize("M, K, group", [(1, 1, 32), (16, 128, 128), (15, 31, 32), (130, 300, 64), (100, 1029, 96), (257, 640, 128)])
@pytest.mark.parametrize("x_name", ["f32", "f16", "bf16"])
def test_linear(N, M, K, group, x_name):
    p = Packed(N * M + K, 1, M, K, group, R.GS4_ZERO if (N + M) & 1 else R.GS4_SYM, "f16" if K & 1 else "bf16")
    x = np.random.default_rng(N + K).standard_normal((N, K))
    y, ref, absum = run_linear(p, x, x_name, x_name)
    check_close(y, ref, absum, x_name, 48 + K / 128)


@pytest.mark.parametrize("x_name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("y_name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("mode", [R.GS4_SYM, R.GS4_ZERO])
@pytest.mark.parametrize("N, pad_x, pad_y", [(1, 0, 0), (4, 8, 8), (7, 3, 1), (40, 5, 16)])
def test_types_and_strides(x_name, y_name, mode, N, pad_x, pad_y):
    p = Packed(N, 1, 75, 424, 64, mode, "f16")
    x = np.random.default_rng(N).standard_normal((N, 424))
    y, ref, absum = run_linear(p, x, x_name, y_name, pad_x, pad_y)
    check_close(y, ref, absum, y_name, 52)


@pytest.mark.parametrize("group", [32, 64, 96, 128, 256, 1 << 20])
@pytest.mark.parametrize("K", [32, 127, 129, 1000])
@pytest.mark.parametrize("mode", [R.GS4_SYM, R.GS4_ZERO])
def test_groups(group, K, mode):
    p = Packed(K, 1, 50, K, group, mode)
    for N, name in ((1, "bf16"), (6, "f32"), (20, "f16")):
        x = np.random.default_rng(K).standard_normal((N, K))
        y, ref, absum = run_linear(p, x, name, name)
        check_close(y, ref, absum, name, 48 + K / 128)


@pytest.mark.parametrize("M, K, N", [(16, 20000, 1), (64, 9000, 33), (5000, 64, 2), (2500, 2500, 12), (48, 30011, 3), (300, 4096, 200)])
@pytest.mark.parametrize("x_name", ["f32", "bf16"])
def test_long_rows_and_many_rows(M, K, N, x_name):
    p = Packed(M, 1, M, K, 128 if K % 2 == 0 else 32, R.GS4_ZERO)
    x = np.random.default_rng(K).standard_normal((N, K))
    y, ref, absum = run_linear(p, x, x_name, x_name)
    check_close(y, ref, absum, x_name, 48 + K / 128)


@pytest.mark.parametrize("x_name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M, K, N, group, pad_x, pad_y", [(40, 70, 130, 32, 0, 0), (130, 1029, 300, 96, 0, 3), (520, 2304, 150, 64, 8, 4), (129, 640, 257, 128, 1, 0), (300, 130, 513, 64, 0, 2)])
@pytest.mark.parametrize("mode", [R.GS4_SYM, R.GS4_ZERO])
def test_many_tokens(M, K, N, group, pad_x, pad_y, mode, x_name):
    p = Packed(M + N, 1, M, K, group, mode, "f16" if N & 1 else "bf16")
    x = np.random.default_rng(N).standard_normal((N, K))
    y, ref, absum = run_linear(p, x, x_name, x_name, pad_x, pad_y)
    check_close(y, ref, absum, x_name, 48 + K / 128)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("x_name", ["f16", "bf16"])
def test_tiles_of_256_tokens(group, x_name):
    """Enough tiles for every SM, the widest tiles, and more blocks of inputs than the ring of packed codes has slots."""
    p = Packed(group, 1, 4096, 768, group, R.GS4_ZERO)
    x = np.random.default_rng(group).standard_normal((1024, 768))
    for pad in (0, 4):                                  # rows that the copy engine can address, and rows that it cannot
        y, ref, absum = run_linear(p, x, x_name, x_name, pad, 0)
        check_close(y, ref, absum, x_name, 54)


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("N", [745, 768])
@pytest.mark.parametrize("pad", [0, 4])
def test_tiles_of_192_tokens(N, group, pad):
    p = Packed(N + group, 1, 4096, 384, group, R.GS4_ZERO)
    x = np.random.default_rng(N).standard_normal((N, 384))
    y, ref, absum = run_linear(p, x, "bf16", "bf16", pad, 0)
    check_close(y, ref, absum, "bf16", 51)


@pytest.mark.parametrize("x_name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("by_rows", [True, False])
def test_experts_with_many_tokens(x_name, by_rows):
    import torch
    E, M, K, T, k = 5, 200, 400, 260, 2
    p = Packed(E, E, M, K, 32, R.GS4_ZERO)
    ids = route(3, T, k, E, 0.1)
    ids[:, 0] = np.where(ids[:, 0] >= 0, 2, -1)         # one expert with far more than its share, which a token may name twice
    offsets, rows, _ = G.sort_pairs(ids, E)
    x = dev(np.random.default_rng(T).standard_normal((T, K)).astype(np.float32)).to(td(x_name))
    xs = x if by_rows else x[dev(np.maximum(rows, 0)).long()].contiguous()
    yb, y = framed(T * k, M, M + 1, x_name)
    R.rmsmp_gs4_gemm_experts(p.layer, p.packed, xs, TYPES[x_name], xs.shape[0], K, dev(rows) if by_rows else None, dev(offsets), T * k, y, TYPES[x_name], M + 1)
    torch.cuda.synchronize()
    assert R.rmsmp_last_device_status(p.packed) == R.OK
    out, hx = host(y), host(x)
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        if b > a:
            ref, absum = G.product(p.w[e], hx[rows[a:b]])
            check_close(out[a:b, :M], ref, absum, x_name, 52)
    y[:offsets[-1], :M] = float("nan")
    assert torch.isnan(yb).all()


@pytest.mark.parametrize("x_name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("E, T, popular", [(6, 45, 2), (600, 300, 599), (600, 33, 256), (1, 7, 0)])
def test_a_popular_expert_among_few_tokens(E, T, popular, x_name):
    """Few tokens an expert on average, most of them with one: its tokens take several passes; more experts than a CTA has threads."""
    import torch
    M, K, k = 70, 300, 2
    p = Packed(E + T, E, M, K, 32, R.GS4_SYM)
    ids = route(T, T, k, E, 0.1)
    ids[:, 0] = np.where(ids[:, 0] >= 0, popular, -1)
    offsets, rows, _ = G.sort_pairs(ids, E)
    x = dev(np.random.default_rng(T).standard_normal((T, K)).astype(np.float32)).to(td(x_name))
    yb, y = framed(T * k, M, M + 2, x_name)
    R.rmsmp_gs4_gemm_experts(p.layer, p.packed, x, TYPES[x_name], T, K, dev(rows), dev(offsets), T * k, y, TYPES[x_name], M + 2)
    torch.cuda.synchronize()
    assert R.rmsmp_last_device_status(p.packed) == R.OK
    out, hx = host(y), host(x)
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        if b > a:
            ref, absum = G.product(p.w[e], hx[rows[a:b]])
            check_close(out[a:b, :M], ref, absum, x_name, 52)
    y[:offsets[-1], :M] = float("nan")
    assert torch.isnan(yb).all()


def test_rows_of_x_that_are_not_there():
    """Fewer rows of x than of y, with and without an index: zeros."""
    import torch
    for Rn in (6, 100):
        p = Packed(1, 2, 70, 96, 32, R.GS4_SYM)
        for x_name in ("f32", "bf16"):
            x = dev(np.random.default_rng(1).standard_normal((4, 96)).astype(np.float32)).to(td(x_name))
            offsets = dev(np.array([0, Rn // 2, Rn], np.int32))
            rows = np.arange(Rn, dtype=np.int32)
            for index in (None, dev(rows)):
                y = torch.full((Rn, 70), float("nan"), dtype=td(x_name), device="cuda")
                R.rmsmp_gs4_gemm_experts(p.layer, p.packed, x, TYPES[x_name], 4, 96, index, offsets, Rn, y, TYPES[x_name], 70)
                out = host(y)
                for e in range(2):
                    for q in range(e * (Rn // 2), Rn if e else Rn // 2):
                        xr = host(x)[q:q + 1] if q < 4 else np.zeros((1, 96))
                        ref, absum = G.product(p.w[e], xr)
                        check_close(out[q:q + 1], ref, absum, x_name, 52)


@pytest.mark.parametrize("x_name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("Rn", [6, 120])
@pytest.mark.parametrize("by_rows", [True, False])
def test_x_without_any_rows(x_name, Rn, by_rows):
    """No rows of x, and no address either: every row that has an expert is zeros, few and many of them."""
    import torch
    p = Packed(2, 2, 70, 256, 64, R.GS4_ZERO)
    y = torch.full((Rn, 70), float("nan"), dtype=td(x_name), device="cuda")
    index = torch.arange(Rn, dtype=torch.int32, device="cuda") if by_rows else None
    R.rmsmp_gs4_gemm_experts(p.layer, p.packed, None, TYPES[x_name], 0, 256, index, dev(np.array([1, Rn // 3, Rn - 1], np.int32)), Rn, y, TYPES[x_name], 70)
    torch.cuda.synchronize()
    assert R.rmsmp_last_device_status(p.packed) == R.OK
    assert (y[1:-1] == 0).all() and torch.isnan(y[0]).all() and torch.isnan(y[-1]).all()


def test_two_streams_at_once():
    """The same layer on two streams, many tokens on one and few on the other, again and again: nothing is shared but the weights."""
    import torch
    p = Packed(4, 1, 512, 1024, 64, R.GS4_ZERO)
    rng = np.random.default_rng(4)
    xs = [dev(rng.standard_normal((n, 1024)).astype(np.float32)).to(torch.bfloat16) for n in (3, 200)]
    want = []
    for x in xs:
        y = torch.empty((x.shape[0], 512), dtype=torch.bfloat16, device="cuda")
        R.rmsmp_gs4_gemm(p.layer, p.packed, x, R.BF16, x.shape[0], 1024, y, R.BF16, 512)
        want.append(y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [[torch.empty_like(w) for _ in range(20)] for w in want]
    for i in range(20):
        for s, x, o in zip(streams, xs, outs):
            R.rmsmp_gs4_gemm(p.layer, p.packed, x, R.BF16, x.shape[0], 1024, o[i], R.BF16, 512, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for w, os in zip(want, outs) for o in os)
    assert R.rmsmp_last_device_status(p.packed) == R.OK


def test_no_tokens():
    import torch
    p = Packed(1, 1, 20, 40, 32, R.GS4_SYM)
    R.rmsmp_gs4_gemm(p.layer, p.packed, None, R.F32, 0, 40, None, R.F32, 20)
    torch.cuda.synchronize()


def test_exact_where_everything_is_small_integers():
    """Scales of one and whole activations: every sum is a whole number below 2^24, so the result is exact in fp32."""
    for x_name in ("f32", "f16", "bf16"):
        rng = np.random.default_rng(5)
        p = Packed(7, 1, 65, 515, 64, R.GS4_ZERO)
        p2 = Packed(7, 1, 65, 515, 64, R.GS4_ZERO, spread=0.0)
        import torch
        R.rmsmp_gs4_pack_codes(p2.layer, dev(p.codes), dev(np.ones(p.scale.shape, np.float32), "bf16"), dev(p.zero), p2.packed)
        p2.w = G.weights(p.codes, np.ones(p.scale.shape), p.zero, 64)
        x = rng.integers(-9, 10, (11, 515)).astype(np.float64)
        y, ref, _ = run_linear(p2, x, x_name, "f32")
        assert np.array_equal(y, ref)


@pytest.mark.parametrize("x_name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N", [1, 4, 20])
def test_infinities_and_nans_stay_in_their_rows(x_name, N):
    p = Packed(3, 1, 40, 200, 32, R.GS4_SYM)
    x = np.random.default_rng(3).standard_normal((N + 3, 200))
    x[0, 5] = np.inf
    x[1, 100] = -np.inf
    x[2, 199] = np.nan
    import torch
    dx = dev(x.astype(np.float32)).to(td(x_name))
    y = torch.empty((N + 3, 40), dtype=td(x_name), device="cuda")
    R.rmsmp_gs4_gemm(p.layer, p.packed, dx, TYPES[x_name], N + 3, 200, y, TYPES[x_name], 40)
    out = host(y)
    with np.errstate(invalid="ignore"):
        ref = host(dx) @ p.w[0].T
    assert np.array_equal(np.isnan(out[:3]), np.isnan(ref[:3]))
    fin = ~np.isnan(ref[:3])
    assert np.array_equal(out[:3][fin], ref[:3][fin])
    r, a = G.product(p.w[0], host(dx)[3:])
    check_close(out[3:], r, a, x_name, 52)


def test_fp32_activations_over_their_whole_range():
    """The largest and the smallest normal numbers: parts are cut off, not rounded, so none overflows."""
    p = Packed(9, 1, 20, 96, 32, R.GS4_SYM, spread=0.001)
    for size in (3.4e38, 1e-30, 2.0 ** -126):
        x = np.sign(np.random.default_rng(1).standard_normal((2, 96))) * 0
        x[0, 3] = size
        x[1, 90] = -size
        y, ref, absum = run_linear(p, x, "f32", "f32")
        if size == 3.4e38:
            big = np.abs(ref / p.scale[0, :, [0]][0, 0]) < 1e38         # the sum of codes times activations has to fit
            code = p.codes[0].astype(np.int64) - 8
            fits = np.stack([np.abs(code[:, 3]) <= 1, np.abs(code[:, 90]) <= 1])
            y, ref, absum = y[fits], ref[fits], absum[fits]
        tol = 2.0 ** -23 * np.abs(ref) * 4 + 2.0 ** -126 * 2.0 ** -10
        assert np.all(np.abs(y - ref) <= tol)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("x_name", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("by_expert", [False, True])
def test_what_few_tokens_keep_of_an_activation(group, x_name, by_expert):
    """Row m has one code that is not its zero point, at input m, and a scale of one: y is x as the kernel holds it.  fp16 is exact.  The others are off by at
    most 2^-39 of the largest number of their run (half of fp16's smallest step, 2^-25, beside 2^14), and fp32 by 2^-23 of itself: of a number in 2^e..2^(e+1)
    the first fp16 part leaves 2^(e-11) at most, which the second, whose half step is 2^-11 of the power of two below that, keeps to 2^(e-12-11)."""
    import torch
    size = K = 256
    codes = np.full((1, size, K), 8, np.uint8)
    codes[0, np.arange(size), np.arange(K)] = 9
    layer = R.rmsmp_gs4_layer_init(1, size, K, group, R.GS4_SYM, R.F16)
    packed = torch.empty(layer.packed_bytes, dtype=torch.uint8, device="cuda")
    R.rmsmp_gs4_pack_codes(layer, dev(codes), dev(np.ones((1, size, K // group), np.float32), "f16"), None, packed)
    rng = np.random.default_rng(group)
    x = rng.standard_normal((4, K)) * 2.0 ** rng.integers(-42, 1, (4, K))      # far below the largest of their run
    x[1] = 2.0 ** 14 * (1 + rng.random(K))                                     # all in one power of two
    x[1, ::7] = 2.0 ** 14 + 4 + 2.0 ** -9                                      # the first part's half step, and half of the second's
    x[2, ::9] = 2.0 ** -39
    x[2, ::32] = 1.0                                                           # ... beside the largest of every run
    x[2, 1::11] = 1.0078125 * 2.0 ** -32
    x[3] = rng.standard_normal(K) * 2.0 ** -130                                # subnormal ones
    if x_name == "f16":
        x[1] /= 2
    dx = dev(x).to(td(x_name))
    y = torch.empty((4, size), device="cuda")
    if by_expert:
        R.rmsmp_gs4_gemm_experts(layer, packed, dx, TYPES[x_name], 4, K, None, dev(np.array([0, 4], np.int32)), 4, y, R.F32, size)
    else:
        R.rmsmp_gs4_gemm(layer, packed, dx, TYPES[x_name], 4, K, y, R.F32, size)
    want, got = host(dx), host(y)
    run = np.abs(want).reshape(4, -1, min(group, 128)).max(-1).repeat(min(group, 128), axis=1)
    bound = {"f16": 0.0 * run, "bf16": 2.0 ** -39 * run, "f32": 2.0 ** -39 * run + 2.0 ** -23 * np.abs(want)}[x_name]
    assert np.all(np.abs(got - want) <= bound)
    if x_name == "f32":
        assert np.abs((got - want) / want)[1].max() > 2.0 ** -24               # (and no better: what the header says is what there is)


# ------------------------------------------------------------------ experts

def route(seed, T, k, E, padded=0.0, only=None):
    rng = np.random.default_rng(seed)
    ids = np.stack([rng.permutation(E)[:k] if k <= E else rng.integers(0, E, k) for _ in range(T)]) if T else np.zeros((0, k))
    if only is not None:
        ids = rng.choice(only, (T, k))
    ids[rng.random(T) < padded] = -1
    return ids.astype(np.int32)


@pytest.mark.parametrize("T, k, E, kind", [(1, 1, 1, "all"), (1, 2, 8, "all"), (5, 2, 4, "padded"), (40, 3, 7, "all"), (64, 2, 3, "padded"), (9, 2, 6, "none"),
                                           (70, 1, 5, "one"), (300, 4, 16, "padded"), (3, 8, 100, "all")])
@pytest.mark.parametrize("x_name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("by_rows", [True, False])
def test_experts(T, k, E, kind, x_name, by_rows):
    import torch
    M, K = 50, 200
    p = Packed(T + E, E, M, K, 64, R.GS4_ZERO if E & 1 else R.GS4_SYM)
    ids = route(T, T, k, E, {"padded": 0.3, "none": 1.0}.get(kind, 0.0), [E // 2] if kind == "one" else None)
    offsets, rows, _ = G.sort_pairs(ids, E)
    x = np.random.default_rng(T).standard_normal((T, K))
    dx = dev(x.astype(np.float32)).to(td(x_name))
    dxs = dx if by_rows else dx[dev(np.maximum(rows, 0)).long()]
    P = T * k
    yb, y = framed(P, M, M + 3, x_name)
    R.rmsmp_gs4_gemm_experts(p.layer, p.packed, dxs, TYPES[x_name], dxs.shape[0], K, dev(rows) if by_rows else None, dev(offsets), P, y, TYPES[x_name], M + 3)
    torch.cuda.synchronize()
    assert R.rmsmp_last_device_status(p.packed) == R.OK
    out, hx = host(y), host(dx)
    for e in range(E):
        a, b = offsets[e], offsets[e + 1]
        if b > a:
            ref, absum = G.product(p.w[e], hx[rows[a:b]])
            check_close(out[a:b, :M], ref, absum, x_name, 52)
    y[:offsets[-1], :M] = float("nan")
    assert torch.isnan(yb).all()                       # rows behind the last, and everything around, are as they were


def test_experts_with_bad_offsets_and_rows_stay_inside():
    """Offsets beyond the capacity are cut; a row index outside x is a row of zeros; falling offsets fault nothing."""
    import torch
    E, M, K, Rn = 4, 40, 96, 12
    p = Packed(1, E, M, K, 32, R.GS4_SYM)
    x = np.random.default_rng(1).standard_normal((5, K)).astype(np.float32)
    rows = np.array([0, 4, 5, -1, 2, 1 << 30, -(1 << 31), 3, 1, 0, 0, 4], np.int32)
    for offsets in ([-7, 3, 3, 10, 99], [0, 5, 2, 2, 12], [12, 12, 12, 12, 40], [0, 0, 0, 0, 0]):
        yb, y = framed(Rn, M, M, "f32")
        R.rmsmp_gs4_gemm_experts(p.layer, p.packed, dev(x), R.F32, 5, K, dev(rows), dev(np.array(offsets, np.int32)), Rn, y, R.F32, M)
        torch.cuda.synchronize()
        out = host(y)
        claims = [[] for _ in range(Rn)]
        for e in range(E):
            for q in range(max(0, offsets[e]), min(Rn, offsets[e + 1])):
                claims[q].append(e)
        for q, of in enumerate(claims):
            xr = x[rows[q]].astype(np.float64) if 0 <= rows[q] < 5 else np.zeros(K)
            refs = [G.product(p.w[e], xr[None]) for e in of]
            if len(of) == 1:
                check_close(out[q:q + 1], *refs[0], "f32", 52)
            elif of:                                   # falling offsets, which the call does not allow, name a row twice: either's values
                assert all(any(abs(out[q, m] - r[0, m]) <= 1e-4 * a[0, m] for r, a in refs) for m in range(M))
        written = np.array([bool(of) for of in claims])
        y[torch.from_numpy(written).cuda()] = float("nan")
        assert torch.isnan(yb).all()


# ------------------------------------------------------------------ order

@pytest.mark.parametrize("T, k, E", [(0, 2, 8), (1, 1, 1), (1, 2, 8), (7, 3, 5), (33, 1, 2), (100, 8, 64), (1000, 2, 1024), (3000, 4, 17), (20000, 8, 256), (5, 1024, 3), (70001, 1, 33)])
@pytest.mark.parametrize("kind", ["all", "padded", "none", "one", "wild"])
def test_sort(T, k, E, kind):
    import torch
    rng = np.random.default_rng(T + k)
    ids = rng.integers(0, E, (T, k)).astype(np.int32)
    if kind == "padded":
        ids[rng.random((T, k)) < 0.3] = -1
    elif kind == "none":
        ids[:] = E
    elif kind == "one":
        ids[:] = E - 1
    elif kind == "wild":
        ids = rng.integers(-2 ** 31, 2 ** 31, (T, k)).astype(np.int32)
        ids[rng.random((T, k)) < 0.5] = 0
    off = torch.full((E + 3,), -9, dtype=torch.int32, device="cuda")
    rows = torch.full((T * k + 2,), -9, dtype=torch.int32, device="cuda")
    place = torch.full((T * k + 2,), -9, dtype=torch.int32, device="cuda")
    R.rmsmp_expert_sort(dev(ids), T, k, E, off[1:], rows[1:], place[1:])
    want = G.sort_pairs(ids, E)
    assert np.array_equal(off[1:E + 2].cpu().numpy(), want[0])
    assert np.array_equal(rows[1:-1].cpu().numpy(), want[1])
    assert np.array_equal(place[1:-1].cpu().numpy().reshape(T, k), want[2])
    assert all(int(t[0]) == -9 and int(t[-1]) == -9 for t in (off, rows, place))


# ------------------------------------------------------------------ rows

ROWS = [(1, 1, 3, 1, 0), (1, 2, 8, 1024, 0), (5, 4, 16, 777, 0), (30, 2, 4, 64, 8), (30, 2, 4, 64, 3), (200, 8, 32, 2048, 0), (9, 3, 5, 8200, 0), (17, 1, 2, 33, 5),
        (60, 20, 50, 24, 0)]


@pytest.mark.parametrize("T, k, E, H, pad", ROWS)
@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("padded", [0.0, 0.4, 1.0])
def test_gather_and_combine(T, k, E, H, pad, name, padded):
    import torch
    ids = route(T + H, T, k, E, padded)
    offsets, rows, place = G.sort_pairs(ids, E)
    P, kept = T * k, offsets[-1]
    rng = np.random.default_rng(H)
    xb, x = framed(T, H, H + pad, name)
    x[:, :H] = dev(rng.standard_normal((T, H)).astype(np.float32)).to(td(name))
    sb, xs = framed(P, H, H + pad, name)
    R.rmsmp_expert_gather(x, TYPES[name], T, H, H + pad, dev(rows), P, xs, H + pad)
    assert np.array_equal(host(xs[:kept, :H]), host(x[:, :H])[rows[:kept]])
    keep = xs.clone()
    xs[:kept, :H] = float("nan")
    assert torch.isnan(sb).all()
    w = rng.random((T, k)).astype(np.float32)
    for weights in (w, None):
        yb, y = framed(T, H, H + pad, name)
        R.rmsmp_expert_combine(keep, TYPES[name], P, H, H + pad, dev(place), None if weights is None else dev(weights), T, k, y, H + pad)
        ref, absum = G.combine(host(keep[:, :H]), place, weights)
        check_close(host(y[:, :H]), ref, absum, name, k, 2.0 ** -24)
        y[:, :H] = float("nan")
        assert torch.isnan(yb).all()


@pytest.mark.parametrize("T, k, E, H, pad", ROWS)
@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("padded", [0.0, 0.4, 1.0])
def test_combine_backward(T, k, E, H, pad, name, padded):
    import torch
    ids = route(T + H, T, k, E, padded)
    _, _, place = G.sort_pairs(ids, E)
    P = T * k
    rng = np.random.default_rng(H + 1)
    fill = lambda rows: dev(rng.standard_normal((rows, H)).astype(np.float32)).to(td(name))
    _, dy = framed(T, H, H + pad, name)
    _, ys = framed(P, H, H + pad, name)
    dy[:, :H], ys[:, :H] = fill(T), fill(P)
    w = rng.random((T, k)).astype(np.float32)
    for weights in (w, None):
        ref, dw_ref, absum = G.combine_backward(host(dy[:, :H]), host(ys[:, :H]), place, weights)
        for want_dys, want_dw in ((True, True), (True, False), (False, True)):
            sb, dys = framed(P, H, H + pad, name)
            dwb = torch.full((T * k + 2,), -9.0, device="cuda")
            R.rmsmp_expert_combine_backward(dy, TYPES[name], T, k, H, H + pad, ys if want_dw else None, P, H + pad, dev(place),
                                            None if weights is None else dev(weights), dys if want_dys else None, H + pad, dwb[1:] if want_dw else None)
            if want_dys:
                out, kept = host(dys[:, :H]), ~np.isnan(ref[:, 0])
                assert np.isnan(out[~kept]).all()
                check_close(out[kept], ref[kept], np.abs(ref[kept]), name, 1, 2.0 ** -24)
                dys[:, :H] = float("nan")
            assert torch.isnan(sb).all()
            if want_dw:
                check_close(host(dwb[1:-1]).reshape(T, k), dw_ref, absum, "f32", H / 16 + 24, 2.0 ** -24)
            assert float(dwb[0]) == -9.0 and float(dwb[-1]) == -9.0


@pytest.mark.parametrize("H", [8, 777, 2048])
def test_pairs_that_share_a_place(H):
    """Each value of the row is one of those pairs'; dw is right for all of them, and no other row is touched."""
    import torch
    T, k, P = 40, 2, 9
    rng = np.random.default_rng(H)
    dy, ys = rng.standard_normal((T, H)).astype(np.float32), rng.standard_normal((P, H)).astype(np.float32)
    place = np.full((T, k), -1, np.int32)
    place[:, 1] = 5
    place[3] = (7, 7)                                   # ... and twice by one token
    dys, dw = torch.full((P, H), float("nan"), device="cuda"), torch.empty((T, k), device="cuda")
    R.rmsmp_expert_combine_backward(dev(dy), R.F32, T, k, H, H, dev(ys), P, H, dev(place), None, dys, H, dw)
    _, dw_ref, absum = G.combine_backward(dy, ys, place, None)
    check_close(host(dw), dw_ref, absum, "f32", H / 16 + 24, 2.0 ** -24)
    out = host(dys)
    others = np.delete(dy, 3, 0)
    assert (out[5][None] == others).any(0).all() and np.array_equal(out[7], dy[3])
    assert np.isnan(np.delete(out, (5, 7), 0)).all()


@pytest.mark.parametrize("H", [8, 33, 4096])
def test_sums_back_without_any_rows(H):
    """A capacity of none: sums and weights' gradients are zeros, and the rows' gradient, whose empty tensor has no address, is nothing."""
    import torch
    T, k = 7, 3
    rows, place = torch.empty((0, H), device="cuda"), torch.arange(T * k, dtype=torch.int32, device="cuda").view(T, k)
    w, dy = torch.ones((T, k), device="cuda"), torch.ones((T, H), device="cuda")
    y = torch.full((T, H), float("nan"), device="cuda")
    R.rmsmp_expert_combine(rows, R.F32, 0, H, H, place, w, T, k, y, H)
    assert (y == 0).all()
    for want_dw in (True, False):
        dw = torch.full((T, k), float("nan"), device="cuda")
        R.rmsmp_expert_combine_backward(dy, R.F32, T, k, H, H, rows, 0, H, place, w, torch.empty_like(rows), H, dw if want_dw else None)
        assert (dw == 0).all() if want_dw else torch.isnan(dw).all()


def test_gradients_against_differences():
    """The sum is linear in the rows and in the weights: differences of the call itself give its gradient up to rounding."""
    import torch
    T, k, E, H = 6, 2, 3, 16
    ids = route(4, T, k, E, 0.2)
    _, rows, place = G.sort_pairs(ids, E)
    P = T * k
    rng = np.random.default_rng(8)
    ys, w, dy = rng.standard_normal((P, H)).astype(np.float32), rng.random((T, k)).astype(np.float32), rng.standard_normal((T, H)).astype(np.float32)

    def loss(a, b):
        y = torch.empty((T, H), device="cuda")
        R.rmsmp_expert_combine(dev(a), R.F32, P, H, H, dev(place), dev(b), T, k, y, H)
        return float((host(y) * dy).sum())
    dys, dw = torch.zeros((P, H), device="cuda"), torch.empty((T, k), device="cuda")
    R.rmsmp_expert_combine_backward(dev(dy), R.F32, T, k, H, H, dev(ys), P, H, dev(place), dev(w), dys, H, dw)
    room = 64 * 2.0 ** -24 * (1 + np.abs(dy).max()) * H          # two sums of T * H fp32 values, one of which moved by one
    for p in range(0, P, 3):
        d = np.zeros_like(ys)
        d[p, p % H] = 1
        assert abs(loss(ys + d, w) - loss(ys, w) - float(dys[p, p % H])) < room
    for t in range(T):
        d = np.zeros_like(w)
        d[t, t % k] = 1
        assert abs(loss(ys, w + d) - loss(ys, w) - float(dw[t, t % k])) < room


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T", [1, 24])
def test_a_layer_of_experts_as_it_is_used(name, T):
    """Sort, first product by the sorted rows, activation, second product, weighted sum back; then once more from a captured graph with new inputs."""
    import torch
    E, k, K, F = 6, 2, 96, 160
    up, down = Packed(1, E, F, K, 32, R.GS4_ZERO), Packed(2, E, K, F, 64, R.GS4_SYM)
    P, t = T * k, TYPES[name]
    x = torch.empty((T, K), dtype=td(name), device="cuda")
    ids, w = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")
    off, rows = torch.empty(E + 1, dtype=torch.int32, device="cuda"), torch.empty(P, dtype=torch.int32, device="cuda")
    place = torch.empty((T, k), dtype=torch.int32, device="cuda")
    h, z, y = torch.zeros((P, F), dtype=td(name), device="cuda"), torch.zeros((P, K), dtype=td(name), device="cuda"), torch.empty((T, K), dtype=td(name), device="cuda")

    def step():
        R.rmsmp_expert_sort(ids, T, k, E, off, rows, place)
        R.rmsmp_gs4_gemm_experts(up.layer, up.packed, x, t, T, K, rows, off, P, h, t, F)
        h.relu_()
        R.rmsmp_gs4_gemm_experts(down.layer, down.packed, h, t, P, F, None, off, P, z, t, K)
        R.rmsmp_expert_combine(z, t, P, K, K, place, w, T, k, y, K)

    def new_inputs(seed):
        rng = np.random.default_rng(seed)
        x.copy_(dev(rng.standard_normal((T, K)).astype(np.float32)))
        ids.copy_(dev(route(seed, T, k, E, 0.2)))
        w.copy_(dev(rng.random((T, k)).astype(np.float32)))

    def check():
        torch.cuda.synchronize()
        hid, hx, hw = ids.cpu().numpy(), host(x), host(w)
        ref = np.zeros((T, K))
        size = np.zeros((T, K))
        for a in range(T):
            for j in range(k):
                e = hid[a, j]
                if e >= 0:
                    hh, ha = G.product(up.w[e], hx[a:a + 1])
                    zz, za = G.product(down.w[e], np.maximum(hh, 0))
                    ref[a] += hw[a, j] * zz[0]
                    size[a] += hw[a, j] * (np.abs(down.w[e]) @ (ha[0]))          # magnitudes carried through both products
        # h, z and y are each rounded to the type; everything else is fp32
        assert np.all(np.abs(host(y) - ref) <= 3 * half_step(name) * (size + np.abs(ref)) + 200 * 2.0 ** -23 * size + TINY[name])
    new_inputs(1)
    step()
    check()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (2, 3):
        new_inputs(seed)
        graph.replay()
        check()


def test_results_repeat_bit_for_bit():
    import torch
    p = Packed(3, 1, 1024, 4096, 128, R.GS4_SYM)
    x = dev(np.random.default_rng(1).standard_normal((3, 4096)).astype(np.float32))
    ys = [torch.empty((3, 1024), device="cuda") for _ in range(4)]
    for y in ys:
        R.rmsmp_gs4_gemm(p.layer, p.packed, x, R.F32, 3, 4096, y, R.F32, 1024)
    assert all(torch.equal(ys[0], y) for y in ys)


@pytest.mark.parametrize("N", [3, 2100])
def test_x_and_y_beyond_2_to_the_31(N):
    """Rows of 2^31 / 2 elements apart for few tokens, of 2^20 for many: the last row is past 2^31 elements and 2^32 bytes."""
    import torch
    ld = (1 << 30) + 8 if N == 3 else 1 << 20
    p = Packed(N, 1, 40, 200, 64, R.GS4_ZERO)
    xb, yb = (torch.empty((N - 1) * ld + 256, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x, y = (torch.as_strided(b, (N, c), (ld, 1)) for b, c in ((xb, 200), (yb, 40)))
    x.copy_(torch.from_numpy(np.random.default_rng(N).standard_normal((N, 200)).astype(np.float32)))
    R.rmsmp_gs4_gemm(p.layer, p.packed, x, R.BF16, N, ld, y, R.BF16, ld)
    torch.cuda.synchronize()
    ref, absum = G.product(p.w[0], host(x.contiguous()))
    check_close(host(y.contiguous()), ref, absum, "bf16", 50)
    rows = dev(np.array([N - 1, 0, N - 1], np.int32))
    out = torch.empty((3, 200), dtype=torch.bfloat16, device="cuda")
    R.rmsmp_expert_gather(x, R.BF16, N, 200, ld, rows, 3, out, 200)
    assert torch.equal(out, x[rows.long()])
    place = dev(np.array([[N - 1, 0]], np.int32))
    R.rmsmp_expert_combine(x, R.BF16, N, 200, ld, place, None, 1, 2, out, 200)
    assert torch.equal(out[0], (x[N - 1].float() + x[0].float()).bfloat16())
    R.rmsmp_expert_combine_backward(out, R.BF16, 1, 2, 40, 200, None, N, ld, place, None, y, ld, None)
    assert torch.equal(y[N - 1], out[0, :40]) and torch.equal(y[0], out[0, :40])


def test_weights_beyond_2_to_the_32():
    """More than 2^32 weights, the last matrix the only one that is not zero; then more than 2^32 bytes of packed ones."""
    import torch
    E, M, K = 260, 4096, 4096
    W = torch.zeros((E, M, K), dtype=torch.bfloat16, device="cuda")
    W[-1].copy_(torch.from_numpy(np.random.default_rng(8).standard_normal((M, K)).astype(np.float32)))
    layer, last = R.rmsmp_gs4_layer_init(E, M, K, 128, R.GS4_ZERO, R.F16), R.rmsmp_gs4_layer_init(1, M, K, 128, R.GS4_ZERO, R.F16)
    packed, want = (torch.empty(l.packed_bytes, dtype=torch.uint8, device="cuda") for l in (layer, last))
    R.rmsmp_gs4_quantize_pack(layer, W, R.BF16, packed)
    R.rmsmp_gs4_quantize_pack(last, W[-1].contiguous(), R.BF16, want)
    blocks = last.tiles * (last.Kp // 128) * last.block_bytes
    at = layer.off_blocks + (E - 1) * blocks
    assert torch.equal(packed[at:at + blocks], want[256:256 + blocks])
    sizes = W[-1].double().abs()
    del W, packed
    E = 500
    layer = R.rmsmp_gs4_layer_init(E, M, K, 128, R.GS4_ZERO, R.F16)
    packed = torch.zeros(layer.packed_bytes, dtype=torch.uint8, device="cuda")
    assert layer.packed_bytes > 1 << 32
    packed[layer.off_blocks + (E - 1) * blocks:][:blocks] = want[256:256 + blocks]
    for N in (2, 30 * E):                               # few tokens an expert; many
        rows = torch.randn((N, K), device="cuda").bfloat16()
        few = min(N, 300)
        offsets = np.full(E + 1, N - few, np.int32)
        offsets[0], offsets[-1] = 0, N
        y, ref = torch.empty((N, M), dtype=torch.bfloat16, device="cuda"), torch.empty((few, M), dtype=torch.bfloat16, device="cuda")
        R.rmsmp_gs4_gemm_experts(layer, packed, rows, R.BF16, N, K, None, dev(offsets), N, y, R.BF16, M)
        one_offsets = dev(np.array([0, few], np.int32))
        R.rmsmp_gs4_gemm_experts(last, want, rows[-few:].contiguous(), R.BF16, few, K, None, one_offsets, few, ref, R.BF16, M)
        assert (y[:N - few] == 0).all()                 # (the first matrix has scales of zero)
        # (both within 52 + K / 128 steps of 2^-23 of the sum of the terms' sizes, and rounded once each; a quantized weight is at most a half larger than the
        # weight, or half a step of a fifteenth of its group's range, under 0.5 for these)
        a, b = y[-few:].double(), ref.double()
        absum = rows[-few:].double().abs() @ (1.5 * sizes + 0.5).T
        assert ((a - b).abs() <= 2 * 2.0 ** -8 * torch.maximum(a.abs(), b.abs()) + 2 * (52 + K / 128) * 2.0 ** -23 * absum).all()


def test_captured_twice_and_replayed_together():
    """Two graphs of the same layer on two streams, replayed at the same time, with inputs changed in place between replays."""
    import torch
    E, T, k, M = 6, 24, 2, 192
    p = Packed(11, E, M, M, 64, R.GS4_ZERO)
    rng = np.random.default_rng(11)

    class Pass:
        def __init__(self):
            self.x = torch.empty((T, M), dtype=torch.bfloat16, device="cuda")
            self.ids = torch.empty((T, k), dtype=torch.int32, device="cuda")
            self.off, self.rows, self.place = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (E + 1, T * k, T * k))
            self.z, self.y, self.l = (torch.zeros((n, M), dtype=torch.bfloat16, device="cuda") for n in (T * k, T, T))

        def run(self, s):
            R.rmsmp_expert_sort(self.ids, T, k, E, self.off, self.rows, self.place, stream=s)
            R.rmsmp_gs4_gemm_experts(p.layer, p.packed, self.x, R.BF16, T, M, self.rows, self.off, T * k, self.z, R.BF16, M, stream=s)
            R.rmsmp_expert_combine(self.z, R.BF16, T * k, M, M, self.place, None, T, k, self.y, M, stream=s)
            R.rmsmp_gs4_gemm(q.layer, q.packed, self.y, R.BF16, T, M, self.l, R.BF16, M, stream=s)

        def fill(self):
            self.x.copy_(torch.from_numpy(rng.standard_normal((T, M)).astype(np.float32)))
            self.ids.copy_(torch.from_numpy(rng.integers(-1, E, (T, k)).astype(np.int32)))

    q = Packed(12, 1, M, M, 32, R.GS4_SYM)
    passes, graphs, streams = [Pass(), Pass()], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for one, s in zip(passes, streams):
        one.fill()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            one.run(s)
        graphs.append(g)
    for _ in range(5):
        for one in passes:
            one.fill()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        got = [one.l.clone() for one in passes]
        for one, want in zip(passes, got):
            one.l.zero_()
            one.run(torch.cuda.current_stream())
            torch.cuda.synchronize()
            assert torch.equal(one.l, want)
