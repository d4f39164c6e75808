"""Group-scaled 4-bit layers and expert operators: what needs no GPU -- descriptions, refusals, and the oracle against its own definitions."""
import numpy as np
import pytest

from oracle import gs4_oracle as G
from paper_2111_00153_b200 import binding as R
from paper_2111_00153_b200 import build as B

BUF = 1 << 20          # an aligned address that no refused call looks at


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build_library()


def refused(status, call, *args):
    with pytest.raises(R.RmsmpError) as e:
        call(*args, stream=0)
    assert e.value.status == status, e.value


def test_layout_of_a_layer():
    for E, M, K, group, mode in [(1, 1, 1, 32, R.GS4_SYM), (1, 17, 129, 64, R.GS4_ZERO), (3, 130, 777, 128, R.GS4_ZERO), (2, 16, 128, 96, R.GS4_SYM),
                                 (1, 5, 100, 256, R.GS4_ZERO), (4096, 1, 1, 1 << 20, R.GS4_SYM), (1, 1 << 20, 1 << 20, 32, R.GS4_ZERO)]:
        L = R.rmsmp_gs4_layer_init(E, M, K, group, mode, R.F16)
        assert (L.E, L.M, L.K, L.group, L.mode, L.scale_type) == (E, M, K, group, mode, R.F16)
        assert L.Kp == (K + 127) // 128 * 128 and L.tiles == (M + 31) // 32
        assert L.sums == {0: 1, 64: 2}.get(group % 128, 4) and group % (128 // L.sums) == 0
        assert L.block_bytes % 16 == 0 and L.block_bytes == 2048 + 64 * L.sums + (16 * L.sums if mode == R.GS4_ZERO else 0)
        assert L.off_blocks % 256 == 0 and L.off_blocks >= 256 and L.packed_bytes % 256 == 0
        assert L.packed_bytes >= L.off_blocks + E * L.tiles * (L.Kp // 128) * L.block_bytes


@pytest.mark.parametrize("bad, status", [
    (dict(E=0), R.ERR_SHAPE), (dict(E=4097), R.ERR_SHAPE), (dict(M=0), R.ERR_SHAPE), (dict(M=(1 << 20) + 1), R.ERR_SHAPE),
    (dict(K=0), R.ERR_SHAPE), (dict(K=-5), R.ERR_SHAPE), (dict(group=0), R.ERR_SHAPE), (dict(group=16), R.ERR_SHAPE), (dict(group=48), R.ERR_SHAPE),
    (dict(group=(1 << 20) + 32), R.ERR_SHAPE), (dict(mode=2), R.ERR_SCHEME), (dict(mode=-1), R.ERR_SCHEME), (dict(scale_type=R.F32), R.ERR_SCHEME),
    (dict(scale_type=3), R.ERR_SCHEME)])
def test_layer_init_refuses(bad, status):
    a = dict(E=1, M=16, K=64, group=32, mode=R.GS4_SYM, scale_type=R.BF16)
    a.update(bad)
    with pytest.raises(R.RmsmpError) as e:
        R.rmsmp_gs4_layer_init(a["E"], a["M"], a["K"], a["group"], a["mode"], a["scale_type"])
    assert e.value.status == status


def test_packing_refuses():
    L = R.rmsmp_gs4_layer_init(1, 16, 64, 32, R.GS4_ZERO, R.BF16)
    n = L.packed_bytes
    refused(R.ERR_NULL, R.rmsmp_gs4_quantize_pack, L, None, R.F32, BUF, n)
    refused(R.ERR_NULL, R.rmsmp_gs4_quantize_pack, L, BUF, R.F32, None, n)
    refused(R.ERR_SCHEME, R.rmsmp_gs4_quantize_pack, L, BUF, 3, BUF, n)
    refused(R.ERR_BUFFER_TOO_SMALL, R.rmsmp_gs4_quantize_pack, L, BUF, R.F32, BUF, n - 1)
    refused(R.ERR_ALIGN, R.rmsmp_gs4_quantize_pack, L, BUF, R.F32, BUF + 128, n)
    refused(R.ERR_ALIGN, R.rmsmp_gs4_quantize_pack, L, BUF + 2, R.F32, BUF, n)
    refused(R.ERR_NULL, R.rmsmp_gs4_pack_codes, L, BUF, None, BUF, BUF, n)
    refused(R.ERR_NULL, R.rmsmp_gs4_pack_codes, L, BUF, BUF, None, BUF, n)
    refused(R.ERR_BUFFER_TOO_SMALL, R.rmsmp_gs4_pack_codes, L, BUF, BUF, BUF, BUF, 0)
    refused(R.ERR_ALIGN, R.rmsmp_gs4_pack_codes, L, BUF, BUF + 1, BUF, BUF, n)
    refused(R.ERR_NULL, R.rmsmp_gs4_unpack, L, BUF, None)
    for field, value in (("magic", 1), ("Kp", 256), ("tiles", 2), ("sums", 1), ("off_blocks", 1 << 40), ("block_bytes", 16), ("packed_bytes", 0), ("M", 33), ("mode", 5)):
        bad = R.rmsmp_gs4_layer.from_buffer_copy(L)
        setattr(bad, field, value)
        refused(R.ERR_BAD_LAYER, R.rmsmp_gs4_quantize_pack, bad, BUF, R.F32, BUF, 1 << 30)
        refused(R.ERR_BAD_LAYER, R.rmsmp_gs4_unpack, bad, BUF, BUF)
        refused(R.ERR_BAD_LAYER, R.rmsmp_gs4_gemm, bad, BUF, BUF, R.F32, 1, 64, BUF, R.F32, 32)


def test_products_refuse():
    L = R.rmsmp_gs4_layer_init(1, 16, 64, 32)
    L3 = R.rmsmp_gs4_layer_init(3, 16, 64, 32)
    g = R.rmsmp_gs4_gemm
    refused(R.ERR_NULL, g, L, None, BUF, R.F32, 1, 64, BUF, R.F32, 16)
    refused(R.ERR_NULL, g, L, BUF, None, R.F32, 1, 64, BUF, R.F32, 16)
    refused(R.ERR_NULL, g, L, BUF, BUF, R.F32, 1, 64, None, R.F32, 16)
    refused(R.ERR_SHAPE, g, L3, BUF, BUF, R.F32, 1, 64, BUF, R.F32, 16)            # experts need their own call
    refused(R.ERR_SHAPE, g, L, BUF, BUF, R.F32, -1, 64, BUF, R.F32, 16)
    refused(R.ERR_SHAPE, g, L, BUF, BUF, R.F32, (1 << 30) + 1, 64, BUF, R.F32, 16)
    refused(R.ERR_SHAPE, g, L, BUF, BUF, R.F32, 1, 63, BUF, R.F32, 16)
    refused(R.ERR_SHAPE, g, L, BUF, BUF, R.F32, 1, 64, BUF, R.F32, 15)
    refused(R.ERR_SCHEME, g, L, BUF, BUF, 3, 1, 64, BUF, R.F32, 16)
    refused(R.ERR_SCHEME, g, L, BUF, BUF, R.F32, 1, 64, BUF, -1, 16)
    refused(R.ERR_ALIGN, g, L, BUF + 16, BUF, R.F32, 1, 64, BUF, R.F32, 16)
    refused(R.ERR_ALIGN, g, L, BUF, BUF + 2, R.F32, 1, 64, BUF, R.F32, 16)
    refused(R.ERR_ALIGN, g, L, BUF, BUF, R.F32, 1, 64, BUF + 1, R.BF16, 16)
    x = R.rmsmp_gs4_gemm_experts
    refused(R.ERR_NULL, x, L3, BUF, BUF, R.F16, 4, 64, BUF, None, 8, BUF, R.F16, 16)
    refused(R.ERR_SHAPE, x, L3, BUF, BUF, R.F16, -1, 64, BUF, BUF, 8, BUF, R.F16, 16)
    refused(R.ERR_SHAPE, x, L3, BUF, BUF, R.F16, 4, 64, BUF, BUF, -8, BUF, R.F16, 16)
    refused(R.ERR_ALIGN, x, L3, BUF, BUF, R.F16, 4, 64, BUF + 2, BUF, 8, BUF, R.F16, 16)
    refused(R.ERR_ALIGN, x, L3, BUF, BUF, R.F16, 4, 64, BUF, BUF + 1, 8, BUF, R.F16, 16)


def test_expert_calls_refuse():
    s = R.rmsmp_expert_sort
    refused(R.ERR_NULL, s, None, 4, 2, 8, BUF, BUF, BUF)
    refused(R.ERR_NULL, s, BUF, 4, 2, 8, None, BUF, BUF)
    for T, k, E in ((-1, 2, 8), (4, 0, 8), (4, 1025, 8), (4, 2, 0), (4, 2, 1025), (1 << 30, 2, 8)):
        refused(R.ERR_SHAPE, s, BUF, T, k, E, BUF, BUF, BUF)
    refused(R.ERR_ALIGN, s, BUF + 2, 4, 2, 8, BUF, BUF, BUF)
    g = R.rmsmp_expert_gather
    refused(R.ERR_NULL, g, None, R.F32, 4, 8, 8, BUF, 8, BUF, 8)
    refused(R.ERR_SCHEME, g, BUF, 7, 4, 8, 8, BUF, 8, BUF, 8)
    refused(R.ERR_SHAPE, g, BUF, R.F32, 4, 0, 8, BUF, 8, BUF, 8)
    refused(R.ERR_SHAPE, g, BUF, R.F32, 4, 8, 7, BUF, 8, BUF, 8)
    refused(R.ERR_SHAPE, g, BUF, R.F32, 4, 8, 8, BUF, 8, BUF, 7)
    refused(R.ERR_ALIGN, g, BUF + 2, R.F32, 4, 8, 8, BUF, 8, BUF, 8)
    c = R.rmsmp_expert_combine
    refused(R.ERR_NULL, c, BUF, R.F32, 8, 8, 8, None, BUF, 4, 2, BUF, 8)
    refused(R.ERR_SHAPE, c, BUF, R.F32, 8, 8, 8, BUF, BUF, 4, 0, BUF, 8)
    refused(R.ERR_SHAPE, c, BUF, R.F32, 8, 8, 8, BUF, BUF, -4, 2, BUF, 8)
    refused(R.ERR_ALIGN, c, BUF, R.F32, 8, 8, 8, BUF, BUF + 2, 4, 2, BUF, 8)
    b = R.rmsmp_expert_combine_backward
    refused(R.ERR_NULL, b, BUF, R.F32, 4, 2, 8, 8, BUF, 8, 8, BUF, BUF, None, 8, None)
    refused(R.ERR_NULL, b, BUF, R.F32, 4, 2, 8, 8, None, 8, 8, BUF, BUF, BUF, 8, BUF)
    refused(R.ERR_SHAPE, b, BUF, R.F32, 4, 2, 8, 8, BUF, 8, 7, BUF, BUF, BUF, 8, BUF)
    refused(R.ERR_SHAPE, b, BUF, R.F32, 4, 2, 8, 7, BUF, 8, 8, BUF, BUF, BUF, 8, BUF)
    refused(R.ERR_ALIGN, b, BUF, R.F32, 4, 2, 8, 8, BUF, 8, 8, BUF, BUF, BUF, 8, BUF + 1)


def test_host_tensors_and_other_element_sizes_are_refused_before_the_call():
    torch = pytest.importorskip("torch")
    L = R.rmsmp_gs4_layer_init(1, 16, 64, 32)
    x = torch.zeros(64)
    with pytest.raises(ValueError, match="CUDA"):
        R.rmsmp_gs4_gemm(L, BUF, x, R.F32, 1, 64, BUF, R.F32, 16, stream=0)
    with pytest.raises(ValueError, match="elements"):

        class Ids:                                  # as torch.topk gives them
            def get_device(self): return 0
            def element_size(self): return 8
            def data_ptr(self): return BUF
        R.rmsmp_expert_sort(Ids(), 4, 2, 8, BUF, BUF, BUF, stream=0)


class Fake:
    """A tensor as the binding sees one: on the first device, elements of `size` bytes, an address that no refused call looks at."""

    def __init__(self, size):
        self.size = size

    def get_device(self): return 0
    def element_size(self): return self.size
    def numel(self): return 1 << 20
    def data_ptr(self): return BUF


# every argument whose type is a code beside it: (call, arguments with `x` in its place and `t` in the code's; `bad`: a size that the library refuses)
TYPED = [
    ("rmsmp_gs4_quantize_pack", lambda L, x, t, bad: (L, x, t, BUF, 0 if bad else L.packed_bytes)),
    ("rmsmp_gs4_gemm", lambda L, x, t, bad: (L, BUF, x, t, -1 if bad else 1, 64, BUF, R.F32, 16)),
    ("rmsmp_gs4_gemm", lambda L, x, t, bad: (L, BUF, BUF, R.F32, -1 if bad else 1, 64, x, t, 16)),
    ("rmsmp_gs4_gemm_experts", lambda L, x, t, bad: (L, BUF, x, t, 4, 64, BUF, BUF, -1 if bad else 4, BUF, R.F32, 16)),
    ("rmsmp_gs4_gemm_experts", lambda L, x, t, bad: (L, BUF, BUF, R.F32, 4, 64, BUF, BUF, -1 if bad else 4, x, t, 16)),
    ("rmsmp_expert_gather", lambda L, x, t, bad: (x, t, 4, 0 if bad else 8, 8, BUF, 4, BUF, 8)),
    ("rmsmp_expert_gather", lambda L, x, t, bad: (BUF, t, 4, 0 if bad else 8, 8, BUF, 4, x, 8)),
    ("rmsmp_expert_combine", lambda L, x, t, bad: (x, t, 4, 0 if bad else 8, 8, BUF, BUF, 2, 2, BUF, 8)),
    ("rmsmp_expert_combine", lambda L, x, t, bad: (BUF, t, 4, 0 if bad else 8, 8, BUF, BUF, 2, 2, x, 8)),
    ("rmsmp_expert_combine_backward", lambda L, x, t, bad: (x, t, 2, 2, 0 if bad else 8, 8, BUF, 4, 8, BUF, BUF, BUF, 8, BUF)),
    ("rmsmp_expert_combine_backward", lambda L, x, t, bad: (BUF, t, 2, 2, 0 if bad else 8, 8, x, 4, 8, BUF, BUF, BUF, 8, BUF)),
    ("rmsmp_expert_combine_backward", lambda L, x, t, bad: (BUF, t, 2, 2, 0 if bad else 8, 8, BUF, 4, 8, BUF, BUF, x, 8, BUF)),
]


@pytest.mark.parametrize("name, args", TYPED, ids=["%s-%d" % (n, i) for i, (n, _) in enumerate(TYPED)])
@pytest.mark.parametrize("t, size", [(R.F32, 4), (R.F16, 2), (R.BF16, 2)])
def test_elements_of_another_size_than_their_type_are_refused(name, args, t, size):
    """A bf16 tensor given as F32 would be read past its end.  (Nothing is launched: every call here is refused, the right size by the library.)"""
    L = R.rmsmp_gs4_layer_init(1, 16, 64, 32)
    call = getattr(R, name)
    for other in (1, 2, 4, 8):
        if other == size:
            with pytest.raises(R.RmsmpError) as e:
                call(*args(L, Fake(size), t, True), stream=0)
            assert e.value.status in (R.ERR_SHAPE, R.ERR_BUFFER_TOO_SMALL)
        else:
            with pytest.raises(ValueError, match="elements"):
                call(*args(L, Fake(other), t, True), stream=0)
    with pytest.raises(R.RmsmpError):                   # a code that is no type is the library's to refuse
        call(*args(L, Fake(4), 7, True), stream=0)


# ------------------------------------------------------------------ the oracle itself

@pytest.mark.parametrize("mode", [G.SYM, G.ZERO])
@pytest.mark.parametrize("scale_type", ["f16", "bf16"])
def test_quantizer_is_nearest(mode, scale_type):
    rng = np.random.default_rng(1)
    W = (rng.standard_normal((5, 100)) * 0.02).astype(np.float32)
    W[2, :64] = 0
    codes, scale, zero = G.quantize(W, 32, mode, scale_type)
    w = G.weights(codes, scale, zero, 32)
    at = np.arange(100) // 32
    s, z = scale.astype(np.float64)[:, at], zero.astype(np.float64)[:, at]
    lo, hi = (1, 15) if mode == G.SYM else (0, 15)
    levels = np.arange(lo, hi + 1)
    best = np.abs((levels[None, None] - z[..., None]) * s[..., None] - W.astype(np.float64)[..., None]).min(-1)
    assert np.all(np.abs(w - W) <= best * (1 + 1e-5) + 1e-12)          # (the fp32 quotient can fall on the other side of a tie)
    assert np.all(w[2, :64] == 0)


def test_combine_gradient_against_differences():
    rng = np.random.default_rng(2)
    T, k, E, H = 5, 3, 4, 7
    ids = rng.integers(-1, E, (T, k)).astype(np.int32)
    _, _, place = G.sort_pairs(ids, E)
    ys, w, dy = rng.standard_normal((T * k, H)), rng.standard_normal((T, k)), rng.standard_normal((T, H))
    dys, dw, _ = G.combine_backward(dy, ys, place, w)
    loss = lambda a, b: float((G.combine(a, place, b)[0] * dy).sum())
    for idx in np.ndindex(*ys.shape):
        d = np.zeros_like(ys)
        d[idx] = 0.5
        num = loss(ys + d, w) - loss(ys - d, w)                          # linear: exact up to rounding
        assert abs(num - (0.0 if np.isnan(dys[idx]) else dys[idx])) < 1e-12
    for idx in np.ndindex(T, k):
        d = np.zeros((T, k))
        d[idx] = 0.5
        assert abs(loss(ys, w + d) - loss(ys, w - d) - dw[idx]) < 1e-12
