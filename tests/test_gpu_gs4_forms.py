"""Group-scaled products on the GPU in every form that the launchers choose (tests/gs4_shapes.py; tests/test_gs4_plan.py says that they are all there), against
64-bit products of the same codes: bit for bit where every sum is a whole number, else within the bounds that test_gpu_gs4.py derives."""
import pytest

from paper_2111_00153_b200 import binding as R
from tests import gs4_shapes as S
from tests.test_gpu_gs4 import TINY, TYPES, half_step, td

pytestmark = pytest.mark.gpu
NAMES = {S.F32: "f32", S.F16: "f16", S.BF16: "bf16"}


def offsets_of(g, rows, E):
    """Rows spread over E matrices: some have none, one has many, and some rows at both ends belong to nobody."""
    import torch
    first, last = rows // 40, rows - rows // 25
    if E == 1:
        return torch.tensor([first, last], dtype=torch.int32, device="cuda")
    cuts = torch.randint(first, last + 1, (E - 1,), generator=g, device="cuda")
    cuts[:E // 3] = cuts[0].clone()
    ends = torch.tensor([first, last], device="cuda")
    return torch.cat([ends[:1], cuts.sort().values, ends[1:]]).int()


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("shape", S.SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_form(shape, whole):
    import torch
    rows_y, E, M, K, group, zero, x_type, experts, in_order, x_vec = shape
    name = NAMES[x_type]
    y_name = "f32" if whole else name
    g = torch.Generator(device="cuda").manual_seed(rows_y + M + K)
    draw = lambda hi, *size: torch.randint(0, hi, size, generator=g, device="cuda")
    Gn = -(-K // group)
    codes, z = draw(16, E, M, K).byte(), draw(16, E, M, Gn).byte()
    # whole: scales of one and two, activations up to four; sums stay below 2 * 15 * 4 * 96845 < 2^24
    scale = (draw(2, E, M, Gn) + 1).half() if whole else (0.02 * (0.5 + torch.rand((E, M, Gn), generator=g, device="cuda"))).half()
    layer = R.rmsmp_gs4_layer_init(E, M, K, group, R.GS4_ZERO if zero else R.GS4_SYM, R.F16)
    packed = torch.empty(layer.packed_bytes, dtype=torch.uint8, device="cuda")
    R.rmsmp_gs4_pack_codes(layer, codes, scale, z if zero else None, packed)
    x_rows = rows_y if in_order else rows_y // 2 + 1
    ld_x = (K + 7) // 8 * 8 if x_vec else K if K % 8 else K + 1
    xb = torch.full((x_rows, ld_x), float("nan"), dtype=td(name), device="cuda")
    x = xb[:, :K]
    x.copy_(draw(9, x_rows, K) - 4 if whole else torch.randn((x_rows, K), generator=g, device="cuda"))
    ld_y = M + (0 if x_vec else 3)
    yb = torch.full((rows_y + 2, ld_y), float("nan"), dtype=td(y_name), device="cuda")
    y = yb[1:-1]
    if experts:
        offsets = offsets_of(g, rows_y, E)
        index = None if in_order else draw(x_rows + 1, rows_y).int() - 1          # (-1: zeros)
        R.rmsmp_gs4_gemm_experts(layer, packed, xb, TYPES[name], x_rows, ld_x, index, offsets, rows_y, y, TYPES[y_name], ld_y)
        ends, of = offsets.tolist(), torch.arange(rows_y, device="cuda") if in_order else index.long()
    else:
        R.rmsmp_gs4_gemm(layer, packed, xb, TYPES[name], rows_y, ld_x, y, TYPES[y_name], ld_y)
        ends, of = [0, rows_y], torch.arange(rows_y, device="cuda")
    torch.cuda.synchronize()
    assert R.rmsmp_last_device_status(packed) == R.OK
    at = torch.arange(K, device="cuda") // group
    for e in range(E):
        a, b = ends[e], ends[e + 1]
        if a == b:
            continue
        inputs = torch.where((of[a:b] >= 0)[:, None], x[of[a:b].clamp(min=0)].double(), 0.0)
        w = (codes[e].double() - (z[e].double()[:, at] if zero else 8.0)) * scale[e].double()[:, at]
        want, got = inputs @ w.T, y[a:b, :M].double()
        if whole:
            assert torch.equal(got, want), (e, (got != want).nonzero()[:5].tolist())
        else:
            room = half_step(y_name) * want.abs() * (1 + 2.0 ** -10) + (48 + K / 128) * 2.0 ** -23 * (inputs.abs() @ w.abs().T) + TINY[y_name]
            assert ((got - want).abs() <= room).all(), (e, ((got - want).abs() / room).max().item())
        del w
    y[ends[0]:ends[-1], :M] = float("nan")
    assert torch.isnan(yb).all()                            # rows of nobody, and everything around, are as they were
