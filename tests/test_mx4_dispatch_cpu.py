"""Which kernels the 4-bit products and FFN calls of the GPU tests take, on the CPU: the tests named after a path reach it."""
import pytest

from launches import P, record
from paper_2211_10017_amd import binding as B
from test_gpu_mx4_fused import LOADS, SIZES, batch


@pytest.mark.parametrize("dtype", [B.MOE_F16, B.MOE_BF16])
def test_fc1_quantises_its_rows(dtype):
    for load, d, F in SIZES:
        _, E, _, R, T, _ = batch(load, 0)
        call = record([("moe_grouped_ffn_mx4", [P, dtype, T, P, 2, P, R, E, 0, d, F, 0, P, P, None, P, P, None, P, dtype, P, [1 << 40], None])])[0]
        assert call.rc == 0 and len(call.launches) == 2
        assert call.launches[0].kernel == "mx4_stream_kernel<%d, 1, 1, -1, %d>" % (4 if d <= 1024 else 8, dtype)
    assert {load for load, _, _ in SIZES} == set(LOADS)


def test_rows_of_four_bytes_are_quantised_before_fc1():
    call = record([("moe_grouped_ffn_mx4", [P, B.MOE_F32, 6, P, 2, P, 12, 6, 0, 192, 320, 0, P, P, None, P, P, None, P, 0, P, [1 << 40], None])])[0]
    assert [k.kernel for k in call.launches] == ["mx4_quantize_rows_kernel<2>", "mx4_stream_kernel<4, 1, 1, -1, -1>", "mx4_stream_kernel<4, 1, 1, 0, -1>"]


def test_fc1_takes_every_shape_of_block():
    from test_gpu_mx4_chain import SHAPES
    for shape, (d, F, rows, types) in SHAPES.items():
        R = sum(rows) + 3 + (sum(rows) + 3) % 2
        for t in types:
            x = {"f16": B.MOE_F16, "bf16": B.MOE_BF16, "f32": B.MOE_F32}[t]
            call = record([("moe_grouped_ffn_mx4", [P, x, R // 2, P, 2, P, R, len(rows), 0, d, F, 0, P, P, None, P, P, None, P, 0, P, [1 << 40], None])])[0]
            kernel = "mx4_tile_kernel" if shape.count(",") == 4 else "mx4_stream_kernel"
            assert call.rc == 0 and [k.kernel for k in call.launches][:2] == ["mx4_quantize_rows_kernel<%d>" % x, kernel + shape.split(" few")[0].split(" more")[0] + (
                ", -1>" if kernel == "mx4_tile_kernel" else ", -1, -1>")], (shape, t, call.launches)
