"""Every kernel of the products with weights in 4-bit floats: a case whose rows of x are
whole 16-byte cells and one whose rows are not, each with columns that end inside a
tile and rows that end inside a group. Sums that are exact in fp32 must be equal,
others within the bounds of the other tests of these products."""
import pytest

from test_gpu_f4 import check_gated, check_product

pytestmark = pytest.mark.gpu

PRODUCTS = [
    (1, 40, 328, "f4_matmul_few<4, 1, 1, 4, 1>"),
    (1, 40, 356, "f4_matmul_few<4, 1, 1, 4, 1>"),
    (1, 4247, 1280, "f4_matmul_few<4, 2, 1, 4, 1>"),
    (1, 4372, 1166, "f4_matmul_few<4, 2, 1, 4, 1>"),
    (5, 41, 368, "f4_matmul_few<8, 1, 1, 4, 1>"),
    (5, 43, 339, "f4_matmul_few<8, 1, 1, 4, 1>"),
    (5, 4151, 680, "f4_matmul_few<8, 2, 1, 4, 1>"),
    (5, 4250, 644, "f4_matmul_few<8, 2, 1, 4, 1>"),
    (5, 25306, 320, "f4_matmul_few<8, 2, 2, 4, 1>"),
    (5, 24905, 335, "f4_matmul_few<8, 2, 2, 4, 1>"),
    (9, 43, 304, "f4_matmul_few<16, 1, 1, 3, 1>"),
    (9, 40, 333, "f4_matmul_few<16, 1, 1, 3, 1>"),
    (9, 4394, 520, "f4_matmul_few<16, 2, 1, 3, 1>"),
    (9, 4306, 545, "f4_matmul_few<16, 2, 1, 3, 1>"),
    (9, 8214, 520, "f4_matmul_few<16, 2, 2, 4, 1>"),
    (9, 8519, 517, "f4_matmul_few<16, 2, 2, 4, 1>"),
    (9, 25838, 1032, "f4_matmul_few<16, 2, 4, 4, 1>"),
    (9, 26754, 1025, "f4_matmul_few<16, 2, 4, 4, 1>"),
    (18, 41, 352, "f4_matmul_few<32, 2, 1, 2, 1>"),
    (18, 42, 359, "f4_matmul_few<32, 2, 1, 2, 1>"),
    (18, 9083, 392, "f4_matmul_few<32, 2, 2, 3, 1>"),
    (17, 8235, 454, "f4_matmul_few<32, 2, 2, 3, 1>"),
    (18, 26292, 784, "f4_matmul_few<32, 2, 4, 3, 1>"),
    (18, 17373, 1307, "f4_matmul_few<32, 2, 4, 3, 1>"),
    (33, 41, 352, "f4_matmul_few<48, 2, 1, 2, 1>"),
    (36, 41, 309, "f4_matmul_few<48, 2, 1, 2, 1>"),
    (68, 4108, 328, "f4_matmul_few<48, 2, 2, 3, 1>"),
    (33, 8235, 303, "f4_matmul_few<48, 2, 2, 3, 1>"),
    (68, 8642, 304, "f4_matmul_few<48, 2, 3, 3, 1>"),
    (70, 8514, 301, "f4_matmul_few<48, 2, 3, 3, 1>"),
    (109, 8647, 392, "f4_matmul_few<48, 2, 4, 3, 1>"),
    (101, 8744, 398, "f4_matmul_few<48, 2, 4, 3, 1>"),
    (50, 42, 352, "f4_matmul_few<64, 2, 1, 2, 1>"),
    (50, 43, 301, "f4_matmul_few<64, 2, 1, 2, 1>"),
    (56, 8434, 312, "f4_matmul_few<64, 2, 2, 3, 1>"),
    (50, 8386, 302, "f4_matmul_few<64, 2, 2, 3, 1>"),
    (49, 32895, 320, "f4_matmul_few<64, 2, 4, 3, 1>"),
    (50, 33519, 310, "f4_matmul_few<64, 2, 4, 3, 1>"),
    (69, 77684, 312, "f4_matmul_tiled<4, 2, 4, 1, 1>"),
    (68, 74905, 353, "f4_matmul_tiled<4, 2, 4, 1, 1>"),
    (104, 44660, 448, "f4_matmul_tiled<4, 2, 4, 2, 1>"),
    (102, 49313, 388, "f4_matmul_tiled<4, 2, 4, 2, 1>")]

GATED = [
    (1, 41, 320, "f4_matmul_few<4, 2, 1, 4, 2>"),
    (1, 40, 385, "f4_matmul_few<4, 2, 1, 4, 2>"),
    (5, 40, 368, "f4_matmul_few<8, 2, 1, 4, 2>"),
    (5, 41, 313, "f4_matmul_few<8, 2, 1, 4, 2>"),
    (5, 12343, 328, "f4_matmul_few<8, 2, 2, 4, 2>"),
    (5, 12994, 330, "f4_matmul_few<8, 2, 2, 4, 2>"),
    (10, 40, 304, "f4_matmul_few<16, 2, 1, 3, 2>"),
    (9, 41, 357, "f4_matmul_few<16, 2, 1, 3, 2>"),
    (9, 4127, 744, "f4_matmul_few<16, 2, 2, 4, 2>"),
    (9, 4117, 607, "f4_matmul_few<16, 2, 2, 4, 2>"),
    (9, 12355, 1144, "f4_matmul_few<16, 2, 4, 4, 2>"),
    (9, 13001, 1050, "f4_matmul_few<16, 2, 4, 4, 2>"),
    (18, 40, 376, "f4_matmul_few<32, 2, 1, 2, 2>"),
    (19, 44, 308, "f4_matmul_few<32, 2, 1, 2, 2>"),
    (18, 4127, 464, "f4_matmul_few<32, 2, 2, 3, 2>"),
    (17, 4408, 457, "f4_matmul_few<32, 2, 2, 3, 2>"),
    (19, 12671, 840, "f4_matmul_few<32, 2, 4, 3, 2>"),
    (18, 12301, 771, "f4_matmul_few<32, 2, 4, 3, 2>"),
    (33, 40, 328, "f4_matmul_few<48, 2, 1, 2, 2>"),
    (33, 42, 338, "f4_matmul_few<48, 2, 1, 2, 2>"),
    (67, 2249, 312, "f4_matmul_few<48, 2, 2, 3, 2>"),
    (71, 2102, 330, "f4_matmul_few<48, 2, 2, 3, 2>"),
    (72, 4162, 304, "f4_matmul_few<48, 2, 3, 3, 2>"),
    (68, 4408, 307, "f4_matmul_few<48, 2, 3, 3, 2>"),
    (104, 4121, 424, "f4_matmul_few<48, 2, 4, 3, 2>"),
    (65, 6290, 421, "f4_matmul_few<48, 2, 4, 3, 2>"),
    (52, 41, 368, "f4_matmul_few<64, 2, 1, 2, 2>"),
    (50, 42, 333, "f4_matmul_few<64, 2, 1, 2, 2>"),
    (50, 4201, 376, "f4_matmul_few<64, 2, 2, 3, 2>"),
    (50, 4248, 334, "f4_matmul_few<64, 2, 2, 3, 2>"),
    (51, 17134, 328, "f4_matmul_few<64, 2, 4, 3, 2>"),
    (50, 16478, 308, "f4_matmul_few<64, 2, 4, 3, 2>"),
    (70, 39926, 304, "f4_matmul_tiled<4, 2, 4, 1, 2>"),
    (66, 37084, 305, "f4_matmul_tiled<4, 2, 4, 1, 2>"),
    (108, 22845, 400, "f4_matmul_tiled<4, 2, 4, 2, 2>"),
    (103, 22102, 406, "f4_matmul_tiled<4, 2, 4, 2, 2>")]


@pytest.mark.parametrize("m,n,k,kernel", PRODUCTS)
def test_product(m, n, k, kernel, rng):
    check_product(rng, m, n, k, "bf16", "bf16")
    check_product(rng, m, n, k, "f16", "f32")


@pytest.mark.parametrize("m,n,k,kernel", GATED)
def test_gated(m, n, k, kernel, rng):
    check_gated(rng, m, n, k, "bf16", "f32", "silu")
    check_gated(rng, m, n, k, "f16", "f16", "gelu_tanh")
