"""The linear layer by every form that its plan chooses, with the checks of tests/test_gpu_linear.py, at sizes that these leave out.  Which size takes
which form is counted, without a GPU, in tests/test_linear_forms.py."""
import pytest

import block_checks as T
import test_gpu_linear as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return T.device()


#              N, K, C
FORWARD = {"f32": [(1, 552, 1), (409, 8041, 1126),                                  # 128 x 64 tiles, parts
                   (309, 6406, 69), (955, 6807, 21), (2690, 55, 91), (4319, 17, 17)],       # few rows: 32 columns by 32 rows, in parts and whole
           "bf16": [(1510, 65, 2121), (10863, 664, 136),                            # 128 x 128 tiles, four stages
                    (653, 4226, 68), (1094, 6950, 5), (683, 42, 719), (4300, 18, 17), (1382, 222, 216), (139, 98, 4865)]}
#              B, P, K, C
BACKWARD = {"f32": [(5, 1757, 736, 62), (1143, 1, 1570, 168),                       # 256 x 128 tiles
                    (3, 91, 2706, 3989), (1, 1, 1, 546),                            # 128 x 64 tiles, parts
                    (2, 57, 163, 2883), (1, 21, 895, 2251), (4, 67, 87, 5874), (2872, 1, 19, 3038), (1, 1044, 21, 6247), (31, 163, 13, 206), (2, 2692, 83, 30)],
            "bf16": [(3, 541, 3218, 491), (2, 3174, 1263, 320),                     # 128 x 128 tiles, two workgroups a compute unit
                     (2, 214, 809, 8602), (823, 1, 1040, 2931), (1, 15478, 47, 4968),       # four stages, parts
                     (1, 164, 5163, 2887), (3, 17, 8020, 6871),                     # narrow, parts
                     (2, 5752, 27, 7210), (4, 125, 11, 8405), (3, 1267, 148, 4574), (64, 1, 4444, 9048), (7, 104, 96, 5742), (1, 17, 2048, 6910),     # few rows, parts
                     (4, 3352, 28, 6346), (13517, 1, 82, 2458), (3, 4205, 30, 12), (2183, 1, 221, 228), (2, 34, 6214, 6614), (5, 78, 1108, 5644), (2, 2744, 154, 3396),
                     (3, 141, 973, 37), (2, 73, 2805, 677)]}


@pytest.mark.parametrize("dtype,N,K,C", [(t, *q) for t, qs in FORWARD.items() for q in qs])
def test_forward(dev, dtype, N, K, C):
    L._forward(dev, N, K, C, list(T.ACTS)[(N + K + C) % 4], dtype, p=[0.25, 0.0][(N + K) % 2])


@pytest.mark.parametrize("dtype,B,P,K,C", [(t, *q) for t, qs in BACKWARD.items() for q in qs])
def test_backward(dev, dtype, B, P, K, C):
    L._backward(dev, B, P, K, C, list(T.ACTS)[(B + P + K + C) % 4], dtype, add=(P + K) % 2 == 0, p=[0.25, 0.0][(P + C) % 2])
