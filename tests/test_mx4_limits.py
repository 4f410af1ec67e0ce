"""Largest sizes of the microscaled 4-bit calls, from the launches that they are made of (argument checks, no device needed)."""
from paper_2603_19172_amd import binding as B

lib = B.lib
P = 0x10000  # a non-null, aligned dummy "pointer"; never dereferenced by validation

def matmul(T, N, K=64, coded=False):
    Kp = -(-K // 256) * 256
    return lib.dymoe_matmul_mx4(None, P, 4 if coded else 0, P, Kp if coded else K, P, P, None, T, N, K, 0, P, N, P, 1 << 60, None)


def test_products_of_as_many_tiles_as_a_launch_takes():
    """2^24 - 64 workgroups of 256 threads, one for each tile of 128 x 256."""
    for T, N in ((65536, 131072), (32768, 262144), (1 << 24, 4096), (128, 1 << 24), (1, 1 << 24), (32, 1 << 24), (33, 1 << 24), (32641, (1 << 24) - 256 * 255)):
        assert matmul(T, N) == matmul(T, N, coded=True) == B.ENOCTX, (T, N)
    # 255 x 65792 tiles is 2^24 - 256, 256 x 65536 2^24
    for T, N in ((32641, 1 << 24), (1 << 20, 1 << 20), (1 << 24, 1 << 24), (1 << 24, 32768)):
        assert matmul(T, N) == matmul(T, N, coded=True) == B.ENOTSUP, (T, N)


def experts(T, H, F, E, k):
    return lib.dymoe_moe_ffn_mx4(None, P, 0, P, P, P, T, H, F, E, k, 0, P, P, 1 << 60, None)


def test_experts_of_as_many_tiles_as_a_launch_takes():
    for size in ((131072, 4096, 14336, 8, 8), (66000, 32, 131072, 4, 1), (1 << 21, 1024, 3000, 8, 8), (1 << 22, 256, 3000, 1, 1), (32, 131072, 131072, 1024, 1024),
                 (20, 131072, 131072, 1024, 1024)):
        assert experts(*size) == B.ENOCTX, size
    # pairs / 128 + experts, times blocks of 128 of F up to a multiple of 256: 2^24 - 64 groups at most
    for size, want in (((((1 << 14) - 2) * 128, 256, 131072, 1, 1), B.ENOCTX), (((1 << 14) * 128, 256, 131072, 1, 1), B.ENOTSUP),
                       ((1 << 23, 256, 32768, 1, 1), B.ENOTSUP), ((1 << 24, 512, 256, 1, 1), B.ENOTSUP)):
        assert experts(*size) == want, size
