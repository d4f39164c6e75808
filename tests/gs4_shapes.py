"""Shapes of group-scaled products that between them take every form the launchers choose, for the tests of that choice and of the results."""
import itertools
import math

F32, F16, BF16 = 0, 1, 2

FEW = ("nt", "wr", "wk", "split", "per", "groups", "slice", "slab", "alone", "single", "tokens", "parts", "smem", "grid")
MANY = ("bn", "split", "units", "mtiles", "ntiles")

# rows of y, matrices, rows and inputs of each, group, zero points, type of x, by expert, rows in order, rows of x on 16 bytes
SHAPES = [
    # few tokens
    (8, 1, 8192, 8192, 128, 1, F16, 0, 1, 1),
    (1, 1, 65536, 4096, 128, 0, BF16, 0, 1, 1),
    (256, 64, 1408, 2048, 128, 0, BF16, 1, 0, 1),
    (1024, 64, 1408, 2048, 128, 1, BF16, 1, 0, 1),
    (32, 8, 4096, 4096, 64, 0, BF16, 1, 1, 1),
    (5, 1, 42, 1156, 256, 0, F32, 1, 0, 1),
    (325, 17, 38, 837, 256, 1, F16, 1, 1, 0),
    (1, 1, 34, 74180, 32, 0, F32, 1, 0, 1),
    (3, 1, 84891, 135, 256, 0, F32, 0, 1, 0),
    (8, 1, 1028, 1200, 256, 1, BF16, 0, 1, 0),
    (30, 2, 44, 96845, 256, 1, F16, 1, 1, 0),
    (76, 10, 58, 1187, 96, 1, F16, 1, 1, 0),
    (268, 50, 44, 12411, 256, 0, F32, 1, 0, 0),
    (185, 51, 66, 2496, 128, 1, F32, 1, 1, 1),
    (7, 1, 46, 91808, 96, 0, BF16, 0, 1, 1),
    (1769, 105, 70, 6214, 64, 1, F16, 1, 1, 1),
    (78, 4, 2368, 1122, 96, 1, F16, 1, 1, 1),
    (6, 8, 138, 77146, 32, 1, BF16, 1, 1, 0),
    (1, 1, 6489, 18176, 32, 1, F16, 0, 1, 1),
    (121, 70, 75, 39176, 32, 0, F32, 1, 0, 1),
    (3, 1, 9983, 2652, 256, 1, F32, 0, 1, 1),
    (4, 1, 19428, 2506, 256, 1, F32, 0, 1, 1),
    (730, 111, 34, 12356, 64, 0, F32, 1, 0, 1),
    (2, 1, 33, 136, 32, 1, F32, 0, 1, 1),
    (85, 12, 269, 23217, 256, 0, F32, 1, 1, 1),
    (1957, 171, 138, 150, 128, 1, F16, 1, 1, 1),
    (73, 38, 927, 136, 256, 0, F16, 1, 0, 0),
    (156, 17, 2233, 137, 256, 1, F32, 1, 1, 0),
    (3, 1, 4220, 56146, 64, 1, F32, 0, 1, 0),
    (81, 52, 132, 44206, 96, 0, F16, 1, 0, 1),
    (6, 1, 34, 131, 64, 0, F32, 0, 1, 1),
    # many
    (2419, 5, 35, 135, 32, 0, BF16, 1, 1, 0),
    (1669, 1, 44, 395, 256, 1, F16, 0, 1, 1),
    (89, 1, 44, 12401, 256, 0, BF16, 1, 0, 1),
    (671, 1, 34, 8673, 32, 1, F32, 0, 1, 0),
    (3666, 2, 353, 165, 64, 1, F16, 1, 1, 1),
    (3070, 11, 293, 414, 32, 1, F16, 1, 0, 0),
    (3546, 1, 580, 390, 96, 0, BF16, 0, 1, 1),
    (1779, 5, 278, 148, 32, 1, F32, 1, 1, 1),
    (2972, 1, 42, 709, 64, 1, BF16, 0, 1, 0),
    (2109, 1, 1213, 141, 128, 0, BF16, 0, 1, 1),
    (2531, 1, 37, 5960, 256, 1, F32, 0, 1, 0),
    (1368, 1, 540, 410, 256, 1, F16, 1, 0, 1),
    (16, 1, 40, 12135, 64, 0, F16, 0, 1, 1),
    (27, 1, 5255, 476, 256, 0, F16, 0, 1, 1),
    (19, 1, 33, 175, 96, 1, BF16, 0, 1, 0),
    (3313, 2, 138, 486, 64, 0, F16, 1, 0, 1),
    (3834, 55, 56, 489, 128, 1, F16, 1, 0, 1),
    (803, 1, 3874, 144, 64, 1, BF16, 0, 1, 0),
    (1347, 1, 37, 211, 64, 0, F32, 0, 1, 1),
    (2228, 2, 46, 401, 64, 1, BF16, 1, 1, 0),
    (1789, 21, 392, 2284, 96, 1, F16, 1, 1, 1),
    (2665, 1, 148, 9539, 256, 0, BF16, 0, 1, 1),
    (1959, 1, 785, 4165, 32, 0, F16, 0, 1, 1),
]


def features(kind, plan, shape):
    """What a form is made of: every pair of these that shapes have is to be tested."""
    R, E, M, K, group, zero, x_type, experts, in_order, x_vec = shape
    if kind == "few":
        ranks = -(-(-(-K // 128) * 128) // plan["slice"])
        return ["%s of %d columns" % ("experts" if experts else "dense", 8 * plan["nt"]), "x%d" % x_type, "wr%d" % plan["wr"], "split%d" % plan["split"],
                "rounds" if plan["per"] > plan["wr"] else "one round", "single" if plan["single"] else "alone" if plan["alone"] else "shared",
                "stages%d" % min(3, -(-plan["slice"] // plan["slab"])), "an idle rank" if ranks < plan["split"] else "all ranks"]
    how = "tensor copies" if in_order and x_vec and x_type != F32 else "16 bytes" if x_vec else "single values"
    return ["experts" if experts else "dense", "x%d" % x_type, "tiles of %d" % plan["bn"], "split%d" % plan["split"], how, "long" if plan["units"] > 16 else "short",
            "%d runs" % (1 if group % 128 == 0 else 2 if group % 64 == 0 else 4)]


def pairs(kind, features):
    return {(kind,) + c for c in itertools.combinations(sorted(features), 2)}


def any_shape(rng):
    """A shape of the whole range, small enough for a test."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    while True:
        experts = rng.random() < 0.5
        M, K = log(33, 100000), log(130, 100000 if rng.random() < 0.4 else 8192)
        E = log(1, 200) if experts else 1
        if rng.random() < 0.4:
            R = log(1, 4000) if experts else log(9, 4000)
        else:
            R = log(1, 24 * E) if experts else log(1, 8)
        x_vec = rng.random() < 0.5
        if E * M * K <= 4e8 and R * M * K <= 4e10 and R * max(M, K) <= 4e7:
            return (R, E, M, K, rng.choice([32, 64, 96, 128, 256]), int(rng.random() < 0.5), rng.choice([F32, F16, BF16]), int(experts),
                    int(not experts or rng.random() < 0.5), int(x_vec))
