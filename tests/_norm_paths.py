"""Shapes that take the group norm's kernels one by one: for each way a slab can
be kept, each width of a vector, each number of groups among a thread's channels
and each pair of types.  test_group_norm_plan.py holds the plans to the ways
named here, test_gpu_group_norm_paths.py runs the shapes."""
TYPES = [("f", "f"), ("f", "b"), ("b", "f"), ("b", "b")]

# (vector, groups among its channels) -> channels, groups
FORWARD_GROUPS = {(1, 1): (33, 11), (4, 1): (64, 8), (4, 2): (64, 32), (4, 4): (60, 20), (8, 1): (64, 8), (8, 2): (64, 16),
                  (8, 4): (64, 32)}
# images, pixels: few enough to stay in shared memory; more than the SMs hold at a time, of at most and of more pixels
# than a block's registers take, the latter by single blocks and by clusters; images that clusters cannot take alone.
# Every thread count of pixels ends inside a batch of loads.
FORWARD_SIZES = {"shared": (5, 231), "held": (470, 111), "reread": (630, 283), "reread_cluster": (231, 851),
                 "chunks": (3, 20011)}
FORWARD_SINGLE = {"held": (470, 111), "reread": (630, 231), "reread_cluster": (130, 801), "chunks": (3, 20011)}

BACKWARD_GROUPS = {1: [(33, 11)], 4: [(64, 8), (60, 20)], 8: [(64, 8), (64, 32)]}
BACKWARD_SIZES = {"shared": (5, 231), "held": (310, 111), "reread": (470, 283), "reread_cluster": (70, 1301),
                  "stream": (3, 20011)}
BACKWARD_SINGLE = {"held": (310, 111), "reread": (310, 231), "reread_cluster": (130, 801), "stream": (3, 20011)}


def forward_cases():
    """[(case of test_gpu_group_norm, way, vector, groups among its channels)]"""
    out = []
    for tx, ty in TYPES:
        for k, ((V, GPT), (C, G)) in enumerate(FORWARD_GROUPS.items()):
            # eight values a vector are bf16 on both sides, where four are what rows of 8-byte multiples get
            if V == 8 and (tx, ty) != ("b", "b"):
                continue
            ld = C + 4 if V == 4 and (tx, ty) == ("b", "b") else C
            for j, (way, (B, P)) in enumerate((FORWARD_SINGLE if V == 1 else FORWARD_SIZES).items()):
                out.append(((B, P, C, G, ld, 0, tx, ty, (j + k) % 4), way, V, GPT))
    # groups too wide for a block's lanes
    for tx, ty, C, V in [("f", "f", 4104, 4), ("b", "b", 4104, 8), ("f", "b", 2051, 1)]:
        out.append(((3, 130, C, 1, C, 0, tx, ty, 3), "stream", V, None))
    return out


def backward_cases():
    """The same; the vector alone."""
    out = []
    for tx, td in TYPES:
        for V, groups in BACKWARD_GROUPS.items():
            if V == 8 and (tx, td) != ("b", "b"):
                continue
            for k, (C, G) in enumerate(groups):
                ld = C + 4 if V == 4 and (tx, td) == ("b", "b") else C
                for j, (way, (B, P)) in enumerate((BACKWARD_SINGLE if V == 1 else BACKWARD_SIZES).items()):
                    out.append(((B, P, C, G, ld, 0, tx, td, (j + 2 * k) % 4), way, V))
    return out
