"""Sizes at which the products of the token-model operators take their larger
tiles, with what the plan has to say of them (imported by tests only)."""

# kind, type, M, N (F), K: (tile, whether in slices) of the forward product, of dx and of dw.  bf16 sizes of whole
# multiples of 8 are copied to LDS as they lie ("direct"), all others go through registers.
TILES = [
    ("linear", "bfloat16", 3603, 3640, 3592, ((256, False), (256, False), (256, False))),
    ("linear", "bfloat16", 2503, 2520, 2536, ((128, False), (128, False), (128, False))),
    ("linear", "bfloat16", 1003, 1000, 4104, ((128, True), (64, False), (64, False))),
    ("linear", "bfloat16", 4100, 1000, 1000, ((64, False), (64, False), (128, True))),
    ("linear", "bfloat16", 2503, 2519, 2531, ((128, False), (128, False), (128, False))),
    ("linear", "bfloat16", 1003, 1001, 4104, ((128, True), (64, False), (64, False))),
    ("linear", "float32", 2503, 2519, 2531, ((128, False), (128, False), (128, False))),
    ("linear", "float32", 2504, 2520, 2528, ((128, False), (128, False), (128, False))),
    ("linear", "float32", 1003, 1001, 4103, ((128, True), (64, False), (64, False))),
    ("gated", "bfloat16", 3603, 1848, 3592, ((256, False), (256, False), (256, False))),
    ("gated", "bfloat16", 2503, 1264, 2536, ((128, False), (128, False), (128, False))),
    ("gated", "bfloat16", 1003, 504, 4104, ((128, True), (64, False), (64, False))),
    ("gated", "bfloat16", 2503, 1259, 2531, ((128, False), (128, False), (128, False))),
    ("gated", "float32", 2503, 1259, 2531, ((128, False), (128, False), (128, False))),
    ("gated", "float32", 1003, 501, 4103, ((128, True), (64, False), (64, False))),
]


def direct(dtype, *cols):
    return dtype == "bfloat16" and all(c % 8 == 0 for c in cols)


def products(kind, dtype, M, N, K, activation=True):
    """The three products of a layer with its gradients as (M, N, K, fp32,
    staged, gated, terms, sets) of the plan."""
    f32, gated = dtype == "float32", kind == "gated"
    parts = 2 if not f32 and (gated or activation) else 1
    each = 2 if gated else 1
    return [(M, N, K, f32, not direct(dtype, K), gated, 1, 1),
            (M, K, N, f32, not direct(dtype, N, K), False, parts * each, 1),
            (N, K, M, f32, not direct(dtype, N, K), False, parts, each)]
