"""Calls of anpd_attention that take the form whose rows share keys through LDS, with rules: (heads, key / value heads, head dim, [(pos0, rows)]),
types of the rows, rules ("document": positions per document).  Numbers alone: read where there is no torch as well."""

SEVERAL = [(2000, 513), (0, 3), (2400, 777)]
WINDOWS = [{"window": 1000}, {"window": 1501}, {"window": 1500, "prefix": 700}, {"prefix": 700}]
DOCUMENTS = [{"document": 611}, {"document": 1700, "prefix": 100}, {"document": 1699, "window": 1500}, {"document": 611, "window": 2001, "prefix": 33}]

SHARED_WITH_RULES = [
    ((32, 2, 64, SEVERAL), ("bf16", "f32"), WINDOWS),
    ((32, 2, 128, SEVERAL), ("bf16", "f32"), WINDOWS),
    ((32, 4, 64, [(0, 2222)]), ("bf16", "f32"), [{"prefix": 1}, {"prefix": 1000}, {"prefix": 5000}]),
    ((48, 48, 64, [(0, 1700)]), ("bf16", "f32"), [{"window": 1201}, {"window": 1500, "prefix": 700}]),
    ((32, 32, 128, [(0, 2400)]), ("bf16", "f32"), [{"window": 2000}, {"window": 999, "prefix": 65}]),
    ((16, 1, 64, [(9000, 500)]), ("bf16", "f32"), [{"window": 8000}, {"prefix": 9300}, {"window": 7000, "prefix": 300}]),
    ((32, 2, 64, [(0, 3000)]), ("bf16",), DOCUMENTS),
    ((32, 2, 128, [(0, 3000)]), ("bf16",), DOCUMENTS),
]


def cases():
    return [(shape, q, rules) for shape, types, some in SHARED_WITH_RULES for q in types for rules in some]
