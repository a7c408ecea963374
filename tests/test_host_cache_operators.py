"""The operators on caches on the stand-in for the HIP runtime: what they refuse (before anything is launched), which memory they ask
for, whose device they run on, and what a failed launch leaves behind."""
import ctypes as C
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
from test_host_path import stub  # noqa: E402,F401

DEVICES = r"""
// the current device, for the stand-in
extern "C" {
static int g_device = 0, g_set = 0;
int hipGetDevice(int *d) { *d = g_device; return 0; }
int hipSetDevice(int d) { g_device = d; ++g_set; return 0; }
int stub_device_switches(void) { return g_set; }
}
"""


def run(stub, name, *args, tmp=None):
    env = dict(os.environ, ANPD_HIP_STUB=stub, PYTHONPATH=os.path.dirname(HERE))
    if tmp is not None:
        (tmp / "devices.cpp").write_text(DEVICES)
        subprocess.run(["g++", "-O1", "-fPIC", "-shared", str(tmp / "devices.cpp"), "-o", str(tmp / "devices.so")], check=True)
        env["ANPD_DEVICES_STUB"] = str(tmp / "devices.so")
    r = subprocess.run([sys.executable, os.path.abspath(__file__), name, *map(str, args)], capture_output=True, text=True, timeout=120, env=env)
    assert r.returncode == 0, r.stdout + r.stderr


# ------------------------------------------------------------------------------------------- in the child

class Caches:
    def __init__(self):
        sys.modules["torch"] = None           # (it would bring a HIP runtime of its own)
        if "ANPD_DEVICES_STUB" in os.environ:
            self.devices = C.CDLL(os.environ["ANPD_DEVICES_STUB"], mode=C.RTLD_GLOBAL)
        self.stub = C.CDLL(os.environ["ANPD_HIP_STUB"], mode=C.RTLD_GLOBAL)
        self.stub.stub_name.restype = C.c_char_p
        self.stub.stub_memory.argtypes = [C.c_void_p, C.c_size_t, C.c_int]
        from paper_2404_08698_amd import binding as B
        self.B, self.L, self.keep = B, B.lib(), []

    def memory(self, n, device=0):
        buf = C.create_string_buffer(n + 512)
        self.keep.append(buf)
        at = (C.addressof(buf) + 255) // 256 * 256
        self.stub.stub_memory(at, n, device)
        return at

    def cache(self, max_tokens, length=0, heads=4, kv_heads=2, dim=64, layers=2, dtype=1, page=16, device=0):
        cfg = self.B.CacheCfg(layers, heads, dim, kv_heads, dtype, page)
        n = self.L.anpd_cache_pool_bytes(C.byref(cfg), max_tokens)
        assert n > 0, self.L.anpd_last_error()
        kv, pool = C.c_void_p(), self.memory(n, device)
        assert self.L.anpd_cache_create(C.byref(cfg), pool, n, max_tokens, C.byref(kv)) == 0
        assert self.L.anpd_kv_truncate(kv, length, None) == 0
        return kv

    def names(self):
        return [self.stub.stub_name(i).decode() for i in range(self.stub.stub_launches())]

    def attention(self, kvs, rows, pos0=None, layer=0, q=None, ldq=256, dtype=1, rules=None, out=None, ldo=256, lse=None, ws=None, nb=0, n=None):
        q = self.memory(1 << 16) if q is None else q
        out = self.memory(1 << 16) if out is None else out
        return self.L.anpd_attention((C.c_void_p * max(1, len(kvs)))(*kvs), len(kvs) if n is None else n, (C.c_int32 * max(1, len(rows)))(*rows),
                                     None if pos0 is None else (C.c_int32 * len(pos0))(*pos0), layer, q, ldq, dtype,
                                     None if rules is None else C.addressof(rules), out, ldo, lse, ws, nb, None)

    def mass(self, kvs, rows, masses, pos0=None, ld=512, layer=0, q=None, lse=None, dtype=1, ldq=256, ws=None, nb=0):
        return self.L.anpd_key_mass((C.c_void_p * len(kvs))(*kvs), len(kvs), (C.c_int32 * len(rows))(*rows),
                                    None if pos0 is None else (C.c_int32 * len(pos0))(*pos0), layer, self.memory(1 << 16) if q is None else q, ldq, dtype, None,
                                    self.memory(1 << 12) if lse is None else lse, (C.c_void_p * len(masses))(*masses), ld, ws, nb, None)

    def evict(self, src, dst, keep, first=0, last=0, rope=0.0, mass=1, ld=512, kept=1, out=None, ld_out=512):
        mass = self.memory(1 << 16) if mass == 1 else mass
        kept = self.memory(1 << 16) if kept == 1 else kept
        return self.L.anpd_kv_evict(src, dst, mass, ld, keep, first, last, rope, kept, out, ld_out, None)


def child_refusals():
    c = Caches()
    B, E = c.B, c.B
    kv, other, wide = c.cache(300, 100), c.cache(300, 40), c.cache(300, 100, heads=8)
    plain, layers, far = c.cache(300, 100, dtype=0), c.cache(300, 100, layers=3), c.cache(300, 100, page=8)
    c.stub.stub_forget()

    def refused(code, rc, word=None):
        assert rc == code, (rc, c.L.anpd_last_error())
        if word:
            assert word in c.L.anpd_last_error().decode(), c.L.anpd_last_error()
        assert c.names() == []

    A = c.attention
    refused(E.E_INVAL, A([kv], [1], n=0), "n_seq")
    refused(E.E_INVAL, A([kv] * 65, [1] * 65), "n_seq")
    refused(E.E_INVAL, A([kv, None], [1, 1], pos0=[5, 5]), "NULL cache")
    for bad in (wide, plain, layers, far):
        refused(E.E_INVAL, A([kv, bad], [1, 1], pos0=[5, 5]), "shape")
    refused(E.E_INVAL, A([kv], [-1], pos0=[5]))
    refused(E.E_INVAL, A([kv], [1], pos0=[-1]))
    refused(E.E_CAPACITY, A([kv], [2], pos0=[299]), "capacity")
    refused(E.E_CAPACITY, A([kv], [2147483647], pos0=[2147483647]), "capacity")
    refused(E.E_INVAL, A([kv], [50], pos0=[70]), "no page")       # 100 positions: pages up to 111
    refused(E.E_INVAL, A([kv, other], [1, 10], pos0=[99, 39]), "no page")
    refused(E.E_INVAL, A([kv], [1], pos0=[5], layer=2), "layer")
    refused(E.E_INVAL, A([kv], [1], pos0=[5], layer=-1), "layer")
    refused(E.E_INVAL, A([kv], [1], pos0=[5], dtype=2), "dtype")
    refused(E.E_INVAL, A([kv], [1], pos0=[5], ldq=255))
    refused(E.E_INVAL, A([kv], [1], pos0=[5], ldo=255), "ldo")
    m = c.memory(4096)
    refused(E.E_INVAL, A([kv], [1], pos0=[5], q=m + 1), "aligned")
    refused(E.E_INVAL, A([kv], [1], pos0=[5], out=m + 1), "aligned")
    refused(E.E_INVAL, A([kv], [1], pos0=[5], q=m + 2, dtype=0), "aligned")
    inf, nan = float("inf"), float("nan")
    for scale, cap, window, prefix in ((-1.0, 0, 0, 0), (inf, 0, 0, 0), (nan, 0, 0, 0), (0, -1.0, 0, 0), (0, inf, 0, 0), (0, nan, 0, 0), (0, 0, -1, 0), (0, 0, 0, -1)):
        refused(E.E_INVAL, A([kv], [1], pos0=[5], rules=B.AttnRules(scale, cap, window, prefix)), "finite")
    for cap, scale in ((1e-45, 0), (3e38, 0), (1e30, 1e-20), (1e-30, 1e20)):
        refused(E.E_INVAL, A([kv], [1], pos0=[5], rules=B.AttnRules(scale, cap)), "range")
    for rules in (B.AttnRules(slopes=m + 2), B.AttnRules(first_key=m + 1)):
        refused(E.E_INVAL, A([kv], [1], pos0=[5], rules=rules), "aligned")
    refused(E.E_INVAL, A([kv], [1], pos0=[5], lse=m + 2), "aligned")
    for args in (([kv], None), (None, [1])):
        kvs = None if args[0] is None else (C.c_void_p * 1)(*args[0])
        rows = None if args[1] is None else (C.c_int32 * 1)(*args[1])
        refused(E.E_INVAL, c.L.anpd_attention(kvs, 1, rows, None, 0, m, 256, 1, None, m, 256, None, None, 0, None), "NULL")
        assert c.L.anpd_attention_workspace_bytes(kvs, 1, rows, None, None) == 0
    one = (C.c_void_p * 1)(kv)
    refused(E.E_INVAL, c.L.anpd_attention(one, 1, (C.c_int32 * 1)(1), (C.c_int32 * 1)(5), 0, None, 256, 1, None, m, 256, None, None, 0, None), "NULL")
    refused(E.E_INVAL, c.L.anpd_attention(one, 1, (C.c_int32 * 1)(1), (C.c_int32 * 1)(5), 0, m, 256, 1, None, None, 256, None, None, 0, None), "NULL")
    # nothing to do is no error, and launches nothing
    refused(0, c.L.anpd_attention(one, 1, (C.c_int32 * 1)(0), None, 0, None, 256, 1, None, None, 256, None, None, 0, None))

    M = c.mass
    a = c.memory(1 << 16)
    refused(E.E_INVAL, M([kv], [1], [None], pos0=[5]), "NULL mass")
    refused(E.E_CAPACITY, M([kv], [1], [a], pos0=[5], ld=5), "ld_mass")
    refused(E.E_INVAL, M([kv, other], [1, 1], [a, a], pos0=[5, 5]), "share")
    refused(E.E_INVAL, M([kv, other], [1, 1], [a, a + 4 * 5], pos0=[5, 5], ld=6), "share")
    refused(E.E_INVAL, M([kv], [1], [a], pos0=[5], layer=7), "layer")
    refused(E.E_INVAL, M([kv], [50], [a], pos0=[70]), "no page")
    refused(E.E_INVAL, M([kv], [1], [a + 2], pos0=[5]), "aligned")
    refused(E.E_INVAL, M([kv], [1], [a], pos0=[5], lse=m + 1), "aligned")
    refused(0, M([kv], [0], [None]))

    V = c.evict
    refused(E.E_INVAL, c.L.anpd_kv_evict(None, kv, a, 512, 1, 0, 0, 0.0, a, None, 512, None), "NULL cache")
    refused(E.E_INVAL, V(kv, None, 5), "NULL cache")
    for bad in (wide, plain, layers, far):
        if bad is not wide:
            refused(E.E_INVAL, V(kv, bad, 5), "shape")
    refused(E.E_INVAL, V(kv, other, 5, 3, 3), "first")
    refused(E.E_INVAL, V(kv, other, 5, -1, 3), "first")
    refused(E.E_INVAL, V(kv, other, 5, 2147483647, 2147483647), "first")
    refused(E.E_INVAL, V(kv, other, -1), "keep")
    refused(E.E_CAPACITY, V(kv, other, 101))
    small = c.cache(30)
    c.stub.stub_forget()
    refused(E.E_CAPACITY, V(kv, small, 31))
    for rope in (1.0, 0.5, -2.0, inf, nan):
        refused(E.E_INVAL, V(kv, other, 5, rope=rope), "rope_base")
    refused(E.E_INVAL, V(kv, other, 5, mass=None), "NULL")
    refused(E.E_INVAL, V(kv, other, 5, kept=None), "NULL")
    refused(E.E_CAPACITY, V(kv, other, 5, ld=99))
    refused(E.E_CAPACITY, V(kv, other, 5, out=a, ld_out=4))
    refused(E.E_INVAL, V(kv, other, 5, mass=a, out=a), "overlaps")
    refused(E.E_INVAL, V(kv, other, 5, mass=a, out=a + 4 * (512 + 99)), "overlaps")
    refused(E.E_INVAL, V(kv, other, 5, mass=a, kept=a + 400), "out_kept overlaps")
    refused(E.E_INVAL, V(kv, other, 5, mass=a, kept=a + 16000, out=a + 16004), "out_kept overlaps")
    for change in (dict(mass=a + 2), dict(kept=a + 16001), dict(out=a + 16002)):
        refused(E.E_INVAL, V(kv, other, 5, **{**dict(mass=a, kept=a + 20000), **change}), "aligned")
    assert [c.L.anpd_kv_length(x) for x in (kv, other, small)] == [100, 40, 0]

    good = dict(n_layers=1, n_heads=4, head_dim=64, n_kv_heads=2, dtype=1, page_tokens=16)
    for change in (dict(n_layers=0), dict(n_heads=0), dict(head_dim=96), dict(n_kv_heads=3), dict(n_kv_heads=-1), dict(dtype=2), dict(page_tokens=24),
                   dict(page_tokens=4), dict(page_tokens=512)):
        assert c.L.anpd_cache_pool_bytes(C.byref(B.CacheCfg(**{**good, **change})), 64) == 0, change
    cfg = B.CacheCfg(**good)
    for n in (0, -1, (1 << 20) + 1):
        assert c.L.anpd_cache_pool_bytes(C.byref(cfg), n) == 0
    assert c.L.anpd_cache_pool_bytes(None, 64) == 0
    n, h = c.L.anpd_cache_pool_bytes(C.byref(cfg), 64), C.c_void_p()
    pool = c.memory(n + 256)
    assert c.L.anpd_cache_create(C.byref(cfg), pool + 16, n, 64, C.byref(h)) == E.E_INVAL and not h.value
    assert c.L.anpd_cache_create(C.byref(cfg), pool, n - 1, 64, C.byref(h)) == E.E_CAPACITY
    assert c.L.anpd_cache_create(C.byref(cfg), None, n, 64, C.byref(h)) == E.E_INVAL
    assert c.L.anpd_cache_create(C.byref(cfg), pool, n, 64, None) == E.E_INVAL
    # a cache without a model belongs to no model
    acc = C.c_int32()
    assert c.L.anpd_verify(None, kv, (C.c_int32 * 1)(0), 1, 0, C.byref(acc), C.byref(acc), None, None, None) == E.E_INVAL


def test_refusals(stub):
    run(stub, "child_refusals")


def child_workspace():
    """As much as asked for is enough, a byte less is refused before anything is launched; short caches need none."""
    c = Caches()
    import random
    rng = random.Random(0)
    asked = 0
    for turn in range(60):
        dtype, page = rng.choice(((1, 16), (0, 16), (1, 64)))
        n = rng.randint(1, 5000)
        heads, kv_heads = rng.choice(((4, 2), (4, 4), (8, 1)))
        kvs = [c.cache(n, n, heads, kv_heads, dtype=dtype, page=page, layers=1) for _ in range(rng.choice((1, 1, 3)))]
        rows = [rng.randint(0, min(n, rng.choice((1, 4, 300)))) for _ in kvs]
        pos0 = [rng.choice((0, n - r)) for r in rows]
        rules = c.B.AttnRules(0, 0, rng.choice((0, 0, 100, 2000)), rng.choice((0, 0, 70, 3000)))
        h, r, p = (C.c_void_p * len(kvs))(*kvs), (C.c_int32 * len(kvs))(*rows), (C.c_int32 * len(kvs))(*pos0)
        m = c.memory(1 << 12)    # (nothing is read or written here)
        for fn in ("attention", "key_mass"):
            need = getattr(c.L, "anpd_%s_workspace_bytes" % fn)(h, len(kvs), r, p, C.addressof(rules))
            masses = [c.memory(4 * n * kv_heads) for _ in kvs]

            def call(ws, nb):
                c.stub.stub_forget()
                if fn == "attention":
                    return c.L.anpd_attention(h, len(kvs), r, p, 0, m, heads * 64, 1, C.addressof(rules), m, heads * 64, None, ws, nb, None)
                return c.L.anpd_key_mass(h, len(kvs), r, p, 0, m, heads * 64, 1, C.addressof(rules), m, (C.c_void_p * len(kvs))(*masses), n, ws, nb, None)
            if need:
                asked += 1
                ws = c.memory(need)
                assert call(ws, need) == 0 and any("join" in x for x in c.names())
                assert call(ws, need - 1) == c.B.E_CAPACITY and c.names() == []
                assert call(None, need) == c.B.E_INVAL and c.names() == []
                assert call(ws + 16, need) == c.B.E_INVAL and c.names() == []
            else:
                assert call(None, 0) == 0 and not any("join" in x for x in c.names()) and len(c.names()) == (1 if sum(rows) else 0)
    assert asked > 10


def test_workspaces(stub):
    run(stub, "child_workspace")


def child_observed():
    """What is asked for observed prompts suffices for their rows at every length."""
    c = Caches()
    import random
    rng = random.Random(1)
    for heads, kv_heads, dim in ((4, 2, 64), (32, 32, 128), (32, 2, 128), (64, 1, 64), (71, 1, 64)):
        for cap in (40, 700, 9000, 200000):
            kv = c.cache(cap, cap, heads, kv_heads, dim, layers=1)
            for _ in range(40):
                rows = rng.randint(1, min(cap, 32))
                n = rng.choice((cap, rng.randint(rows, cap)))
                h, r, p = (C.c_void_p * 1)(kv), (C.c_int32 * 1)(rows), (C.c_int32 * 1)(n - rows)
                need = max(c.L.anpd_attention_workspace_bytes(h, 1, r, p, None), c.L.anpd_key_mass_workspace_bytes(h, 1, r, p, None))
                assert c.L.anpd_kv_observe_workspace_bytes(kv, rows) >= need + 8 * rows * heads * dim + 4 * rows * heads, (heads, cap, rows, n)
    assert c.L.anpd_kv_observe_workspace_bytes(kv, 0) == c.L.anpd_kv_observe_workspace_bytes(kv, 33) == c.L.anpd_kv_observe_workspace_bytes(None, 1) == 0
    m = c.memory(1 << 12)
    assert c.L.anpd_kv_observe(kv, m, 10, 1, m, 1 << 12) == c.B.E_INVAL      # no model
    assert c.L.anpd_kv_observe(None, m, 10, 1, m, 1 << 12) == c.B.E_INVAL
    assert c.L.anpd_kv_observe(kv, None, 0, 0, None, 0) == 0


def test_observed_prompts_workspace(stub):
    run(stub, "child_observed")


def child_device():
    c = Caches()
    kv = c.cache(100, 50, device=3)
    ready = c.devices.stub_device_switches()
    m = c.memory(1 << 16, 3)
    assert c.attention([kv], [1], pos0=[49], q=m, out=m) == 0
    assert c.devices.stub_device_switches() == ready + 2      # there and back
    assert c.mass([kv], [1], [m], pos0=[49], q=m, lse=m) == 0
    assert c.evict(kv, kv, 10) == 0 and c.devices.stub_device_switches() == ready + 6
    near = c.cache(100, 50)
    assert c.attention([near], [1], pos0=[49]) == 0 and c.devices.stub_device_switches() == ready + 6
    assert c.attention([near, kv], [1, 1], pos0=[49, 5]) == c.B.E_INVAL


def test_calls_run_on_the_caches_device(stub, tmp_path):
    run(stub, "child_device", tmp=tmp_path)


def child_failures():
    """Each launch of an eviction fails once: it is reported, and no length has changed."""
    c = Caches()
    for n in (1, 2):
        kv, dst = c.cache(300, 200), c.cache(300, 30)
        c.stub.stub_fail_launch(n)
        assert c.evict(kv, dst, 100) == c.B.E_HIP
        assert (c.L.anpd_kv_length(kv), c.L.anpd_kv_length(dst)) == (200, 30)
        c.stub.stub_fail_launch(0)
        c.stub.hipGetLastError()
        assert c.evict(kv, dst, 100) == 0 and c.L.anpd_kv_length(dst) == 100 and c.L.anpd_kv_length(kv) == 200
        assert c.evict(kv, kv, 7) == 0 and c.L.anpd_kv_length(kv) == 7
    kv = c.cache(300, 200)
    c.stub.stub_fail_launch(1)
    assert c.attention([kv], [1], pos0=[5]) == c.B.E_HIP


def test_failed_launches_are_reported(stub):
    run(stub, "child_failures")


def child_forms():
    """Shapes whose rows share keys through LDS, which tests elsewhere rely on; a token and a short prompt do not."""
    sys.path.insert(0, HERE)
    c = Caches()
    import ast
    named = {n.targets[0].id: n.value for n in ast.parse(open(os.path.join(HERE, "cache_reference.py")).read()).body if isinstance(n, ast.Assign)}
    shapes = ast.literal_eval(named["SHARED_SHAPES"])
    assert len(shapes) >= 4
    for heads, kv_heads, dim, spans in shapes + [(32, 32, 128, [(500, 1)]), (32, 32, 128, [(0, 500)])]:
        kvs = [c.cache(p + n, p + n, heads, kv_heads, dim, layers=1) for p, n in spans]
        ws = c.memory(64 << 20)
        large = (heads, kv_heads, dim, spans) in shapes
        for dtype in (0, 1):
            for rules, able in (({}, True), ({"prefix": 2040}, True), ({"cap": 4.0}, False), ({"slopes": ws}, False)):
                c.stub.stub_forget()
                given = c.B.AttnRules(**rules)
                assert c.attention(kvs, [n for _, n in spans], [p for p, _ in spans], dtype=dtype, ldq=heads * dim, ldo=heads * dim, ws=ws, nb=64 << 20, rules=given) == 0, c.L.anpd_last_error()
                shared = "cache_attn_tile_kernel" in c.names()[0]
                assert shared == (large and able), (heads, spans, dtype, rules, c.names())
        if (heads, kv_heads, dim, spans) == shapes[0]:   # (as tested elsewhere)
            for window in (6900, 7000):
                c.stub.stub_forget()
                assert c.attention(kvs, [n for _, n in spans], [p for p, _ in spans], ldq=heads * dim, ldo=heads * dim, ws=ws, nb=64 << 20, rules=c.B.AttnRules(window=window)) == 0
                assert "cache_attn_tile_kernel" in c.names()[0]
    heads, kv_heads, dim, ((_, n),) = ast.literal_eval(named["SHARED_DOCUMENTS"])
    kv = c.cache(n, n, heads, kv_heads, dim, layers=1)
    for dtype in (0, 1):
        for rules in ({}, {"prefix": 100}, {"prefix": 100, "window": 2500}):
            c.stub.stub_forget()
            assert c.attention([kv], [n], [0], dtype=dtype, ldq=heads * dim, ldo=heads * dim, ws=ws, nb=64 << 20, rules=c.B.AttnRules(first_key=ws, **rules)) == 0
            assert ("cache_attn_tile_kernel" in c.names()[0]) == (dtype == 1), (dtype, rules, c.names())


def test_forms(stub):
    run(stub, "child_forms")


def child_interleaved():
    """Masses of several sequences may lie between each other's rows; whether they share any is said for every distance."""
    c = Caches()
    for kv_heads, total, other, ld in ((1, 6, 3, 9), (2, 6, 6, 12), (2, 6, 2, 11), (4, 5, 9, 14), (4, 1, 1, 1), (4, 1, 1, 2), (4, 7, 7, 7)):
        a, b = (c.cache(64, 32, heads=4, kv_heads=kv_heads) for _ in range(2))
        m = c.memory(1 << 12)
        base = m + 4 * 256
        rows = lambda at, n: {at + g * ld + j for g in range(kv_heads) for j in range(n)}      # noqa: E731
        free = 0
        for d in range(-4 * ld - 12, 4 * ld + 13):
            shared = bool(rows(0, total) & rows(d, other))
            free += not shared
            c.stub.stub_forget()
            rc = c.mass([a, b], [1, 1], [base, base + 4 * d], pos0=[total - 1, other - 1], ld=ld)
            assert rc == (c.B.E_INVAL if shared else 0), (kv_heads, total, other, ld, d)
            assert bool(c.names()) != shared and (not shared or "share" in c.L.anpd_last_error().decode())
        assert free


def test_interleaved_masses(stub):
    run(stub, "child_interleaved")


def child_forms_with_rules():
    """Every call that shared_forms.py lists takes the form whose rows share keys, in the instance that it is listed for."""
    sys.path.insert(0, HERE)
    from shared_forms import cases
    c = Caches()
    ws, seen = c.memory(64 << 20), set()
    for (heads, kv_heads, dim, spans), q, rules in cases():
        kvs = [c.cache(p + n, p + n, heads, kv_heads, dim, layers=1) for p, n in spans]
        rules = dict(rules)
        given = c.B.AttnRules(first_key=ws if rules.pop("document", 0) else None, **rules)
        c.stub.stub_forget()
        assert c.attention(kvs, [n for _, n in spans], [p for p, _ in spans], dtype=c.B.F32 if q == "f32" else c.B.BF16, ldq=heads * dim, ldo=heads * dim,
                           ws=ws, nb=64 << 20, rules=given) == 0, c.L.anpd_last_error()
        name = c.names()[0]
        assert "cache_attn_tile_kernel" in name, (heads, kv_heads, dim, spans, q, rules, name)
        seen.add((name, len(c.names())))
    assert len({name for name, _ in seen}) == 4 and {n for _, n in seen} == {1, 2}, seen


def test_forms_with_rules(stub):
    run(stub, "child_forms_with_rules")


NO_MEMORY = r"""
// operator new, which gives nothing from the n-th time on if told so
#include <cstdlib>
#include <new>
static long g_left = -1;
extern "C" void stub_news_left(long n) { g_left = n; }
void *operator new(std::size_t n)
{
    if (g_left == 0) throw std::bad_alloc();
    if (g_left > 0) --g_left;
    if (void *p = std::malloc(n)) return p;
    throw std::bad_alloc();
}
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, std::size_t) noexcept { std::free(p); }
"""


def child_no_memory():
    """Host memory that runs out in the middle is reported: an exception must not leave a C entry."""
    news = C.CDLL(os.environ["ANPD_NO_MEMORY"], mode=C.RTLD_GLOBAL)
    news.stub_news_left.argtypes = [C.c_long]
    c = Caches()
    cfg = c.B.CacheCfg(2, 4, 64, 2, 1, 16)
    n, kv = c.L.anpd_cache_pool_bytes(C.byref(cfg), 1 << 16), C.c_void_p()
    pool = c.memory(n)
    failed = 0
    for left in range(8):
        news.stub_news_left(left)
        rc = c.L.anpd_cache_create(C.byref(cfg), pool, n, 1 << 16, C.byref(kv))
        news.stub_news_left(-1)
        if rc == 0:
            break
        failed += 1
        assert rc == c.B.E_NOMEM and not kv.value and "memory" in c.L.anpd_last_error().decode()
    assert failed == 4 and rc == 0       # the handle and three lists
    # growing and shrinking takes no more
    assert c.L.anpd_kv_truncate(kv, 1 << 16, None) == 0
    news.stub_news_left(0)
    rcs = [c.L.anpd_kv_truncate(kv, m, None) for m in (0, 1 << 16, 17, 0)]
    news.stub_news_left(-1)
    assert rcs == [0] * 4
    c.L.anpd_kv_destroy(kv)


def test_host_memory_that_runs_out(stub, tmp_path):
    (tmp_path / "news.cpp").write_text(NO_MEMORY)
    subprocess.run(["g++", "-O1", "-fPIC", "-shared", str(tmp_path / "news.cpp"), "-o", str(tmp_path / "news.so")], check=True)
    env = dict(os.environ, ANPD_HIP_STUB=stub, PYTHONPATH=os.path.dirname(HERE), ANPD_NO_MEMORY=str(tmp_path / "news.so"))
    r = subprocess.run([sys.executable, os.path.abspath(__file__), "child_no_memory"], capture_output=True, text=True, timeout=120, env=env)
    assert r.returncode == 0, r.stdout + r.stderr


def test_types_of_a_cache():
    """Any other word, or a type of torch, is no fp32 cache."""
    import torch
    from paper_2404_08698_amd import binding as B
    for bad in ("bfloat16", "BF16", "fp32", "float32", "fp16", "", None, torch.bfloat16, torch.float32, B.BF16):
        with pytest.raises(ValueError):
            B.LayerCache(1, 4, 64, 64, dtype=bad)


def test_rules_beyond_32_bits():
    """A prefix or window of 2^32 would be none at all."""
    from paper_2404_08698_amd import binding as B
    for bad in (1 << 31, 1 << 32, (1 << 32) + 5, -1, -(1 << 32)):
        for name in ("window", "prefix"):
            with pytest.raises(ValueError):
                B.AttentionRules(**{name: bad})
    r = B.AttentionRules(window=(1 << 31) - 1, prefix=(1 << 31) - 1)
    assert (r.struct.window, r.struct.prefix) == ((1 << 31) - 1, (1 << 31) - 1)


if __name__ == "__main__":
    globals()[sys.argv[1]](*sys.argv[2:])
