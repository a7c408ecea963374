"""Trees over caches, rows into caches, commits and sampling on the stand-in for the HIP runtime: what they refuse before anything is launched, which memory they
ask for, and whose device they run on (no GPU needed)."""
import ctypes as C
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
from test_host_cache_operators import Caches as Stub  # noqa: E402
from test_host_cache_operators import DEVICES  # noqa: E402
from test_host_path import stub  # noqa: E402,F401

MORE = DEVICES + r"""
extern "C" {
static int g_capturing = 0;
void stub_capture(int on) { g_capturing = on; }
int hipStreamIsCapturing(void *, int *status) { *status = g_capturing; return 0; }
}
"""


def run(stub, name, tmp_path):  # noqa: F811
    (tmp_path / "devices.cpp").write_text(MORE)
    subprocess.run(["g++", "-O1", "-fPIC", "-shared", str(tmp_path / "devices.cpp"), "-o", str(tmp_path / "devices.so")], check=True)
    env = dict(os.environ, ANPD_HIP_STUB=stub, PYTHONPATH=os.path.dirname(HERE), ANPD_DEVICES_STUB=str(tmp_path / "devices.so"))
    r = subprocess.run([sys.executable, os.path.abspath(__file__), name], capture_output=True, text=True, timeout=120, env=env)
    assert r.returncode == 0, r.stdout + r.stderr


def test_trees(stub, tmp_path):  # noqa: F811
    run(stub, "child_trees", tmp_path)


def test_rows(stub, tmp_path):  # noqa: F811
    run(stub, "child_rows", tmp_path)


def test_commits(stub, tmp_path):  # noqa: F811
    run(stub, "child_commits", tmp_path)


def test_samples(stub, tmp_path):  # noqa: F811
    run(stub, "child_samples", tmp_path)


# ------------------------------------------------------------------------------------------- in the child

class Draft(Stub):
    def tree(self, kvs, rows, parent=1, pos0=None, layer=0, q=None, ldq=256, dtype=1, rules=None, out=None, ldo=256, ws=None, nb=0):
        q, out = self.memory(1 << 17) if q is None else q, self.memory(1 << 17) if out is None else out
        parent = self.memory(1 << 12) if parent == 1 else parent
        return self.L.anpd_tree_attention((C.c_void_p * len(kvs))(*kvs), len(kvs), (C.c_int32 * len(rows))(*rows), None if pos0 is None else (C.c_int32 * len(pos0))(*pos0),
                                          layer, q, ldq, dtype, parent, None if rules is None else C.addressof(rules), out, ldo, None, ws, nb, None)

    def rows(self, fn, kvs, rows, pos0=None, layer=0, k=1, ldk=128, v=1, ldv=128, dtype=1, n=None):
        k, v = (self.memory(1 << 17) if t == 1 else t for t in (k, v))
        return fn((C.c_void_p * max(1, len(kvs)))(*kvs), len(kvs) if n is None else n, (C.c_int32 * max(1, len(rows)))(*rows),
                  None if pos0 is None else (C.c_int32 * len(pos0))(*pos0), layer, k, ldk, v, ldv, dtype, None)

    def sample(self, rows=2, vocab=100, ld=None, dtype=0, rules=None, logits=1, uniform=1, token=1, logprob=None, ws=None, nb=0):
        logits, uniform, token = (self.memory(1 << 17) if t == 1 else t for t in (logits, uniform, token))
        return self.L.anpd_sample(logits, vocab if ld is None else ld, dtype, rows, vocab, None if rules is None else C.addressof(rules), uniform, token, logprob, ws, nb, None)


def refused(c, code, rc, word=""):
    assert rc == code and word in c.L.anpd_last_error().decode(), (rc, c.L.anpd_last_error())
    assert not c.names(), c.names()


def child_trees():
    c = Draft()
    E = c.B
    for dtype in (0, 1, 8):
        kv, other = c.cache(128, 40, dtype=dtype), c.cache(128, 40, dtype=dtype, heads=8)
        for rows in (1, 24):
            assert c.L.anpd_kv_truncate(kv, 40 + 64, None) == 0
            refused(c, E.E_INVAL, c.tree([kv], [rows], parent=None, pos0=[40]), "parent")
            refused(c, E.E_INVAL, c.tree([kv], [rows], parent=c.memory(64) + 2, pos0=[40]), "parent")
        refused(c, E.E_CAPACITY, c.tree([kv], [65], pos0=[10]), "64 at most")
        refused(c, E.E_CAPACITY, c.tree([kv], [64], pos0=[65]), "capacity")
        refused(c, E.E_INVAL, c.tree([kv, other], [1, 1], pos0=[0, 0]), "shape")
        refused(c, E.E_INVAL, c.tree([kv], [1], pos0=[100], layer=2), "layer")
        refused(c, E.E_INVAL, c.tree([kv], [1], pos0=[100], dtype=8), "dtype")
        assert c.L.anpd_kv_truncate(kv, 40, None) == 0
        refused(c, E.E_INVAL, c.tree([kv], [20], pos0=[40]), "no page")
        assert c.tree([kv], [0]) == 0 and not c.names()
    kv = c.cache(1 << 14, 9000, dtype=8)
    n = c.L.anpd_tree_attention_workspace_bytes((C.c_void_p * 1)(kv), 1, (C.c_int32 * 1)(30), (C.c_int32 * 1)(8000), None)
    assert n > 0
    refused(c, E.E_INVAL, c.tree([kv], [30], pos0=[8000]), "workspace")
    refused(c, E.E_CAPACITY, c.tree([kv], [30], pos0=[8000], ws=c.memory(n), nb=n - 1), "workspace")
    assert c.tree([kv], [30], pos0=[8000], ws=c.memory(n), nb=n) == 0
    assert ["attn8" in x for x in c.names()] == [True, False] and "join" in c.names()[1]


def child_rows():
    c = Draft()
    E, store, load = c.B, c.L.anpd_kv_store, c.L.anpd_kv_load
    for dtype, page in ((0, 8), (1, 16), (1, 32), (8, 16)):
        kv, two, other = c.cache(64, 10, dtype=dtype, page=page), c.cache(64, 10, dtype=dtype, page=page), c.cache(64, 10, dtype=dtype, page=page, layers=3)
        for fn in (store, load):
            refused(c, E.E_INVAL, c.rows(fn, [], [], n=0), "n_seq")
            refused(c, E.E_INVAL, c.rows(fn, [kv], [1], n=65), "n_seq")
            refused(c, E.E_INVAL, c.rows(fn, [kv, other], [1, 1]), "shape")
            refused(c, E.E_INVAL, c.rows(fn, [kv], [-1]), "rows")
            refused(c, E.E_INVAL, c.rows(fn, [kv], [1], pos0=[-1]))
            refused(c, E.E_CAPACITY, c.rows(fn, [kv], [55]), "capacity")
            refused(c, E.E_CAPACITY, c.rows(fn, [kv], [1], pos0=[(1 << 31) - 1]), "capacity")
            refused(c, E.E_INVAL, c.rows(fn, [kv], [1], layer=2, pos0=[0]), "layer")
            refused(c, E.E_INVAL, c.rows(fn, [kv], [1], layer=-1, pos0=[0]), "layer")
            refused(c, E.E_INVAL, c.rows(fn, [kv], [1], dtype=8, pos0=[0]), "dtype")
            refused(c, E.E_INVAL, c.rows(fn, [kv], [1], ldk=127, pos0=[0]), "wide")
            refused(c, E.E_INVAL, c.rows(fn, [kv], [1], ldv=127, pos0=[0]), "wide")
            refused(c, E.E_INVAL, c.rows(fn, [kv], [1], k=None, pos0=[0]), "NULL")
            refused(c, E.E_INVAL, c.rows(fn, [kv], [1], v=c.memory(4096) + 1, pos0=[0]), "aligned")
            assert c.rows(fn, [kv], [0], k=None, v=None) == 0
        refused(c, E.E_INVAL, c.rows(store, [kv, two, kv], [1, 1, 1]), "share")
        refused(c, E.E_INVAL, c.rows(load, [kv], [40]), "no page")
        # a captured stream: not with pages to add
        c.devices.stub_capture(1)
        refused(c, E.E_INVAL, c.rows(store, [kv], [40]), "captured")
        assert c.rows(store, [kv], [1], pos0=[3]) == 0 and len(c.names()) == 1
        c.devices.stub_capture(0)
        assert c.rows(store, [kv, two], [40, 3]) == 0
        assert c.rows(load, [kv, kv], [40, 2]) == 0
        names = c.names()
        assert len(names) == 3 and all("cache_rows" in n for n in names)
        c.stub.stub_forget()
    # the caches' device, whichever is the current one
    kv = c.cache(64, 10, dtype=8, device=1)
    before = c.devices.stub_device_switches()
    assert c.rows(store, [kv], [1]) == 0 and c.devices.stub_device_switches() == before + 2


def child_commits():
    c = Draft()
    E = c.B

    def commit(kv, rows, n=None):
        return c.L.anpd_kv_commit(kv, (C.c_int32 * max(1, len(rows)))(*rows), len(rows) if n is None else n, None)

    for dtype, page in ((0, 8), (1, 16), (1, 32), (8, 16)):
        kv = c.cache(64, 10, dtype=dtype, page=page)
        refused(c, E.E_INVAL, c.L.anpd_kv_commit(None, None, 0, None))
        refused(c, E.E_INVAL, c.L.anpd_kv_commit(kv, None, 1, None))
        for rows, code in (([0, 0], E.E_INVAL), ([3, 1], E.E_INVAL), ([-1], E.E_INVAL), ([64], E.E_INVAL), ([54], E.E_CAPACITY), ([0, 40], E.E_INVAL), (list(range(65)), E.E_INVAL)):
            refused(c, code, commit(kv, rows))
        refused(c, E.E_INVAL, commit(kv, [0], n=-1))
        assert c.L.anpd_kv_length(kv) == 10
        assert c.rows(c.L.anpd_kv_store, [kv], [20]) == 0
        c.stub.stub_forget()
        # a path that lies where it belongs moves nothing
        assert commit(kv, [0, 1]) == 0 and not c.names() and c.L.anpd_kv_length(kv) == 12
        assert c.rows(c.L.anpd_kv_store, [kv], [20]) == 0
        c.stub.stub_forget()
        assert commit(kv, [0, 7]) == 0 and len(c.names()) == 1 and c.L.anpd_kv_length(kv) == 14
        c.stub.stub_forget()
        assert commit(kv, []) == 0 and c.L.anpd_kv_length(kv) == 14 and not c.names()


def child_samples():
    c = Draft()
    E, R = c.B, c.B.SampleRules
    refused(c, E.E_INVAL, c.sample(dtype=8), "dtype")
    refused(c, E.E_INVAL, c.sample(rows=-1), "rows")
    for vocab in (0, -1, (1 << 20) + 1):
        refused(c, E.E_INVAL, c.sample(vocab=vocab), "vocab")
        assert c.L.anpd_sample_workspace_bytes(1, vocab) == 0
    refused(c, E.E_INVAL, c.sample(ld=99), "apart")
    for rules in (R(-1.0, 0, 1.0, 0.0), R(float("nan"), 0, 1.0, 0.0), R(float("inf"), 0, 1.0, 0.0), R(1.0, -1, 1.0, 0.0), R(1.0, 0, 1.01, 0.0), R(1.0, 0, float("nan"), 0.0),
                  R(1.0, 0, 1.0, -0.1), R(1.0, 0, 1.0, float("nan")), R(1.0, 0, 1.0, 1.5)):
        refused(c, E.E_INVAL, c.sample(rules=rules))
        refused(c, E.E_INVAL, c.sample(rules=rules, rows=0))
    refused(c, E.E_INVAL, c.sample(rules=R(1.0, 0, 1.0, 0.0, c.memory(64) + 1, None, None, None)), "aligned")
    for name in ("logits", "uniform", "token"):
        refused(c, E.E_INVAL, c.sample(**{name: None}), "NULL")
        refused(c, E.E_INVAL, c.sample(**{name: c.memory(4096) + 2}), "aligned")
    refused(c, E.E_INVAL, c.sample(logprob=c.memory(64) + 2), "aligned")
    assert c.sample(rows=0, logits=None, uniform=None, token=None) == 0 and not c.names()
    assert c.sample() == 0 and len(c.names()) == 1
    c.stub.stub_forget()
    # sums of a row stay below 2^62 for every vocabulary, memory for 256 rows at most
    assert c.L.anpd_sample_workspace_bytes(5, 8192) == 0
    one = c.L.anpd_sample_workspace_bytes(1, 8193)
    assert one > 0 and c.L.anpd_sample_workspace_bytes(256, 8193) == c.L.anpd_sample_workspace_bytes(10000, 8193) > one
    need = c.L.anpd_sample_workspace_bytes(2, 9000)
    refused(c, E.E_INVAL, c.sample(vocab=9000), "workspace")
    refused(c, E.E_INVAL, c.sample(vocab=9000, ws=c.memory(need) + 64, nb=need), "workspace")
    refused(c, E.E_CAPACITY, c.sample(vocab=9000, ws=c.memory(need), nb=need - 1), "workspace")
    assert c.sample(vocab=9000, ws=c.memory(need), nb=need) == 0 and len(c.names()) == 2
    # the logits' device
    before = c.devices.stub_device_switches()
    c.stub.stub_forget()
    assert c.sample(logits=c.memory(1 << 16, 1)) == 0 and c.devices.stub_device_switches() == before + 2


if __name__ == "__main__":
    globals()[sys.argv[1]]()
