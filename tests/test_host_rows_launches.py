"""Rows of keys and values by the million, on the stand-in for the HIP runtime: a call is launched whole or refused (no GPU needed)."""
import ctypes as C
import os
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
import test_host_draft_operators as T  # noqa: E402
from test_host_path import stub  # noqa: E402,F401


def test_many_rows(stub, tmp_path, monkeypatch):  # noqa: F811
    monkeypatch.setattr(T, "__file__", os.path.abspath(__file__))      # (the child is this file)
    T.run(stub, "child_many_rows", tmp_path)


def child_many_rows():
    """A launch has fewer than 2^32 threads, of which 16 positions of a head have two waves."""
    c = T.Draft()
    c.stub.stub_blocks.restype, c.stub.stub_blocks.argtypes = C.c_uint, [C.c_int]
    n, heads = 1 << 20, 8
    kv = c.cache(n, n, heads=heads, kv_heads=heads, dim=64, layers=1, dtype=8)
    spans = n // 16
    for seqs, rows in ((1, n), (63, n), (64, n - 16), (64, n)):
        c.stub.stub_forget()
        rc = c.rows(c.L.anpd_kv_load, [kv] * seqs, [rows] * seqs, pos0=[0] * seqs, ldk=512, ldv=512)
        fits = seqs * (rows // 16) * heads * 2 * 64 < 1 << 32
        if not fits:
            T.refused(c, c.B.E_CAPACITY, rc, "too many rows")
            continue
        assert rc == 0 and len(c.names()) == 1
        assert c.stub.stub_blocks(0) * 256 < 1 << 32 and c.stub.stub_blocks(0) * 4 == seqs * (rows // 16) * heads * 2
    assert spans * 64 * heads * 2 * 64 == 1 << 32


if __name__ == "__main__":
    globals()[sys.argv[1]]()
