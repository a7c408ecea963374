"""How anpd_sample divides many rows among launches, on the stand-in for the HIP runtime (no GPU needed)."""
import ctypes as C
import os
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
from test_host_draft_operators import Draft, run as run_there  # noqa: E402
from test_host_path import stub  # noqa: E402,F401


def test_many_rows(stub, tmp_path, monkeypatch):  # noqa: F811
    import test_host_draft_operators
    monkeypatch.setattr(test_host_draft_operators, "__file__", os.path.abspath(__file__))      # (the child is this file)
    run_there(stub, "child_many_rows", tmp_path)


def child_many_rows():
    """A launch has fewer than 2^32 threads, of which a row's block is 1024; every row is in one launch."""
    c = Draft()
    c.stub.stub_blocks.restype, c.stub.stub_blocks.argtypes = C.c_uint, [C.c_int]
    for rows in (1, 1 << 22, (1 << 22) + 1, (1 << 23) + 5, (1 << 31) - 1):
        c.stub.stub_forget()
        # (nothing is read: kernels are written down, not run)
        assert c.sample(rows=rows, vocab=2) == 0
        blocks = [c.stub.stub_blocks(i) for i in range(c.stub.stub_launches())]
        assert sum(blocks) == rows and max(blocks) * 1024 < 1 << 32, (rows, blocks)


if __name__ == "__main__":
    globals()[sys.argv[1]]()
