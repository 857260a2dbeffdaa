"""Under python -O, which takes assert statements out, fork_blocks without a source is still refused: the call below it takes None for "free these"."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import sys, types
sys.path.insert(0, {root!r})
from paper_2512_11920_amd import kvc
freed = []
kvc._call = types.SimpleNamespace(fork=lambda *a: freed.append(a) or 0)
codec = kvc.Codec.__new__(kvc.Codec)
codec._ctx, codec._leaving = types.SimpleNamespace(value=1), []
codec.close = lambda: None
stream = types.SimpleNamespace(cuda_stream=0)
try:
    codec.fork_blocks(None, object(), 1, 4, stream=stream)
except AssertionError:
    print("refused", len(freed))
else:
    print("freed", len(freed))
"""


def test_fork_without_a_source_frees_nothing():
    for flags in ([], ["-O"]):
        p = subprocess.run([sys.executable, *flags, "-c", PROGRAM.format(root=ROOT)], capture_output=True, text=True, timeout=120)
        assert p.returncode == 0 and p.stdout.strip() == "refused 0", (flags, p.stdout, p.stderr[-500:])
