"""A workspace of tree attention, or of a decoder layer's verify step, made for some numbers
of sequences, drafts and positions serves every smaller call.

The sizes follow launch plans for the device's SMs, so the library is loaded in a
process of its own, where two runtime queries answer for a GPU of 152 SMs.
"""
import os
import subprocess
import sys

import pytest

from test_workspace_sizes import FAKE, PRELUDE, ROOT


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    import __graft_entry__
    __graft_entry__.build()
    d = tmp_path_factory.mktemp("fake")
    (d / "f.c").write_text(FAKE)
    so = str(d / "libfake.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", so, str(d / "f.c")], check=True)

    def go(code):
        r = subprocess.run([sys.executable, "-c", PRELUDE + code, so], cwd=ROOT, capture_output=True, text=True,
                           env=dict(os.environ, CUDA_VISIBLE_DEVICES=""))
        assert r.returncode == 0, r.stdout + r.stderr
    return go


@pytest.mark.parametrize("H,kv,hd", [(32, 8, 128), (64, 8, 64), (4, 4, 128), (16, 1, 64), (5, 1, 128)])
def test_tree_attention(run, H, kv, hd):
    run(f"""
f = lambda b, t, n: L.wq_attn_tree_workspace_bytes(b, t, {H}, {kv}, {hd}, n)
for t in (1, 2, 9, 33, 128):
    for n in (1, 500, 4001, 32768):
        grows((b, f(b, t, n)) for b in range(1, 70))
for b in (1, 3, 16):
    for n in (1, 500, 4001, 32768):
        grows((t, f(b, t, n)) for t in range(1, 129))
    for t in (1, 2, 9, 33, 128):
        grows((n, f(b, t, n)) for n in list(range(1, 1200, 7)) + list(range(1200, 70000, 411)))
""")


def test_verify_step(run):
    run("""
w = lambda n, k, g, bits: wq._QWeight(256, 256, n, k, g, bits)
lay = wq._DecoderLayer()
lay.n_heads, lay.n_kv, lay.head_dim = 8, 2, 128
lay.qkv, lay.o = w(12 * 128, 1024, 64, 4), w(1024, 1024, 64, 4)
lay.mlp.gate, lay.mlp.up, lay.mlp.down = w(1536, 1024, 64, 2), w(1536, 1024, 64, 2), w(1024, 1536, 64, 4)
f = lambda b, t, n: L.wq_decoder_tree_workspace_bytes(b, t, ctypes.byref(lay), n)
for t in (1, 5, 61):
    grows((b, f(b, t, 4096)) for b in range(1, 40))
for b in (1, 8):
    grows((t, f(b, t, 4096)) for t in range(1, 129))
    grows((n, f(b, 7, n)) for n in range(1, 20000, 131))
""")
