"""Tensors that have no storage (those of a function that torch.func.vmap runs) come back from every native call as "look at it in
Python", where torch says what is wrong with them; nothing that torch throws leaves a call while it does not hold the
interpreter's lock, which ends the process.  On the host: csrc/calls.cpp is built for CPU tensors, in a process of its own."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2601_02360_amd import binding as B
from paper_2601_02360_amd import build

SCRIPT = """
import sys, torch
sys.path.insert(0, sys.argv[1])
import _calls
F, I = torch.float32, torch.int32
fp = lambda *shape: torch.zeros(*shape, dtype=F)
rows, vocab, d, k = 6, 5, 16, 4
ids, u, ws = torch.zeros(rows, dtype=I), fp(d, k), torch.zeros(1 << 16, dtype=torch.uint8)
x, table, narrow, coeff = fp(rows, d), fp(vocab, d), fp(rows, k), fp(vocab * k)
CALLS = {
    "embedding_lookup": [table, ids, x, table, x, 1.0, 0],
    "embedding_grad": [x, ids, table, ws, 1.0, -1, 0, 0],
    "project": [x, u, narrow, table, ids, x, 0, 0],
    "reconstruct": [narrow, u, x, table, ids, x, 0, 0],
    "reproject": [table, table, u, coeff, 0, 0],
    "grad_norm": [None, None, 0, 1.0, fp(2), torch.zeros(16384, dtype=torch.uint8), 0],
    "adamw_step": [None, None, None, None, None, 0, 1e-3, 0.9, 0.95, 1e-8, 0.1, 1, fp(1), 2, fp(2), None, 0],
}
for name, args in CALLS.items():
    for at, t in enumerate(args):
        if not isinstance(t, torch.Tensor):
            continue
        def one(wrapped):
            assert type(wrapped) is torch.Tensor
            try:
                wrapped.data_ptr()
            except RuntimeError:
                pass
            else:
                raise AssertionError("it has storage")
            got = getattr(_calls, name)(*args[:at], wrapped, *args[at + 1:])
            assert got is None, (name, at, got)
            return torch.zeros(())
        print(name, at, flush=True)
        torch.func.vmap(one)(torch.stack([t, t]))
print("every call came back")
"""


def test_tensors_without_storage_are_handed_back(tmp_path, monkeypatch):
    commands = []
    monkeypatch.setattr(build, "_run", lambda cmd, out, verbose: commands.append(cmd))
    build.build_calls()
    source = os.path.join(build.HERE, "csrc", "calls.cpp")
    text = open(source).read()
    assert ".is_cuda()" in text
    here = tmp_path / "calls.cpp"
    here.write_text(text.replace(".is_cuda()", ".is_cpu()"))
    cmd = [{source: str(here), "-O2": "-O0", "-Wl,-rpath,$ORIGIN": "-Wl,-rpath," + build.HERE}.get(a, a) for a in commands[0]]
    subprocess.run(cmd + ["-o", str(tmp_path / "_calls.so")], check=True)
    out = subprocess.run([sys.executable, "-c", SCRIPT, str(tmp_path)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True,
                         timeout=300)
    assert out.returncode == 0 and out.stdout.rstrip().endswith("every call came back"), out.stdout[-3000:]


@pytest.mark.gpu
def test_the_calls_say_what_is_wrong():
    rows, vocab, d = 6, 5, 16
    x, table, ids = torch.zeros(rows, d, device="cuda"), torch.ones(vocab, d, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    ws = B.embedding_grad_workspace(rows, vocab, d)
    for call in (lambda i: B.sparseloco_embedding_lookup(table, i, x), lambda i: B.sparseloco_embedding_grad(x, i, table, ws)):
        with pytest.raises(RuntimeError, match="storage"):
            torch.func.vmap(lambda i: call(i) or torch.zeros(()))(torch.stack([ids, ids]))
    assert not x.any() and (table == 1.0).all()
