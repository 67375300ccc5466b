"""Calls of the operators around the exchange from several threads share nothing that one of them writes without an atomic."""
import os
import re
import subprocess

from paper_1806_04090_b200 import build

SOURCES = ["atomo_step", "atomo_embedding", "atomo_layernorm"]


def test_the_operators_keep_no_plain_globals():
    build.build()
    shared = []
    for name in SOURCES:
        out = subprocess.run(["nm", "-C", os.path.join(build.OBJ, name + ".o")], check=True, capture_output=True, text=True).stdout
        for line in out.splitlines():
            m = re.match(r"[0-9a-f]+ ([bBdD]) (.*)", line)
            # (the occupancies that the layer norm knows are atomics; the rest is what nvcc registers the kernels with)
            if m and "atomo" in m.group(2) and not m.group(2).endswith("::known"):
                shared.append((name, m.group(2)))
    assert not shared
    with open(os.path.join(build.CSRC, "atomo_layernorm.cu")) as f:
        assert not re.search(r"static (?!std::atomic<)\w[\w:<>]* known\b", f.read())
