"""A wait for TMEM loads has to name the registers that they fill: to the compiler these are written by the load, and reading them is not
tied to a wait that does not mention them."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_07964_b200", "csrc")


def test_every_wait_names_its_registers():
    waits = 0
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        if os.path.basename(path) != "eb_mma.cuh":
            assert "wait::ld" not in text, path
        assert not re.search(r"\btmem_ld_wait\s*\(\s*\)", text), path
        waits += len(re.findall(r"\btmem_ld_wait\(\s*[a-z]", text))
        # a name that is waited for is one that a load fills
        for name in re.findall(r"\btmem_ld_wait\(\s*([a-z_0-9]+)", text):
            assert name == "reinterpret_cast" or re.search(r"\btmem_ld(8|16)\([^;]*\b%s\b" % name, text), (path, name)
    assert waits >= 6
