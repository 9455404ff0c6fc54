"""Kernels whose items may fill several rows of a launch get more workgroups than items (the last row is filled up):
each such workgroup has to leave before it reads or waits for anything that goes by its item.  From the sources, so that
it is known before a GPU runs them."""
import glob
import os
import re

from paper_2510_23938_amd import build as B

# what says that a workgroup's item does not exist
LEAVES = re.compile(r"if \((tile \* kTokens >= x\.m|!job\.found|!place\.found)\) return;")
# what may stand ahead of that: nothing that reads memory by the item, and no barrier
READS = re.compile(r"__syncthreads|adapter_of\(|load_|\bx\.index\[|\bx\.y\b|\bx\.out\b|stage\(\)")


def kernels():
    for path in sorted(glob.glob(os.path.join(B.CSRC, "*.hip"))):
        with open(path) as f:
            source = f.read()
        for m in re.finditer(r"__global__ void[^\n]*?(\w+)\((\w+) x\) \{\n(.*?)\n\}\n", source, re.S):
            if "item_of_block()" in m.group(3) or "kRowOfItems" in m.group(3):
                yield os.path.basename(path), m.group(1), m.group(3)


def test_surplus_workgroups_leave_first():
    found = {name: body for _, name, body in kernels()}
    assert set(found) == {"down_kernel", "up_kernel", "up_tiles_kernel", "write_kernel", "stream_attention", "tile_attention"}
    for name, body in found.items():
        leaves = LEAVES.search(body)
        assert leaves, f"{name}: workgroups past the last item go on"
        ahead = "\n".join(line.split("//")[0] for line in body[:leaves.start()].splitlines())
        assert not READS.search(ahead), (name, READS.search(ahead))
