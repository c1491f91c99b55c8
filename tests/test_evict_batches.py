"""The eviction's choice reads weights in batches into a thread's arrays; compiled for the host, the batches of every instance
write each place once and none behind the last."""
import os
import re
import subprocess

import paper_2608_20530_amd.build as B

SOURCE = """
#include "cache4.hpp"
#include <cstdio>
using namespace lilicorr;
template <int G, int KEYS> void batches() {
  constexpr int slots = KEYS / G, at_once = loads_at_once(slots);
  for (int x0 = 0; x0 < slots; x0 += at_once)
    for (int x = 0; x < at_once; ++x)
      for (int y = 0; y < G; ++y) std::printf("%d %d %d\\n", G, KEYS, (x0 + x) * G + y);
}
int main() { INSTANCES }
"""


def test_batches_stay_in_their_arrays(tmp_path):
    with open(os.path.join(B.CSRC, "evict.hip")) as f:
        text = f.read()
    assert "kAtOnce = loads_at_once(kSlots)" in text
    instances = sorted(set(re.findall(r"evict_select_kernel<(\d+), (\d+)>", text)))
    assert len(instances) == 3
    source = tmp_path / "batches.hip"
    source.write_text(SOURCE.replace("INSTANCES", " ".join(f"batches<{g}, {k}>();" for g, k in instances)))
    flags = [f for f in B.FLAGS if f not in ("-Wall", "-shared")] + ["--offload-host-only", "-w"]
    subprocess.run(["hipcc", *flags, "-I", os.path.join(B.ROOT, "include"), "-I", B.CSRC, "-o", str(tmp_path / "batches"),
                    str(source)], check=True)
    out = subprocess.run([str(tmp_path / "batches")], check=True, capture_output=True, text=True).stdout
    written = {}
    for line in out.splitlines():
        g, keys, place = map(int, line.split())
        written.setdefault((g, keys), []).append(place)
    for (g, keys), places in written.items():
        assert places == list(range(keys)), (g, keys)
