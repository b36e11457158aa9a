"""The recurrence's channel groups (seq_internal.h, compiled for the host): every channel belongs to one group, also
where lanes hold pairs of an odd number of channels.  CPU only."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <stdio.h>
#include "paper_2103_08802_amd/csrc/seq_internal.h"
int main() {
  for (int vec = 1; vec <= 2; ++vec)
    for (int channels = vec == 1 ? 1 : 65; channels <= 1300; ++channels) {
      const int groups = (int)pnn::cdiv64(channels, 64 * vec);
      int next = 0;
      for (int g = 0; g < groups; ++g) {
        const pnn::ScanGroup r = pnn::scan_group(channels, g, vec);
        // groups join without a gap or a channel in common, fill no more than 64 lanes, and hold a lane's channels
        if (r.first != next || r.end - r.first < vec || (r.end - r.first + vec - 1) / vec > 64) {
          printf("%d channels, %d a lane: group %d has %d .. %d\n", channels, vec, g, r.first, r.end);
          return 1;
        }
        next = r.end;
      }
      if (next != channels) {
        printf("%d channels, %d a lane: groups end at %d\n", channels, vec, next);
        return 1;
      }
    }
  return 0;
}
"""


def test_groups_share_no_channel(tmp_path):
    src, exe = tmp_path / "groups.hip", tmp_path / "groups"
    src.write_text(SOURCE)
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-std=c++17", "-I" + ROOT,
                        "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
