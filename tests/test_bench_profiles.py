"""The bench reports the step kernel's measured traffic and counters only while the committed summaries belong
to the committed kernel source."""

import glob
import os
import re

import bench


def test_summaries_belong_to_the_kernel_source():
    assert bench.measured_traffic() is not None and bench.measured_counters() is not None
    sha = bench.kernel_source_sha256()
    for path in glob.glob(os.path.join(bench.ROOT, "profiles", "*.md")):
        for named in re.findall(r"kernel_source_sha256:\s*([0-9a-f]{64})", open(path).read()):
            assert named == sha, f"{os.path.basename(path)}: counters of another source"
