"""The committed counter figures of the learner path's kernels do not go stale with the operators beside it."""
import os
import re
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import bench  # noqa: E402

CSRC = os.path.join(bench.ROOT, "paper_2310_00036_amd", "csrc")


def test_a_digest_covers_nothing_of_the_operators_beside_the_path():
    for key in ("resblock_bwd/bf16/16x16/42x42", "resblock_fwd/bf16/32x32/21x21", "conv_pool/bf16/4x16/84x84/u8",
                "pool_wgrad/bf16/4x16/84x84/u8", "conv_bwd/bf16/16x32/42x42/pool"):
        files = bench.source_files(key)
        assert files and not {"groupnorm.h", "muon.h"} & set(files)
        for f in files:
            assert not re.search(r"groupnorm_|muon_", open(os.path.join(CSRC, f)).read()), (key, f)
