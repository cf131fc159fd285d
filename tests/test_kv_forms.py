"""The shapes of the tests at the ends of the range reach the kernels that they are named for (on the CPU: the library's own
choice)."""
import test_gpu_kv_range as gpu
from test_kv_kernel_choice import FEW, SHORT, SPLIT, STAGES, kernel  # noqa: F401  (kernel is a fixture)

import paper_2501_04304_amd as dgq


def test_forms(kernel):  # noqa: F811
    want = {"few": FEW, "split": SPLIT, "many splits": SPLIT, "short": SHORT, "stages": STAGES, "few, wide": FEW}
    for name, (S, H, d, N, rows, W) in gpu.FORMS.items():
        assert rows <= W * S
        assert kernel(3, N, 0, H, H, d, W, S) == want[name], name
        row = 3 * N * H * (d + 2) * 4
        splits = dgq.dgq_xattn_kv_workspace_bytes(3, N, False, H, H, d, W, S) // row
        if name == "split":
            assert 2 <= splits <= 16 and splits * d <= 2048
        elif name == "many splits":
            assert splits > 16
        else:
            assert splits == 0
