"""The README's example runs as it stands (GPU), and does what it says."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    (block,) = re.findall(r"```python\n(.*?)```", open(os.path.join(ROOT, "README.md")).read(), re.S)
    return block


def test_the_example_compiles():
    compile(example(), "README.md", "exec")


@pytest.mark.gpu
def test_the_example_runs():
    import torch

    import paper_2401_06761_amd as ap

    lens = {}

    class Pool(ap.Pool):
        def close(self):  # (what the pool's books say at the end of the example's block)
            if self.handle:
                lens.update((t, ap.apar_thread_len(self.handle, t)) for t in names["kids"])
            super().close()

    names, kept = {}, ap.Pool
    ap.Pool = Pool
    try:
        exec(compile(example(), "README.md", "exec"), names)
    finally:
        ap.Pool = kept
    torch.cuda.synchronize()
    assert len(lens) == 3 and set(lens.values()) == {301}
    assert torch.isfinite(names["out"]).all() and names["out"].abs().max() > 0
    tokens = names["tokens"].tolist()
    assert len(tokens) == 3 and all(-3 <= t < names["logits"].shape[1] for t in tokens)
