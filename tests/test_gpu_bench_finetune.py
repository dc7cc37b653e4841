"""bench.py --predictor-finetune on the GPU: the fields of its report, and batches that leave nothing to train on."""
import json
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("tokens", [1, 300])
def test_finetuning_report(tokens):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    r = subprocess.run([sys.executable, os.path.join(ROOT, "bench.py"), "--workload", "tiny", "--tokens", str(tokens), "--steps", "2",
                        "--warmup", "1", "--no-achievable-peaks", "--no-hbm-bound", "--predictor-finetune", "3"],
                       cwd=ROOT, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    d = json.loads(r.stdout.strip().splitlines()[-1])["predictor_finetune"]
    assert d["steps"] == 3 and d["tokens"] + d["held_out_tokens"] == tokens
    assert d["clip_us"] > 0.0 and d["losses_and_gradients_us"] > 0.0
    assert 0.0 <= d["token_choices_kept_before"] <= 1.0 and 0.0 <= d["token_choices_kept_after"] <= 1.0
    assert (d["loss_first"] == 0.0) == (d["tokens"] == 0)
