"""Every size of logits that the calls accept has a launch, up to the most
rows and classes. No GPU is needed."""

import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_size_has_a_launch(tmp_path):
    csrc = os.path.join(ROOT, "paper_2201_07705_amd", "csrc")
    out = str(tmp_path / "forms")
    subprocess.check_call(["g++", "-std=c++17", "-O1", *(f"-I{os.path.join(ROOT, 'tests', d)}" for d in ("opstub", "hoststub")),
                           f"-I{csrc}", os.path.join(ROOT, "tests", "answerstub", "forms.cpp"), os.path.join(csrc, "answer_plan.cpp"),
                           "-o", out])
    r = subprocess.run([out], capture_output=True, text=True, check=True)
    bad, tried = map(int, r.stdout.split())
    assert tried > 5000 and bad == 0, r.stderr
