"""The work plan of attention over shared pages, checked by a host program built from the header that the library uses: every
(row, page) once, shared pages only where they need no mask, partial results in slots of their own, joins that name them all."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_plans_cover_every_page_once(tmp_path):
    exe = str(tmp_path / "shared_plan_host")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", os.path.join(ROOT, "tests", "shared_plan_host.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe, "4000"], stdout=subprocess.PIPE, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip() == "ok 4000", out.stdout
