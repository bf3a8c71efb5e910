"""Plans of group norm (pcr_norm_plan.h, compiled for the CPU): the workgroups and threads of every plan reach all pixels and channels of its pictures, with the kernel that the plan names."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_every_plan_reaches_its_pictures(tmp_path):
    exe = str(tmp_path / "plans")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-o", exe, os.path.join(HERE, "host_emul", "norm_plans.cpp")])
    run = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0, run.stdout
    assert all(int(n) > 50000 for n in run.stdout.split()), run.stdout          # (every kind of plan was among them)
