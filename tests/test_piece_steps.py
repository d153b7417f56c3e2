"""How the key axis of long batches is cut: never into more pieces than the workspace has room for."""

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_pieces_stay_within_what_a_workspace_has_room_for(tmp_path):
    exe = str(tmp_path / "piece_steps")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Wextra", "-o", exe, os.path.join(HERE, "models", "piece_steps.cpp")], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout
