"""The walk of the loss kernels over a run's chunks and slots, on the CPU: with slot arrays that
contradict each other no index leaves the arrays' lengths, with sound ones every element and
every partial is met once."""
import os
import subprocess

from paper_2606_19989_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_chunk_walk_stays_inside_the_arrays(tmp_path):
    exe = str(tmp_path / "tile_chunks")
    r = subprocess.run([build.HIPCC, "--offload-host-only", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", build.CSRC,
                        "-I", build.INCLUDE, "-x", "hip", os.path.join(HERE, "host", "tile_chunks.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout)


def test_sound_slots_are_met_whole_unless_offsets_are_out_of_order(tmp_path):
    exe = str(tmp_path / "tile_order")
    r = subprocess.run([build.HIPCC, "--offload-host-only", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", build.CSRC,
                        "-I", build.INCLUDE, "-x", "hip", os.path.join(HERE, "host", "tile_order.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, (r.returncode, r.stdout)
