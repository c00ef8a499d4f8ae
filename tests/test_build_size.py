"""What a build leaves in the working copy: device code is stored compressed, so that a copy
with the library, the debug library and their objects stays easy to move."""
import os

MIB = 1 << 20


def test_built_files_are_small():
    import paper_2607_19368_gb300.build as build
    build.build()
    parts = [build.LIB] + [os.path.join(build.BUILD, os.path.basename(s)[:-3] + ".o")
                           for s in build.sources()]
    size = sum(os.path.getsize(f) for f in parts)
    # half of it is the library; a debug build has as much again
    assert size <= 64 * MIB, f"{size / MIB:.0f} MiB"
