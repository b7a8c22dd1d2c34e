"""No kernel of the scored router and of the adapters keeps values in scratch memory (metadata of the built library's code
objects, no GPU needed): arguments taken by reference or spilled registers made them up to three times as slow."""
import re
import subprocess


from test_kernel_resources import READELF, _code_objects, pytestmark  # noqa: F401


def test_no_scratch(tmp_path):
    seen = 0
    for i, co in enumerate(_code_objects(str(tmp_path))):
        path = tmp_path / f"{i}.co"
        path.write_bytes(co)
        notes = subprocess.run([READELF, "--notes", str(path)], check=True, capture_output=True, text=True).stdout
        for k in re.split(r"\n  - ", notes):
            name = re.search(r"\.name:\s+(_Z\S+)", k)
            scratch = re.search(r"\.private_segment_fixed_size:\s+(\d+)", k)
            if name and scratch and re.search(r"\d(lora_|route_scored|route_bias)", name.group(1)):
                seen += 1
                assert int(scratch.group(1)) == 0, name.group(1)
    assert seen > 60
