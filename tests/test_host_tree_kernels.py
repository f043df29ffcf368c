"""What the compiler gives the kernels of the drafted-token calls (no GPU needed): registers that stay registers, two workgroups to a
compute unit where a form counts on them, and the loop of the 256-row form, 64 products and as many exponentials, free of scratch
memory -- what that kernel spills belongs to its masked and repeated tiles."""
import importlib.util
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _compile(source, *flags, out=os.devnull):
    spec = importlib.util.spec_from_file_location("lvlm_build", os.path.join(ROOT, "paper_2509_00419_amd", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    run = subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", *flags, os.path.join(build.CSRC, source), "-o", out],
                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert run.returncode == 0, run.stdout[-2000:]
    return run.stdout


def _reports(source):
    out = {}
    for part in _compile(source, "-Rpass-analysis=kernel-resource-usage", "-c").split("Function Name: ")[1:]:
        got = {k: int(v) for k, v in re.findall(r"(Scratch|Occupancy)\w* \[[^\]]*\]: (\d+)", part)}
        out[part.split()[0]] = (got["Occupancy"], got["Scratch"])
    return out


def test_registers_and_waves_of_append_and_commit():
    for kernel, (_, scratch) in _reports("append.hip").items():
        assert scratch == 0, kernel


def test_registers_and_waves_of_tree_attention():
    reports = _reports("tree.hip")
    forms = {k: v for k, v in reports.items() if "tree_attn_kernel" in k}
    assert len(forms) == 13 and len(reports) == 13 + 6 + 4, sorted(reports)
    for kernel, (waves, scratch) in reports.items():
        if "tree_attn_kernelILi0ELi128ELi2ELi1E" in kernel:
            continue                                            # (the test below)
        assert scratch == 0, (kernel, scratch)
    for form in ("Li0ELi128ELi1ELi2E", "Li0ELi128ELi1ELi1E", "Li0ELi64ELi1ELi4E", "Li0ELi64ELi1ELi2E", "Li0ELi64ELi1ELi1E"):
        (waves, _), = (v for k, v in forms.items() if form in k)
        assert waves >= 2, form


def test_the_loop_of_the_256_row_form_keeps_its_registers(tmp_path):
    asm = str(tmp_path / "tree.s")
    _compile("tree.hip", "-S", out=asm)
    text = open(asm).read()
    for form, products in (("Li0ELi128ELi2ELi1E", 64), ("Li0ELi64ELi2ELi1E", 32)):
        at = re.search(r"^\S*tree_attn_kernelI" + form + r"\S*:\s*;", text, re.M).start()
        blocks = re.split(r"^\.LBB\S+:", text[at:text.index(".Lfunc_end", at)], flags=re.M)
        loops = [b for b in blocks if len(re.findall(r"^\tv_mfma", b, re.M)) == products and len(re.findall(r"^\tv_exp_f32", b, re.M)) == 64]
        assert len(loops) == 1 and "scratch_" not in loops[0], form
