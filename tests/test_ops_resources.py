"""Registers of the operators for several tokens, as the build records them (no GPU)."""
import os


def test_operator_kernels_keep_their_state_in_registers():
    """No scratch memory, but for one register of the log probabilities' fp32 kernel, whose six waves per SIMD are
    worth more; attention and products fit two waves per SIMD."""
    from paper_2606_09682_amd import build
    if not os.path.exists(build.RESOURCES):
        build.build()
    seen = {"attn_kernel": 0, "attn_join_kernel": 0, "linear_kernel": 0, "logprob_chunk_kernel": 0,
            "logprob_join_kernel": 0}
    for line in open(build.RESOURCES):
        name, *kv = line.split()
        fields = dict(x.split("=") for x in kv)
        for kind in seen:
            if kind in name:
                seen[kind] += 1
                spared = kind == "logprob_chunk_kernel"
                assert int(fields["scratch"]) <= 8 * spared and int(fields["vgpr_spill"]) <= spared, line
                assert int(fields["vgprs"]) <= (80 if spared else 256), line
    assert all(seen.values()), seen
