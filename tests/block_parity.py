"""Shared helpers for the GPU tests of the rotary and block-sparse entry points."""
import numpy as np
import torch

from oracle.ref_sparse_attn import bf16_bits_to_f64
from paper_2608_26523_b200 import api


def f64(t):
    """bf16 tensor -> float64 array, exactly."""
    return bf16_bits_to_f64(t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16))


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def randn(gen, *shape, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(torch.bfloat16)


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def block_args(prob, lists, splits=0, out=None, lse=None):
    """(args, out, lse, status) of one vpp_block_attn_fwd launch; the workspace stays with the args."""
    T, hq = prob.total_q, prob.num_q_heads
    out = torch.full((T, hq, 128), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    lse = torch.full((T, hq), float("nan"), dtype=torch.float32, device="cuda") if lse is None else lse
    status = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    a = api.make_args(prob.q, prob.k_cache, prob.v_cache, prob.block_table, prob.prefix_len, prob.chunk_len, prob.block_size, prob.max_seq_len,
                      prob.scale, num_kv_splits=splits, out=out, lse=lse, status=status, total_q=T)
    a.keep = torch.empty(api.vpp_block_attn_workspace_size(a, lists.shape[2]), dtype=torch.uint8, device="cuda")
    a.keep.fill_(0xff)                          # (contents need no initialisation)
    a.workspace, a.workspace_bytes = a.keep.data_ptr(), a.keep.numel()
    return a, out, lse, status


def check_attn(out, lse, want, label=""):
    """out against (out, lse, weighted |v|) of the oracle.  The weights of a row are rounded to bf16 (half a step: 2^-8 of each, so at most 2^-8 of
    the weighted |v|), the result once more (2^-8 of it); exponentials and sums in 32 bits stay below 1e-4 of the weighted |v|."""
    ref, ref_lse, mag = want
    got, got_lse = f64(out), lse.cpu().numpy().astype(np.float64)
    err = np.abs(got - ref)
    assert np.isfinite(got).all(), label
    assert (err <= 2.0 ** -8 * (np.abs(ref) + mag) + 1e-4 * mag).all(), (label, float((err / (mag + 1e-30)).max()))
    norm = np.linalg.norm(ref)
    assert np.linalg.norm(got - ref) <= 5e-3 * norm, (label, np.linalg.norm(got - ref) / norm)
    none = np.isneginf(ref_lse)
    assert (np.isneginf(got_lse) == none).all(), label
    assert (out[torch.from_numpy(none).cuda()] == 0).all(), label
    assert (np.abs(got_lse[~none] - ref_lse[~none]) <= 1e-5 * np.maximum(1.0, np.abs(ref_lse[~none]))).all(), label
