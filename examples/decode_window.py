"""From a window's best plan to its first tokens.

The plan evaluator says which activations a replica runs first; this example
takes the first batch that the best plan gives one device, admits it to the
replica's paged KV cache, and decodes it with beam search:

  wf_construct_plans, wf_eval_plans, wf_topk   the plan
  wf_kv_extend                                 admission by free blocks, block tables, slots of the prompts
  wf_beam_select, wf_kv_reorder, wf_kv_extend  a step: selection, rows in its order, slots of the new tokens

The language model is a stand-in of random weights: the mean of the row's
cached vectors, read through its block table, times an output matrix.  So what is
decoded depends on every cached token being where the table says.  Sums that
are kept beside the cache, from the parents and tokens alone, check it at the end.

    python examples/decode_window.py [window] [beams] [steps]
"""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import wfgen  # noqa: E402
from paper_2609_03335_gb300 import wf  # noqa: E402

BLOCK_TOKENS = 16
TOKEN_MIB = 1  # cache of a token: an activation's KV memory (peak - weight) is its prompt's length
VOCAB, WIDTH, EOS = 4099, 32, 0


def first_batch(prob, n_plans=256, most=8):
    """The device, and the activations without predecessors of one model that
    the best of n_plans constructed plans runs on it first."""
    ctx = wf.Ctx(prob, max_P=n_plans)
    plans, res = wf.DevicePlans.empty(n_plans, prob.N), wf.Results(n_plans)
    wf.wf_construct_plans(ctx, plans, seed=1, jitter_us=200_000)
    wf.wf_eval_plans(ctx, plans, res)
    ids = torch.empty(1, dtype=torch.int32, device="cuda")
    wf.wf_topk(ctx, res, n_plans, 1, ids)
    wf.wf_ctx_status(ctx)
    best = int(ids[0])
    place, order = (x[best] for x in plans.numpy(prob.N)[:2])
    off, model = np.asarray(prob.pred_off), np.asarray(prob.model)
    ready = [int(n) for n in order if off[n] == off[n + 1]]
    device, batch = int(place[ready[0]]), []
    for n in ready:
        if int(place[n]) == device and model[n] == model[ready[0]] and len(batch) < most:
            batch.append(n)
    ctx.close()
    return device, batch


def cached_sums(vectors, kv):
    """The sum of each row's cached vectors, by its block table."""
    p = torch.arange(int(kv.len.max()), device="cuda")
    slots = kv.table.long()[:, p // BLOCK_TOKENS] * BLOCK_TOKENS + p % BLOCK_TOKENS
    there = p < kv.len[:, None]
    return torch.where(there[:, :, None], vectors[torch.where(there, slots, 0)], 0.0).sum(1)


def decode(prob, device, batch, beams=4, steps=16, seed=0, n_blocks=None):
    """Beam search of `steps` tokens for the activations of the batch that fit the device (n_blocks: with so many blocks
    in place of the device's).  A search that finds no block left in some step, or waits behind one that does, ends there."""
    D = int(prob.D)
    peak, weight = np.asarray(prob.peak_mib).reshape(-1, D), np.asarray(prob.weight_mib)
    kv_mib = np.array([peak[n, device] - weight[prob.model[n]] for n in batch])
    prompt = np.maximum(1, kv_mib // TOKEN_MIB)
    free_mib = int(np.asarray(prob.cap_mib)[device] - weight[prob.model[batch[0]]])
    n_blocks = n_blocks or free_mib // (BLOCK_TOKENS * TOKEN_MIB)
    groups, rows = len(batch), len(batch) * beams
    width = -(-(int(prompt.max()) + steps) // BLOCK_TOKENS)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    embed, out_matrix = rand(VOCAB, WIDTH), rand(WIDTH, VOCAB)
    cache = torch.zeros((1, n_blocks, BLOCK_TOKENS, WIDTH), device="cuda")
    vectors = cache.view(n_blocks * BLOCK_TOKENS, WIDTH)

    scratch = wf.Decode(max_rows=rows, max_row_blocks=width, max_vocab=VOCAB, max_keep=2 * beams)
    kv = wf.Kv.empty(rows, width, BLOCK_TOKENS, n_blocks)
    score = torch.full((rows,), -torch.inf, device="cuda")
    moves, found = wf.KvMoves(rows), wf.BeamOut(groups, beams, 2 * beams, score)  # the scores move on in place
    heads = torch.arange(0, rows, beams, device="cuda")

    # The prompts, each in its search's first row.  A prompt that finds no blocks left waits: here it is left out.
    prefill = wf.KvStep(rows, int(prompt.sum()), kv)
    add = torch.zeros(rows, dtype=torch.int32, device="cuda")
    add[heads] = torch.from_numpy(prompt.astype(np.int32)).cuda()
    wf.wf_kv_extend(scratch, kv, add, prefill)
    admitted = (kv.len[heads] > 0).cpu().numpy()
    tokens = torch.randint(1, VOCAB, (int(prompt.sum()),), generator=gen, device="cuda")
    used = prefill.slot >= 0
    vectors[prefill.slot[used]] = embed[tokens[:int(used.sum())]]
    taken_at_first = int(kv.ends[0])

    # Beside the cache: the sum of the vectors that each row's tokens have.
    state = torch.zeros((rows, WIDTH), device="cuda")
    state.index_add_(0, prefill.row[used].long(), vectors[prefill.slot[used]])
    score[heads] = torch.where(kv.len[heads] > 0, 0.0, -torch.inf)
    step = wf.KvStep(rows, rows, kv)
    parents, tokens = [], []
    lasted = torch.zeros(groups, dtype=torch.int32, device="cuda")  # steps of each search
    going = kv.len[heads] > 0
    for _ in range(steps):
        logits = (cached_sums(vectors, kv) / kv.len.clamp(min=1)[:, None]) @ out_matrix
        wf.wf_beam_select(scratch, logits, score, found, eos=EOS)
        wf.wf_kv_reorder(scratch, kv, beams, found.next_parent.view(-1), kv, moves, cache=cache)
        alive = found.next_parent.view(-1) >= 0
        wf.wf_kv_extend(scratch, kv, alive.int(), step)
        new = found.next_token.view(-1).clone()
        live = step.row >= 0
        vectors[step.slot[live]] = embed[new[step.row[live].long()].long()]
        state = torch.where(alive[:, None], state[found.next_parent.view(-1).clamp(min=0).long()] + embed[new.clamp(min=0).long()], 0.0)
        parents.append(found.next_parent.view(-1).clone())
        tokens.append(new)
        # A row that lost its last tokens, or that waits: its cache is no longer its hypothesis's.  Without scores its search
        # has no candidates, so the next reordering gives its blocks back.
        going &= ((moves.status | step.status) == 0).view(groups, beams).all(1)
        score.masked_fill_(~going.repeat_interleave(beams), -torch.inf)
        lasted += going.int()
    wf.wf_decode_status(scratch)

    # The best hypothesis of each search, from its last row back.
    texts, lasted = [], lasted.tolist()
    for g in range(groups):
        row, text = g * beams, []
        for parent, token in zip(reversed(parents[:lasted[g]]), reversed(tokens[:lasted[g]])):
            if row < 0:
                break
            text.append(int(token[row]))
            row = int(parent[row])
        texts.append(text[::-1] if admitted[g] else [])
    # What the block tables hold is what the running state summed.
    off = torch.where(going.repeat_interleave(beams)[:, None], cached_sums(vectors, kv) - state, 0.0)
    error = float(off.abs().max() / state.abs().max().clamp(min=1))
    blocks = int(kv.ends[0] - (kv.ends[1] - n_blocks))
    wf.wf_kv_reorder(scratch, kv, beams, torch.full((rows,), -1, dtype=torch.int32, device="cuda"), kv, moves)  # all end
    return dict(admitted=admitted, prompt=prompt, texts=texts, steps=lasted, score=score.view(groups, beams)[:, 0].tolist(), error=error,
                prompt_blocks=taken_at_first, blocks=blocks, n_blocks=n_blocks, left=int(kv.ends[1] - kv.ends[0]))


def main(window="mix", beams=4, steps=16):
    prob = wfgen.config(window).problem
    device, batch = first_batch(prob)
    got = decode(prob, device, batch, beams, steps)
    print(f"window {window}: device {device} runs activations {batch} of model {int(prob.model[batch[0]])} first")
    print(f"{got['n_blocks']} blocks of {BLOCK_TOKENS} tokens; {got['prompt_blocks']} for the prompts, "
          f"{got['blocks']} held after {steps} tokens on {beams} beams")
    for n, ok, length, text, score in zip(batch, got["admitted"], got["prompt"], got["texts"], got["score"]):
        end = f"log p {score:.2f}, {text[:8]} ..." if len(text) == steps else f"no block left after {len(text)} tokens, {text[:8]} ..."
        print(f"  activation {n}: {length} tokens, " + (end if ok else "waits for blocks"))
    if not got["error"] < 1e-4:
        raise SystemExit(f"what the block tables hold is off by {got['error']:.1e}")


if __name__ == "__main__":
    main(*(sys.argv[1:2] or ["mix"]), *(int(x) for x in sys.argv[2:4]))
