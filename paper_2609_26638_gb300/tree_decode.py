"""Decoding with drafted trees: several candidate continuations verified a step.

Text repeats itself (table cells, headers, formulas), so what followed the last few
tokens earlier in the sequence is a draft for free: ``lookup_tree`` gathers such
continuations into a tree.  One step runs all of its nodes through the decoder
(``StepDecoder.feed_trees``: ``gs_tree_attention``), chooses a token after each
(``gs_sample``), and keeps the path that was chosen (``gs_tree_accept``,
``gs_tree_commit``).  Each choice is the model's own draw, and a draft counts only where it is that
draw, so the text is distributed as without drafts; with temperature 0 it is the
greedy one.

    python -m paper_2609_26638_gb300.tree_decode --new 128 --bits 4
"""
from __future__ import annotations

import argparse
from typing import List, Optional, Sequence, Tuple

import torch

from . import gs
from .best_of_n import MAX_NODES, Sampler, Shape, StepDecoder, random_weights, uniform_table
from .cache import PAGE_TOKENS
from .qweight import quantize_decoder


def lookup_tree(history: Sequence[int], max_nodes: int, depth: int = 8, ngram: int = 3
                ) -> Tuple[List[int], List[int]]:
    """(tokens, parents) of a tree over what followed the last tokens before.

    The root is the history's last token.  Places where its last ``ngram`` (then fewer)
    tokens stood earlier are taken latest first, and up to ``depth`` tokens behind each
    are added, sharing what they have in common."""
    tokens, parents = [history[-1]], [-1]
    child = {}
    seen = set()
    for n in range(min(ngram, len(history)), 0, -1):
        key = list(history[-n:])
        for at in range(len(history) - n - 1, -1, -1):
            if at + n in seen or list(history[at: at + n]) != key:
                continue
            seen.add(at + n)
            node = 0
            for t in history[at + n: at + n + depth]:
                if (node, t) not in child:
                    if len(tokens) >= max_nodes:
                        return tokens, parents
                    child[node, t] = len(tokens)
                    tokens.append(t)
                    parents.append(node)
                node = child[node, t]
    return tokens, parents


def tree_decode(dec: StepDecoder, prompts: List[List[int]], new: int, *, max_nodes: int = 16, depth: int = 8,
                ngram: int = 3, uniforms: Optional[torch.Tensor] = None, seed: int = 0, eos: int = -1,
                draft=lookup_tree, **settings):
    """``new`` tokens after each prompt (fewer where ``eos`` comes, which is the last);
    (tokens, steps).

    uniforms: [prompts, prompt length + new] of the longest prompt, a number in [0, 1) for
    every position, or drawn from ``seed``; a position's token is drawn with the number of
    the position that it follows, whatever tree it was drafted in.  ``settings`` are
    ``Sampler``'s (temperature 0: the most likely token).  ``draft`` makes (tokens, parents)
    from (history, max_nodes, depth, ngram); its max_nodes is less than the call's where the
    context or the pool's free pages end, so a pool that holds the texts is enough."""
    b = len(prompts)
    if not b or any(not p for p in prompts) or new < 1 or not 1 <= max_nodes <= MAX_NODES:
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "no prompt, an empty one, new < 1 or max_nodes beyond 1 .. 64")
    longest = max(len(p) for p in prompts)
    if b * max_nodes > dec.max_rows or longest + new > dec.pool.table.max_ctx:
        raise gs.GsError(gs.GS_ERR_INVALID_ARG, "more nodes or tokens than the decoder was made for")
    if uniforms is None:
        uniforms = torch.rand(b, longest + new, generator=torch.Generator().manual_seed(seed))
    # the numbers of a step are picked on the host
    u = uniform_table(uniforms, b, longest + new, "cpu")
    sampler = Sampler(b * max_nodes, device=str(dec.device), **settings)
    text = [list(p) for p in prompts]
    left = [new] * b
    seqs: List[int] = []
    table = dec.pool.table
    steps = 0
    try:
        for p in prompts:                    # all but the last token, which is the first root
            seqs.append(dec.pool.open())
            for at in range(0, len(p) - 1, dec.max_rows):
                dec.feed([(seqs[-1], at, p[at: min(at + dec.max_rows, len(p) - 1)])])
        while any(left):
            live = [i for i in range(b) if left[i]]
            trees = []
            cached = [len(text[i]) - 1 for i in live]
            # pages beyond every root's: drafts may have these, and give back what is not kept
            spare = table.free_pages - sum(max(0, n // PAGE_TOKENS + 1 - len(table.pages(seqs[i])))
                                           for i, n in zip(live, cached))
            for i, n in zip(live, cached):
                have = max(len(table.pages(seqs[i])), n // PAGE_TOKENS + 1)
                room = min(max_nodes, table.max_ctx - n, (have + max(spare, 0)) * PAGE_TOKENS - n)
                tokens, parents = draft(text[i], room, min(depth, left[i] - 1), ngram)
                spare -= max(0, -(-(n + len(tokens)) // PAGE_TOKENS) - have)
                trees.append((seqs[i], n, tokens, parents))
            logits = dec.feed_trees(trees)
            nodes = logits.shape[1]
            number = torch.zeros(len(live), nodes)
            for row, i, (_, n, tokens, parents) in zip(number, live, trees):
                deep: List[int] = []
                for j, p in enumerate(parents):
                    deep.append(deep[p] + 1 if j else 0)
                row[: len(tokens)] = u[i, torch.tensor(deep) + n]
            with torch.cuda.stream(dec.stream):
                sampler.draw(logits.view(-1, logits.shape[2]), number.view(-1).to(dec.device), dec.stream)
                choice = sampler.token[: len(live) * nodes].view(len(live), nodes).clone()
            torch.cuda.current_stream(dec.device).wait_stream(dec.stream)
            for i, got in zip(live, dec.keep(trees, choice, most=[left[i] for i in live], eos=eos)):
                if not got or got[-1] < 0:
                    dec.check()
                    raise gs.GsError(gs.GS_ERR_DEVICE_CHECK, "no token could be chosen")
                text[i] += got
                dec.pool.truncate(seqs[i], len(text[i]) - 1)
                left[i] = 0 if got[-1] == eos else left[i] - len(got)
            steps += 1
        dec.check()
    finally:
        for q in seqs:
            dec.pool.close(q)
    return [t[len(p):] for t, p in zip(text, prompts)], steps


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompts", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=300)
    ap.add_argument("--new", type=int, default=64)
    ap.add_argument("--nodes", type=int, default=16)
    ap.add_argument("--bits", type=int, choices=(4, 16), default=16)
    ap.add_argument("--temperature", type=float, default=0.0)
    a = ap.parse_args()
    shape = Shape()
    ctx = a.prompt + a.new + MAX_NODES
    weights = random_weights(shape)
    if a.bits == 4:
        weights = quantize_decoder(weights)
    dec = StepDecoder(shape, weights, n_pages=a.prompts * (ctx // PAGE_TOKENS + 2), max_seqs=a.prompts,
                      max_ctx=ctx)
    g = torch.Generator().manual_seed(1)
    prompts = torch.randint(0, shape.vocab, (a.prompts, a.prompt), generator=g).tolist()
    texts, steps = tree_decode(dec, prompts, a.new, max_nodes=a.nodes, temperature=a.temperature)
    made = sum(len(t) for t in texts)
    print(f"{made} tokens of {a.prompts} prompts in {steps} steps, {made / (steps * a.prompts):.2f} a step and prompt")
    print(texts[0])


if __name__ == "__main__":
    main()
