// The choice of tokens under rules, for its own entry point and for decoding.
#pragma once
#include "common.h"

struct ChooseArgs {
  const float* logits;
  int rows, vocab;
  long long stride;
  float* out;
  long long out_stride;
  int* token;
  long long token_stride;
  float2* best;  // [rows][pieces] the greatest logit of a piece and its token (as bits)
  float repetition, presence, frequency;
  const float* bias;
  long long bias_stride;
  const uint32_t* allowed;
  long long allowed_stride;
  const int *history, *history_len;
  long long history_stride;
  int tokens;
  const int *parents, *drafted;
  // decoding: tokens chosen so far, more[entry * more_stride + 0 .. more_n), and the one before them
  const int* more;
  int more_stride, more_n;
  const int* one;
  int pieces, row0;  // pieces of a row; first row of the launch
  int rule_row0, rule_rows;  // the rules' row of row r: r * rule_rows + rule_row0
};

int check_rules(const vlac_token_rules* r, int vocab);
size_t choose_workspace(int rows, int vocab);
ChooseArgs choose_args(const float* logits, int rows, int vocab, int64_t stride, const vlac_token_rules& r, float* out, int64_t out_stride,
                       int32_t* token, void* ws);
void launch_choose(ChooseArgs a, hipStream_t st);
